"""attend_shared and reserve_shared without a device: what the binding refuses, and how the line of tiles is cut for the two passes."""
import os
import subprocess

import pytest
import torch

import paper_2504_20039_b200 as aj

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
B, N, HQ, HKV, D, PAGE, WIDTH, POOL = 3, 2, 8, 2, 64, 16, 20, 30
BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture(params=[False, True])
def recorder(request):
    from paper_2504_20039_b200.kv import KvHandle

    h = object.__new__(KvHandle)
    h._h, h.calls = None, []
    h._attend_shared = lambda *a: h.calls.append(a) or aj.AJ_OK
    h._take(-1, B, N, HQ, HKV, D, PAGE, aj.AJ_BF16, request.param)
    return h


def arguments():
    z = torch.zeros
    return dict(q=z(B * N, HQ * D, dtype=BF), k_pages=z(POOL, HKV, PAGE, D, dtype=BF), v_pages=z(POOL, HKV, PAGE, D, dtype=BF),
                shared_table=z(16, dtype=I32), shared=256, block_table=z(B, WIDTH, dtype=I32), seq_lens=z(B, dtype=I32),
                out=z(B * N, HQ * D, dtype=BF), B=B, n_q=N, scale=0.1, lse=z(B * N, HQ))


def test_the_binding_passes_on_what_fits(recorder):
    a = arguments()
    assert recorder.attend_shared(**a) == aj.AJ_OK
    got = recorder.calls[-1]
    assert got[5] == POOL and got[6] == a["shared_table"].data_ptr() and got[7] == 256 and got[9] == WIDTH and got[12:14] == (B, N)
    n = len(recorder.calls)
    z = torch.zeros
    for bad in ({"shared_table": z(15, dtype=I32)}, {"shared_table": z(16, dtype=torch.int64)}, {"shared_table": z(32, dtype=I32)[::2]}, {"q": z(B * N, HQ * D)},
                {"out": z(B * N, HQ * D)}, {"lse": z(B * N, HQ, dtype=BF)}, {"seq_lens": z(B, dtype=torch.int64)}, {"q_start": z(B + 1)},
                {"k_pages": z(POOL, PAGE, HKV, D, dtype=BF).transpose(1, 2)}):
        assert recorder.attend_shared(**(a | bad), check=False) == aj.AJ_ERR_INVALID_ARG, bad
    assert len(recorder.calls) == n


PROGRAM = r"""
#include <cstdio>
#include "aj_kv_line.cuh"
using namespace aj::kv;
int main() {
    int bad = 0;
    for (int G : {1, 4, 5, 128})
        for (int S : {128, 384, 4096})
            for (int nq : {1, 7, 31, 32, 33, 64, 65, 1000}) {
                const int tpt = 128 / G;
                View p;  // a chunk of the shared slots: every piece of the batch's tokens sees all of its tiles and no others
                p.Hkv = 1;
                p.shared = S;
                Seq chunk{0, nq, S};
                chunk.ahead = nq;
                chunk.first = S / 2 / 128 * 128;
                const Seqs a = pieces_of(chunk, tpt);
                int tokens = 0;
                for (int i = 0; i < a.n; i++) {
                    const Piece x = piece_of(p, a, i, tpt);
                    tokens += x.n_tok;
                    bad += x.units != (S - chunk.first) / 128 || x.first_tile != chunk.first / 128 || x.first != chunk.first || x.n_sink != 0;
                }
                bad += tokens != nq;
                View v;  // a sequence behind them: tiles from the prefix's end to the last token's
                v.Hkv = 1;
                v.shared = S;
                for (int before : {0, 1, 127, 128, 900}) {
                    Seq s{0, nq, S + before + nq};
                    s.first = S;
                    const Seqs b = pieces_of(s, tpt);
                    for (int i = 0; i < b.n; i++) {
                        const Piece x = piece_of(v, b, i, tpt);
                        const int last = S + before + x.ta + x.n_tok;  // behind the last slot that the piece sees
                        bad += x.first != S || x.first_tile != S / 128 || x.units != (last + 127) / 128 - S / 128 || x.n_sink != 0;
                    }
                }
            }
    printf("%d\n", bad);
}
"""


def test_line_of_the_two_passes(tmp_path):
    (tmp_path / "line.cu").write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2504_20039_b200", "csrc"),
                    "-o", str(tmp_path / "line"), str(tmp_path / "line.cu")], check=True)
    assert subprocess.run([str(tmp_path / "line")], check=True, capture_output=True, text=True).stdout.strip() == "0"
