"""The line of tiles (csrc/aj_kv_line.cuh), compiled for the host: the kind for calls that share nothing cuts them as the general kind does."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "aj_kv_line.cuh"
using namespace aj::kv;
int main() {
    int seen = 0, bad = 0;
    for (int G : {1, 4, 5, 128})
        for (int L : {0, 1, 100, 128, 129, 1000, 5000})
            for (int nq : {0, 1, 17, 33, 64, 65, 200, 1000})
                for (int window : {0, 1, 100, 1024})
                    for (int sinks : {0, 4, 300}) {
                        const int tpt = 128 / G;
                        View v;
                        v.Hkv = 1;
                        v.window = window;
                        v.sinks = sinks;
                        const Seqs q = pieces_of(Seq{0, nq, L}, tpt);
                        bad += units_of<false>(v, q, tpt, 0, 1) != units_of<true>(v, q, tpt, 0, 1);
                        for (int i = 0; i < q.n; i++, seen++) {
                            const Piece a = piece_of<false>(v, q, i, tpt), b = piece_of<true>(v, q, i, tpt);
                            bad += a.ta != b.ta || a.n_tok != b.n_tok || a.tok0 != b.tok0 || a.first != b.first || a.n_sink != b.n_sink ||
                                   a.first_tile != b.first_tile || a.units != b.units || a.places != b.places;
                            for (int unit = -CHARGE; unit < a.units; unit++)
                                for (int left : {1, 3, 1000}) {
                                    Line c;
                                    c.unit = unit;
                                    c.q = q;
                                    c.p = a;
                                    const Part x = part_of<false>(c, left), y = part_of<true>(c, left);
                                    bad += x.line != y.line || x.first != y.first || x.n != y.n;
                                }
                        }
                    }
    printf("%d %d\n", seen, bad);
}
"""


def test_both_kinds_cut_alike(tmp_path):
    (tmp_path / "line.cu").write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2504_20039_b200", "csrc"),
                    "-o", str(tmp_path / "line"), str(tmp_path / "line.cu")], check=True)
    seen, bad = map(int, subprocess.run([str(tmp_path / "line")], check=True, capture_output=True, text=True).stdout.split())
    assert seen > 1000 and bad == 0
