"""How aj_score_tokens cuts its work (csrc/aj_score_umma.cu), compiled for the host: the ring of stages over every number of rows, tile, width
and type, against the shared memory of a block."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <climits>
#include <cstdio>
#include "aj_score_umma.cu"
using namespace aj::score;
int main() {
    int torn = 0;  // calls whose groups do not cover the rows, in order, in as few groups as there can be
    for (int group : {1, 17, 255, 256, 1024, 2560})
        for (int rows : {1, 2, 255, 256, 257, 2560, 2561, 5200, 100000, INT_MAX - 900000, INT_MAX - 3000, INT_MAX - 1, INT_MAX}) {
            if (group < 256 && rows > group) continue;  // (a handle for so few rows)
            const long long each = rows_each(rows, group);
            long long n = 0, r0 = 0;
            for (; r0 < rows; r0 += each) n++;
            torn += each < 1 || each > group || n > ((long long)rows + group - 1) / group || (n > 1 && each % 256 != 0);
        }
    printf("%d\n", torn);
    for (int V : {3000, 8000, 12000, 16000, 32000, 50257, 100352, 128256, 151936, 200064, 256000}) printf("%d ", one_sm_tile(V, 148));
    // a tile of up to 96 entries costs as much as one of 96, a wider one in proportion
    int dear = 0, many = 0;
    for (int V = 1; V <= MAX_V; V += V < 400000 ? 1 : 997) {
        auto cost = [&](int t) { return ((V + t - 1) / t + 147) / 148 * (t > 96 ? t : 96); };
        int least = cost(256);
        for (int t = 32; t < 256; t += 32)
            if ((V + t - 1) / t <= MAX_TILES && cost(t) < least) least = cost(t);
        const int t = one_sm_tile(V, 148);
        dear += cost(t) > 1.15 * least;
        many += t % 32 != 0 || t > 256 || (V + t - 1) / t > MAX_TILES;
    }
    printf("%d %d\n", dear, many);
    const int block = 227 * 1024;  // shared memory of a block
    long long seen = 0, past = 0, thin = 0;
    for (int dtype : {(int)BF16, (int)E4M3})
        for (int d : {16, 64, 128, 192, 256, 1792, 2048, 4096, 4160, 65536})
            for (int tile = 32; tile <= 256; tile += 32)
                for (int rows = 1; rows <= 300; rows++) {
                    const Plan p = plan_umma(rows, d, 50257, dtype, tile, 148, 74);
                    const int entries = p.pair ? p.tile / 2 : p.tile, sub = (p.box_rows + entries) * 128;  // bytes of a k-block
                    seen++;
                    thin += p.stages < 3;
                    for (int s = 0; s < p.stages; s++)
                        for (int j = 0; j < p.kps; j++) {
                            const int at = (s * p.kps + j) * sub;
                            // copies: box_rows, then the entries; products: 128 rows from the k-block's start, its entries
                            const bool bad = at + sub > RING || at + 128 * 128 > block || SMEM > block;
                            if (bad && past++ == 0) printf("dtype %d d %d tile %d rows %d: k-block %d of stage %d of %d at %d\n", dtype, d, tile, rows, j, s, p.stages, at);
                        }
                }
    printf("%lld %lld %lld\n", seen, past, thin);
}
"""


@pytest.fixture(scope="module")
def output(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cu").write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2504_20039_b200", "csrc"),
                    "-o", str(d / "plan"), str(d / "plan.cu")], check=True)
    return subprocess.run([str(d / "plan")], check=True, capture_output=True, text=True).stdout


def test_groups_of_rows(output):
    assert output.splitlines()[0] == "0"


def test_widths_of_tiles(output):
    """Widths that measured within 6 % of the best one of their head (1 to 128 rows, d from 256 to 8192, both types), on 148 SMs."""
    *tiles, dear, many = map(int, output.splitlines()[1].split())
    good = [(32,), (64, 96), (96, 128), (128, 160), (128, 224), (192,), (160, 192, 256), (224,), (160, 224), (224, 256), (160, 224, 256)]
    assert all(t in g for t, g in zip(tiles, good, strict=True)), tiles
    assert dear == many == 0


def test_nothing_past_the_blocks_shared_memory(output):
    seen, past, thin = map(int, output.splitlines()[-1].split())
    assert seen == 2 * 10 * 8 * 300
    assert past == 0, output
    assert thin == 0
