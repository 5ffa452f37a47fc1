"""The line of tiles that the tcgen05 attention cuts into equal shares (csrc/aj_kv_line.cuh), compiled for the host: its
length against plain arithmetic, at sizes that no test could run among them."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "aj_kv_line.cuh"
using namespace aj::kv;
int main(int, char **a) {
    const int nq = atoi(a[1]), L = atoi(a[2]), G = atoi(a[3]), Hkv = atoi(a[4]), window = atoi(a[5]), sinks = atoi(a[6]);
    View v;
    v.Hkv = Hkv;
    v.window = window;
    v.sinks = sinks;
    const int tpt = 128 / G;
    const Seqs q = pieces_of(Seq{0, nq, L}, tpt);
    long long lanes = 0;  // as a warp adds them up
    for (int i = 0; i < 32; i++) lanes += units_of(v, q, tpt, i, 32);
    printf("%lld %lld", units_of(v, q, tpt, 0, 1) * Hkv, lanes * Hkv);
    for (int x = -9; x <= 9; x++) printf(" %d", floor_div(x, 4));
    printf("\n");
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("line")
    (d / "line.cu").write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(ROOT, "paper_2504_20039_b200", "csrc"),
                    "-o", str(d / "line"), str(d / "line.cu")], check=True)
    return str(d / "line")


def places(nq, L, G, Hkv, window, sinks):
    """Tiles of 128 slots with a visible slot, or the one that an item always has, and two places for each item."""
    per_tile = 128 // G
    n = -(-nq // (2 * per_tile))
    total = 0
    for i in range(n):
        t0 = i * (nq // n) + min(i, nq % n)
        t1 = t0 + nq // n + (i < nq % n)
        lo, hi = L - nq + t0, max(0, L - nq + t1)  # slot of the first token, slot behind the last
        first = min(max(0, lo - window + 1), hi) if window else 0
        tiles = -(-hi // 128) - first // 128
        tiles += min(-(-min(sinks, first) // 128), first // 128)
        total += 2 + max(1, tiles)
    return total * Hkv


@pytest.mark.parametrize("nq,L,G,Hkv,window,sinks", [
    (1, 1, 1, 1, 0, 0), (17, 400, 4, 8, 0, 0), (33, 8000, 4, 8, 0, 0), (65, 64, 8, 2, 0, 0), (4096, 4096, 4, 8, 1024, 4), (700, 5000, 7, 3, 129, 300),
    (1 << 20, 1 << 20, 4, 8, 0, 0),
    (1 << 20, 1 << 20, 16, 8, 0, 0),     # 2,148,794,368 places: above 2^31
    (1 << 20, 1 << 20, 4, 32, 0, 0),     # the same with more key heads
    (1 << 18, 1 << 20, 128, 8, 0, 0),
])
def test_length_of_the_line(program, nq, L, G, Hkv, window, sinks):
    out = [int(x) for x in subprocess.run([program, *map(str, (nq, L, G, Hkv, window, sinks))], check=True, capture_output=True, text=True).stdout.split()]
    want = places(nq, L, G, Hkv, window, sinks)
    assert out[:2] == [want, want]
    assert out[2:] == [x // 4 for x in range(-9, 10)]
    if (nq, G) == (1 << 20, 16):
        assert want == 2148794368
