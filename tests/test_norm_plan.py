"""Which shape of the norm's kernel a call gets (csrc/aj_norm.cuh), compiled for the host, against the faster one of both as measured."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "aj_norm.cuh"
int main() {
    for (int bf16 : {1, 0})
        for (int d : {2056, 4096, 5120, 8192})
            for (int rows : {1, 200, 500, 700, 900, 2112, 8000}) printf("%d %d %d %d\n", bf16, d, rows, (int)aj::norm::fewer_threads(rows, d, bf16));
}
"""

# us with more threads per row and with fewer, [rows 1, 200, 500, 700, 900, 2112, 8000]: with residual, to the storage type
MEASURED = {
    (1, 2056): [(2.30, 2.56), (2.79, 3.13), (3.13, 3.39), (3.67, 3.93), (5.97, 4.86), (10.15, 9.21), (30.10, 27.97)],
    (1, 4096): [(2.56, 2.99), (2.87, 3.47), (5.19, 5.55), (6.23, 6.40), (8.19, 7.08), (14.42, 13.91), (42.84, 42.58)],
    (1, 5120): [(2.82, 2.99), (3.41, 3.50), (8.02, 6.23), (8.96, 9.39), (10.92, 10.07), (20.65, 18.94), (69.25, 59.31)],
    (1, 8192): [(2.88, 3.39), (4.78, 4.85), (9.98, 8.02), (11.60, 12.20), (13.74, 13.65), (26.97, 25.60), (87.34, 81.83)],
    (0, 2056): [(2.62, 3.05), (3.41, 3.50), (5.72, 6.06), (6.65, 7.08), (8.35, 8.28), (14.25, 15.10), (43.09, 43.43)],
    (0, 4096): [(2.90, 3.41), (5.03, 5.12), (9.37, 10.24), (11.18, 12.29), (14.65, 14.67), (25.69, 28.76), (81.54, 85.46)],
    (0, 5120): [(3.58, 3.33), (6.74, 7.00), (11.26, 12.12), (13.40, 16.12), (16.47, 18.52), (30.98, 35.58), (104.49, 105.86)],
    (0, 8192): [(4.67, 4.09), (9.81, 9.90), (16.98, 17.83), (19.88, 23.88), (24.92, 26.53), (47.74, 54.10), (163.41, 169.89)],
}


def test_the_faster_shape(tmp_path):
    (tmp_path / "norm.cu").write_text(PROGRAM)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-I", os.path.join(ROOT, "paper_2504_20039_b200", "csrc"), "-o", str(tmp_path / "norm"), str(tmp_path / "norm.cu")], check=True)
    lines = subprocess.run([str(tmp_path / "norm")], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    at = {(bf16, d): iter(times) for (bf16, d), times in MEASURED.items()}
    for line in lines:
        bf16, d, rows, fewer = map(int, line.split())
        times = next(at[bf16, d])
        assert times[fewer] <= (1.15 if rows == 1 else 1.06) * min(times), line  # (one row: 0.6 us between the shapes)
