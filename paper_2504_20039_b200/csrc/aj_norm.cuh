// Declarations of the norm with the residual's addition.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace aj {
namespace norm {

constexpr int MAX_D = 32768;

struct Args {
    const void *x = nullptr, *r = nullptr;
    const float *w = nullptr;
    void *r_out = nullptr, *out = nullptr;
    uint8_t *out8 = nullptr;
    float *scale8 = nullptr;
    long long x_stride = 0, r_stride = 0, r_out_stride = 0, out_stride = 0, out8_stride = 0;
    int rows = 0, d = 0;
    float eps = 0;
};

// Rows of 2049 to 8192 elements: half as many threads per row with twice the pieces each, or not.  In bf16 that pays where the rows pass one
// wave of the wider CTAs (6 of 256 threads on each of 148 SMs up to 4096 elements, 3 of 512 above); in f32 it never does, for a piece
// is 32 bytes there.  Measured with residual, to bf16 / f32, us, more threads and fewer: bf16, 4096 wide, 700 rows 6.2 and 6.4, 900 8.2 and 7.1,
// 2112 14.4 and 13.9; 8192 wide, 400 rows 7.2 and 7.1, 500 10.0 and 8.0, 2112 27.0 and 25.6, 8000 87 and 82 (to 8 bits 85 and 76); f32, 8192 wide, 500 rows
// 17.0 and 17.8, 700 19.9 and 23.9, 8000 163 and 170.
inline bool fewer_threads(int rows, int d, bool bf16) { return bf16 && rows > (d <= 4096 ? 6 : 3) * 148; }

// wide: every row on 16 bytes (8-bit rows on 8) and d a multiple of 8
cudaError_t launch(const Args &a, bool bf16, bool wide, cudaStream_t s);

}  // namespace norm
}  // namespace aj
