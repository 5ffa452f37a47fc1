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

// wide: every row on 16 bytes (8-bit rows on 8) and d a multiple of 8
cudaError_t launch(const Args &a, bool bf16, bool wide, cudaStream_t s);

}  // namespace norm
}  // namespace aj
