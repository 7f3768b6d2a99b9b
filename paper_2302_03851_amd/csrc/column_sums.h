// Sums over the parts that work-groups left: out_s[c] = sum over p of
// part[p][s][c], for one or two arrays s, in an order that the parts' number
// fixes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace edb {
namespace {

// 16 columns by 64 shares of the parts a work-group: each thread adds up every
// 64th part of a column, then the shares are added by halves.
constexpr int kJoinCols = 16, kJoinShares = 64;

__global__ __launch_bounds__(kJoinCols* kJoinShares) void join_columns_kernel(const float* part, int parts, int width, int arrays,
                                                                             float* out0, float* out1) {
    __shared__ float held[kJoinShares][kJoinCols + 1];
    const int col = threadIdx.x % kJoinCols, share = threadIdx.x / kJoinCols, c = blockIdx.x * kJoinCols + col;
    float* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    float sum = 0.f;
    if (c < width) {
        const float* p = part + (int64_t)blockIdx.y * width + c;
#pragma unroll 4
        for (int i = share; i < parts; i += kJoinShares) sum += p[(int64_t)i * arrays * width];
    }
    held[share][col] = sum;
    for (int d = kJoinShares / 2; d; d >>= 1) {
        __syncthreads();
        if (share < d) held[share][col] += held[share + d][col];
    }
    if (share == 0 && c < width) out[c] = held[0][col];
}

// Either result may be NULL.  No parts: zeros.
inline void join_columns(const float* part, int parts, int width, int arrays, float* out0, float* out1, hipStream_t st) {
    join_columns_kernel<<<dim3((unsigned)((width + kJoinCols - 1) / kJoinCols), (unsigned)arrays), kJoinCols * kJoinShares, 0, st>>>(
        part, parts, width, arrays, out0, out1);
}

}  // namespace
}  // namespace edb
