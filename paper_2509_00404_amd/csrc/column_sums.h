// Sums over rows, as partial sums side by side that a second launch adds in their order: the same bits every time.
#pragma once
#include <type_traits>
#include "elementwise.h"

namespace {

// out[c] = sum over p of P[p, c] (parts rows of n), c from `first` on.  Columns from `split` on go to `out2`.  A workgroup has 64 columns, its sixteen waves
// every sixteenth part.
__global__ void __launch_bounds__(1024)
k_join_sums(const float* __restrict__ P, int64_t parts, int64_t n, float* __restrict__ out, int64_t split, float* __restrict__ out2, int64_t first) {
    __shared__ float s_sum[16 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = first + 64 * (int64_t)blockIdx.x + lane;
    float sum = 0.0f;
    if (c < n) {
#pragma unroll 8
        for (int64_t p = wave; p < parts; p += 16) sum += P[p * n + c];
    }
    s_sum[64 * wave + lane] = sum;
    __syncthreads();
    if (wave > 0 || c >= n) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += s_sum[64 * w + lane];
    if (c < split) { if (out) out[c] = sum; }
    else if (out2) out2[c - split] = sum;
}
__global__ void __launch_bounds__(256)
k_clear(float* __restrict__ p, int64_t n) {
    const int64_t i = 256 * (int64_t)blockIdx.x + threadIdx.x;
    if (i < n) p[i] = 0.0f;
}

// Column sums of a workgroup of WAVES waves whose lanes have eight columns each, lane % W of W units, and some of the rows: added over the lanes of a
// wave, then over the waves, in the same order every time; out[8 W * strip ...].  lds: 8 W WAVES floats that nobody else uses meanwhile.
template <int WAVES, int W>
__device__ __forceinline__ void group_columns(float (&sum)[8], float* lds, float* __restrict__ out, int64_t strip, int64_t cols) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = W; d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += __shfl_xor(sum[i], d);
    if (lane < W) {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[8 * W * wave + 8 * lane + i] = sum[i];
    }
    __syncthreads();
    const int64_t c = 8 * W * strip + lane;
    if (wave == 0 && lane < 8 * W && c < cols) {
        float s = lds[lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += lds[8 * W * w + lane];
        out[c] = s;
    }
}

// Strips of a row's lines in turn on one XCD (workgroups go round the eight): strip of workgroup `block` of `strips`.
__device__ __forceinline__ uint32_t xcd_strip(uint32_t block, uint32_t strips) {
    const uint32_t x = block % 8, each = strips / 8, more = strips % 8;
    return x * each + (x < more ? x : more) + block / 8;
}

int launch_join(hipStream_t s, const float* P, int64_t parts, int64_t n, float* out, int64_t split, float* out2) {
    // (1024 threads for 64 columns: from 2^28 columns on, or 2^27 with two sums each, a launch of them all would have 2^32)
    const int64_t most = 1ll << 27;
    for (int64_t first = 0; first < n; first += most) {
        const int64_t columns = n - first < most ? n - first : most;
        hipLaunchKernelGGL(k_join_sums, dim3((unsigned)ceil_div64(columns, 64)), dim3(1024), 0, s, P, parts, n, out, split, out2, first);
        METIS_LAUNCH_CHECK();
    }
    return METIS_OK;
}
int launch_clear(hipStream_t s, float* p, int64_t n) {
    hipLaunchKernelGGL(k_clear, dim3((unsigned)ceil_div64(n, 256)), dim3(256), 0, s, p, n);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

}  // namespace
