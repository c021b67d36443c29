// Sums over rows, as partial sums side by side that a second launch adds in their order: the same bits every time.
#pragma once
#include <type_traits>
#include "elementwise.h"

namespace {

// Eight elements of a row as they lie in memory, so that rows on their way take few registers; the first n of them and zeros where there are
// fewer (all fetched at once, from the last one's place on: one behind the other, each would wait for memory by itself).
template <typename T> struct RawUnit;
template <> struct RawUnit<bf16_t> { ew_u4 w; };
template <> struct RawUnit<float> { ew_f4 w[2]; };
// PAST: past the caches, for what is read or written once and is larger than they are
template <bool PAST, typename V>
__device__ __forceinline__ V load_vector(const V* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool PAST = false>
__device__ __forceinline__ void load_whole(const bf16_t* p, RawUnit<bf16_t>& r) { r.w = load_vector<PAST>(reinterpret_cast<const ew_u4_any*>(p)); }
template <bool PAST = false>
__device__ __forceinline__ void load_whole(const float* p, RawUnit<float>& r) {
    r.w[0] = load_vector<PAST>(reinterpret_cast<const ew_f4_any*>(p));
    r.w[1] = load_vector<PAST>(reinterpret_cast<const ew_f4_any*>(p) + 1);
}
template <bool PAST = false>
__device__ __forceinline__ void load_raw(const bf16_t* p, int64_t n, RawUnit<bf16_t>& r) {
    if (n >= 8) {
        load_whole<PAST>(p, r);
    } else {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[i < n ? i : n - 1];
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = (2 * i < n ? e[2 * i] : 0u) | (2 * i + 1 < n ? e[2 * i + 1] << 16 : 0u);
    }
}
template <bool PAST = false>
__device__ __forceinline__ void load_raw(const float* p, int64_t n, RawUnit<float>& r) {
    if (n >= 8) {
        load_whole<PAST>(p, r);
    } else {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[i < n ? i : n - 1];
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = i < n ? e[i] : 0.0f;
    }
}
template <bool PAST>
__device__ __forceinline__ void store_unit(bf16_t* p, int64_t n, const float (&v)[8]) {
    if (PAST && n >= 8)
        __builtin_nontemporal_store(ew_u4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])},
                                    reinterpret_cast<ew_u4_any*>(p));
    else
        store_part<bf16_t, true>(p, n, v);
}
template <bool PAST>
__device__ __forceinline__ void store_unit(float* p, int64_t n, const float (&v)[8]) {
    if (PAST && n >= 8) {
        __builtin_nontemporal_store(ew_f4{v[0], v[1], v[2], v[3]}, reinterpret_cast<ew_f4_any*>(p));
        __builtin_nontemporal_store(ew_f4{v[4], v[5], v[6], v[7]}, reinterpret_cast<ew_f4_any*>(p) + 1);
    } else {
        store_part<float, true>(p, n, v);
    }
}
__device__ __forceinline__ void unpack(const RawUnit<bf16_t>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16lo_to_f32(r.w[i]);
        v[2 * i + 1] = bf16hi_to_f32(r.w[i]);
    }
}
__device__ __forceinline__ void unpack(const RawUnit<float>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = r.w[i >> 2][i & 3];
}
template <typename T>
__device__ __forceinline__ void load_unit(const T* p, int64_t n, float (&v)[8]) {
    RawUnit<T> r;
    load_raw(p, n, r);
    unpack(r, v);
}

// out[c] = sum over p of P[p, c] (parts rows of n).  Columns from `split` on go to `out2`.  A workgroup has 64 columns, its sixteen waves every
// sixteenth part.
__global__ void __launch_bounds__(1024)
k_join_sums(const float* __restrict__ P, int64_t parts, int64_t n, float* __restrict__ out, int64_t split, float* __restrict__ out2) {
    __shared__ float s_sum[16 * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = 64 * (int64_t)blockIdx.x + lane;
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

int launch_join(hipStream_t s, const float* P, int64_t parts, int64_t n, float* out, int64_t split, float* out2) {
    hipLaunchKernelGGL(k_join_sums, dim3((unsigned)ceil_div64(n, 64)), dim3(1024), 0, s, P, parts, n, out, split, out2);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
int launch_clear(hipStream_t s, float* p, int64_t n) {
    hipLaunchKernelGGL(k_clear, dim3((unsigned)ceil_div64(n, 256)), dim3(256), 0, s, p, n);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

}  // namespace
