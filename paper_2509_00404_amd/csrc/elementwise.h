// Pieces of the kernels that stream rows: eight elements of a row at a time, bf16 or fp32.
#pragma once
#include "common.h"

namespace {

// n / d without the division: the high half of n * ceil(2^64 / d), exact while n d < 2^64 (d = 1 is marked by 0)
struct FastDiv {
    uint64_t magic;
    uint32_t d;
};
inline FastDiv fast_div(uint32_t d) { return {d > 1 ? ~0ull / d + 1 : 0ull, d}; }
__device__ __forceinline__ uint64_t div_by(const FastDiv& f, uint64_t n) { return f.magic ? __umul64hi(n, f.magic) : n; }

typedef uint32_t ew_u4 __attribute__((ext_vector_type(4)));
typedef uint32_t ew_u2 __attribute__((ext_vector_type(2)));
typedef float ew_f4 __attribute__((ext_vector_type(4)));

// (the shared conversion is for finite values; the packed instruction keeps NaN and infinities)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
    typedef float f2_t __attribute__((ext_vector_type(2)));
    const f2_t x = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf2_t));
}

// Eight elements from p, 16-byte aligned, or (ANY) aligned as the elements are: memory takes whole vectors at any address, at the price of
// the lines they straddle
typedef uint32_t ew_u4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float ew_f4_any __attribute__((ext_vector_type(4), aligned(4)));
template <bool ANY = false>
__device__ __forceinline__ void load_row(const bf16_t* p, float (&v)[8]) {
    ew_u4 a;
    if constexpr (ANY) a = *reinterpret_cast<const ew_u4_any*>(p);
    else a = *reinterpret_cast<const ew_u4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16lo_to_f32(a[i]);
        v[2 * i + 1] = bf16hi_to_f32(a[i]);
    }
}
template <bool ANY = false>
__device__ __forceinline__ void load_row(const float* p, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        ew_f4 a;
        if constexpr (ANY) a = reinterpret_cast<const ew_f4_any*>(p)[h];
        else a = reinterpret_cast<const ew_f4*>(p)[h];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * h + i] = a[i];
    }
}
template <bool ANY = false>
__device__ __forceinline__ void store_row(bf16_t* p, const float (&v)[8]) {
    const ew_u4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    if constexpr (ANY) *reinterpret_cast<ew_u4_any*>(p) = w;
    else *reinterpret_cast<ew_u4*>(p) = w;
}
template <bool ANY = false>
__device__ __forceinline__ void store_row(float* p, const float (&v)[8]) {
    const ew_f4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    if constexpr (ANY) {
        reinterpret_cast<ew_f4_any*>(p)[0] = a;
        reinterpret_cast<ew_f4_any*>(p)[1] = b;
    } else {
        reinterpret_cast<ew_f4*>(p)[0] = a;
        reinterpret_cast<ew_f4*>(p)[1] = b;
    }
}
__device__ __forceinline__ float load_one(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ void store_one(bf16_t* p, float v) { *p = (bf16_t)pack_bf16(v, 0.0f); }
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
// the first n of them, zeros for the rest
template <typename T, bool ANY>
__device__ __forceinline__ void load_part(const T* p, int64_t n, float (&v)[8]) {
    if (!ANY || n >= 8) {
        load_row<ANY>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? load_one(p + i) : 0.0f;
    }
}
template <typename T, bool ANY>
__device__ __forceinline__ void store_part(T* p, int64_t n, const float (&v)[8]) {
    if (!ANY || n >= 8) {
        store_row<ANY>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) store_one(p + i, v[i]);
    }
}

// Eight elements of a row as they lie in memory, so that rows on their way take few registers; the first n of them and zeros where there are
// fewer (all fetched at once, from the last one's place on: one behind the other, each would wait for memory by itself).
template <typename T> struct RawUnit;
template <> struct RawUnit<bf16_t> { ew_u4 w; };
template <> struct RawUnit<float> { ew_f4 w[2]; };
// PAST: past the caches, for what is read or written once and is larger than they are.  (Each load names its vector's type: a template's parameter deduced
// from it would lose the alignment that it lacks.)
template <bool PAST = false>
__device__ __forceinline__ void load_whole(const bf16_t* p, RawUnit<bf16_t>& r) {
    const ew_u4_any* at = reinterpret_cast<const ew_u4_any*>(p);
    if constexpr (PAST) r.w = __builtin_nontemporal_load(at);
    else r.w = *at;
}
template <bool PAST = false>
__device__ __forceinline__ void load_whole(const float* p, RawUnit<float>& r) {
    const ew_f4_any* at = reinterpret_cast<const ew_f4_any*>(p);
    if constexpr (PAST) {
        r.w[0] = __builtin_nontemporal_load(at);
        r.w[1] = __builtin_nontemporal_load(at + 1);
    } else {
        r.w[0] = at[0];
        r.w[1] = at[1];
    }
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
// The unit at column c of a row, without a condition of the lane's: where the row ends inside it, the whole vector at the row's end, whose first `back`
// elements are the unit's before it.  (A path of its own for that lane would make its whole wave wait for memory there.)  Rows of fewer than eight
// elements have one unit, back 0.  unpack(r, back, v): the unit's own elements, zeros behind them.
__device__ __forceinline__ int unit_back(int64_t c, int64_t cols) { return cols < 8 || c + 8 <= cols ? 0 : (int)(c + 8 - cols); }
template <bool PAST = false, typename T>
__device__ __forceinline__ void load_back(const T* row, int64_t c, int back, int64_t cols, RawUnit<T>& r) {
    if (cols >= 8) load_whole<PAST>(row + (c - back), r);
    else load_raw<PAST>(row + c, cols, r);
}
template <typename T>
__device__ __forceinline__ void unpack(const RawUnit<T>& r, int back, float (&v)[8]) {
    unpack(r, v);
    if (back) {
#pragma unroll
        for (int s = 4; s > 0; s >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = back & s ? (i + s < 8 ? v[i + s] : 0.0f) : v[i];
    }
}
template <typename T>
__device__ __forceinline__ void load_unit(const T* p, int64_t n, float (&v)[8]) {
    RawUnit<T> r;
    load_raw(p, n, r);
    unpack(r, v);
}

// HIP takes fewer than 2^32 threads along an axis of a grid
inline bool grid_fits(int64_t workgroups, int threads) { return workgroups <= 0xFFFFFFFFll / threads; }
// rows of `units` that a kernel takes a lane each, 256 a workgroup: they fit its grid, and fast_div is exact
inline int units_status(int64_t rows, int64_t units) {
    return units > (1 << 25) || rows > 0xFFFFFFFFll / 256 * 256 / units ? METIS_UNSUPPORTED : METIS_OK;
}
inline bool mat_ok(const metis_mat* m) { return m && m->ptr && (m->dtype == METIS_BF16 || m->dtype == METIS_F32); }
inline int64_t mat_size(const metis_mat* m) { return m->dtype == METIS_BF16 ? 2 : 4; }
inline bool mat_aligned16(const metis_mat* m) { return (uintptr_t)m->ptr % 16 == 0 && m->ld * mat_size(m) % 16 == 0; }

}  // namespace
