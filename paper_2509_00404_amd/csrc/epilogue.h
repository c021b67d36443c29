// What a product's outputs go through on their way to memory -- bias, activation, dropout, residual -- eight neighbouring elements of a row at a
// time, and the pieces of it that other kernels share: the activations with their slopes, and the dropout mask.
#pragma once
#include <type_traits>
#include "mx_tile.h"
#include "elementwise.h"

namespace {

// ---- dropout masks ----
// Element (i, j) has number j % 8 of the eight 16-bit numbers of Philox block (j / 8, i, MASK_TAG, step) under `seed`, low halves first: a
// lane's eight elements cost one block, whatever the rows' stride, and the sixteen bits set p in steps of 2^-16 (32 bits an element would be
// two blocks: the generator, not memory, would then bound the plain dropout).  The third counter word keeps the masks apart from the library's
// other draws under the same seed.
#define MASK_TAG 16u
struct MaskKey {
    uint64_t seed;
    const int64_t* step;                      // device memory, or null: 0
    uint32_t dropped;                         // numbers below this one are dropped; 0: no dropout
    float keep;                               // factor of the others
};
inline int mask_status(const metis_dropout_mask* m) {
    if (!m) return METIS_OK;
    if (!(m->p >= 0.0) || !(m->p < 1.0) || (uintptr_t)m->step % 8) return METIS_INVALID_ARG;
    return (uint32_t)(65536.0 * m->p + 0.5) < 65536u ? METIS_OK : METIS_INVALID_ARG;
}
inline MaskKey mask_key(const metis_dropout_mask* m) {
    if (!m) return {0, nullptr, 0, 1.0f};
    const uint32_t t = (uint32_t)(65536.0 * m->p + 0.5);
    return {m->seed, m->step, t, (float)(65536.0 / (65536.0 - t))};
}
__device__ __forceinline__ uint32_t mask_step(const MaskKey& k) { return k.dropped && k.step ? (uint32_t)*k.step : 0u; }
// The block of unit j / 8 of row i.  A round is two products and two three-input xors (the plain rounds compile to twice the xors).
__device__ __forceinline__ u32x4 mask_block(const MaskKey& key, uint32_t step, uint32_t unit, uint32_t row) {
    const uint32_t M0 = 0xD2511F53u, M1 = 0xCD9E8D57u, W0 = 0x9E3779B9u, W1 = 0xBB67AE85u;
    const uint32_t k0 = (uint32_t)key.seed, k1 = (uint32_t)(key.seed >> 32);
    uint32_t x = unit, y = row, z = MASK_TAG, w = step;
#pragma unroll
    for (uint32_t r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)M0 * x, p1 = (uint64_t)M1 * z;
        x = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), y, k0 + r * W0, 0x96);
        z = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), w, k1 + r * W1, 0x96);
        y = (uint32_t)p1;
        w = (uint32_t)p0;
    }
    return {x, y, z, w};
}
// v = kept ? keep v : 0 (dropped elements are 0 whatever they were)
__device__ __forceinline__ void mask_apply(const MaskKey& key, uint32_t step, uint32_t unit, uint32_t row, float (&v)[8]) {
    const u32x4 b = mask_block(key, step, unit, row);
    const uint32_t w[4] = {b.x, b.y, b.z, b.w}, high = key.dropped << 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (w[i] & 0xFFFFu) >= key.dropped ? v[2 * i] * key.keep : 0.0f;
        v[2 * i + 1] = w[i] >= high ? v[2 * i + 1] * key.keep : 0.0f;
    }
}

// ---- activations ----
// FAST (bf16 results): the hardware's exponential and reciprocal, one unit in the last place of fp32 each, as against a rounding to 8 bits.
__device__ __forceinline__ float act_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
template <bool FAST>
__device__ __forceinline__ float logistic(float x) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + act_exp(-x));
    else return 1.0f / (1.0f + expf(-x));
}
// Upper tail of the normal distribution at a = |z|: exp(-a^2 / 2) R(a), R(a) = erfcx(a / sqrt 2) / 2.  R is smooth and falls from 1/2 as 1 / a; as a
// polynomial in t = 1 / (1 + c a), fitted for the least relative error for a <= 14 (beyond, the exponential is below fp32's range), it is within 1.4e-5
// of its value with degree 5, for results of 8 bits, and within 6e-7 with degree 8 (FINE), for gradients whose sums are fp32; the exponential's rounded argument
// adds up to 2e-5 of what little is left at a = 14, 2e-6 at 5.
template <bool FINE>
__device__ __forceinline__ float normal_tail(float a, float& bell) {
    bell = __builtin_amdgcn_exp2f(a * a * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(fmaf(FINE ? 0.23f : 0.36f, a, 1.0f));
    float p;
    if constexpr (FINE) {
        p = fmaf(-0.0784672665f, t, 0.290412933f);
        p = fmaf(p, t, -0.278125001f);
        p = fmaf(p, t, 0.301470511f);
        p = fmaf(p, t, -0.0329185951f);
        p = fmaf(p, t, 0.119513366f);
        p = fmaf(p, t, 0.0857630961f);
        p = fmaf(p, t, 0.0923784315f);
        p = fmaf(p, t, -2.77609611e-05f);
    } else {
        p = fmaf(-0.0985156898f, t, 0.254387546f);
        p = fmaf(p, t, 0.0351163301f);
        p = fmaf(p, t, 0.168695796f);
        p = fmaf(p, t, 0.140124069f);
        p = fmaf(p, t, 0.000191289818f);
    }
    return bell * p;
}
#define GELU_C 0.797884561f                       // sqrt(2 / pi)
template <bool FAST>
__device__ __forceinline__ float act_value(int act, float z) {
    switch (act) {
        case METIS_ACT_RELU: return z < 0.0f ? 0.0f : z;                          // (NaN stays)
        case METIS_ACT_GELU:
            if constexpr (FAST) {
                float bell;
                const float q = normal_tail<false>(fabsf(z), bell);
                return z * (z < 0.0f ? q : 1.0f - q);
            } else {
                return 0.5f * z * erfcf(z * -0.707106781f);
            }
        case METIS_ACT_GELU_TANH: return z * logistic<FAST>(2.0f * GELU_C * z * fmaf(0.044715f * z, z, 1.0f));
        case METIS_ACT_SILU: return z * logistic<FAST>(z);
        default: return z;
    }
}
// s = sigmoid(x) and s (1 - s), the latter from exp(-|x|) so that it keeps its relative accuracy where s is near 1
template <bool FAST>
__device__ __forceinline__ float logistic_slope(float x, float& s) {
    float e, d;
    if constexpr (FAST) {
        e = act_exp(-fabsf(x));
        d = __builtin_amdgcn_rcpf(1.0f + e);
    } else {
        e = expf(-fabsf(x));
        d = 1.0f / (1.0f + e);
    }
    s = x < 0.0f ? e * d : d;
    return e * d * d;
}
template <bool FAST>
__device__ __forceinline__ float act_slope(int act, float z) {
    switch (act) {
        case METIS_ACT_RELU: return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
        case METIS_ACT_GELU:
            if constexpr (FAST) {
                float bell;
                const float q = normal_tail<true>(fabsf(z), bell);
                return fmaf(0.5f * GELU_C * z, bell, z < 0.0f ? q : 1.0f - q);
            } else {
                return fmaf(0.5f * GELU_C * z, expf(-0.5f * z * z), 0.5f * erfcf(z * -0.707106781f));
            }
        case METIS_ACT_GELU_TANH: {
            // (beyond |z| = 20 the slope is 0 or 1, and z^2 would overflow beyond 1e19)
            float s;
            const float c = fminf(fmaxf(z, -20.0f), 20.0f), d = logistic_slope<FAST>(2.0f * GELU_C * c * fmaf(0.044715f * c, c, 1.0f), s);
            return z != z ? z : fmaf(c * d * (2.0f * GELU_C), fmaf(3.0f * 0.044715f * c, c, 1.0f), s);
        }
        case METIS_ACT_SILU: {
            float s;
            const float d = logistic_slope<FAST>(z, s);
            return fmaf(z, d, s);
        }
        default: return 1.0f;
    }
}
inline bool act_ok(int act) { return act >= METIS_ACT_NONE && act <= METIS_ACT_SILU; }

// ---- the epilogue ----
struct MxPlain {};                                // a product's outputs as they are
struct MxParts {                                  // fp32 sums of a part of the contraction, `units` of it, one part's behind the other's
    float* sums;
    int64_t ld, stride;
    int units;
};
// ACT: the activation, or ACT_ANY, `act`
#define ACT_ANY (-1)
template <typename T, int ACT = ACT_ANY>
struct MxFinish {
    typedef T type;
    T* y;                                         // (residual may be y: no restrict)
    int64_t ldy;
    const float* bias;                            // null: none
    T* pre;                                       // null: not wanted
    int64_t ldp;
    const T* residual;                            // null: none
    int64_t ldr;
    MaskKey mask;
    int act;
    bool narrow;                                  // rows near each other are within 2^31 bytes
    bool lines;                                   // rows of y and pre start at whole lines
};
// the activation and the mask of S units of eight elements, columns c .. c + 7, row(s)
template <int S, typename T, int ACT, typename F>
__device__ __forceinline__ void finish_values(const MxFinish<T, ACT>& f, uint32_t step, int64_t c, const F& row, float (&v)[S][8]) {
    auto all = [&](auto a) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[s][i] = act_value<sizeof(T) == 2>(decltype(a)::value, v[s][i]);
    };
    switch (ACT != ACT_ANY ? ACT : f.act) {           // uniform
        case METIS_ACT_RELU: all(std::integral_constant<int, METIS_ACT_RELU>{}); break;
        case METIS_ACT_GELU: all(std::integral_constant<int, METIS_ACT_GELU>{}); break;
        case METIS_ACT_GELU_TANH: all(std::integral_constant<int, METIS_ACT_GELU_TANH>{}); break;
        case METIS_ACT_SILU: all(std::integral_constant<int, METIS_ACT_SILU>{}); break;
        default: break;
    }
    if (f.mask.dropped) {
#pragma unroll
        for (int s = 0; s < S; ++s) mask_apply(f.mask, step, (uint32_t)(c >> 3), row(s), v[s]);
    }
}
// What the epilogue reads for a unit of eight elements (row r, columns from c on, a multiple of 8), fetched ahead of its use.
template <typename T>
struct UnitInputs {
    RawUnit<float> bias;
    RawUnit<T> residual;
    int back;
};
template <typename T, int ACT>
__device__ __forceinline__ void finish_inputs(const MxFinish<T, ACT>& f, int64_t r, int64_t c, int64_t N, UnitInputs<T>& in) {
    in.back = unit_back(c, N);
    in.bias = RawUnit<float>{};
    if (f.bias) load_back(f.bias, c, in.back, N, in.bias);
    if (f.residual) load_back(f.residual + r * f.ldr, c, in.back, N, in.residual);
}
// One element of each, where there are no registers for all: finish_inputs then finds their lines in the cache.  finish_near_by: after the product.
template <typename T>
struct UnitNear {
    float bias;
    T residual;
};
template <typename T, int ACT>
__device__ __forceinline__ UnitNear<T> finish_near(const MxFinish<T, ACT>& f, int64_t r, int64_t c, int64_t N) {
    const int64_t at = c < N ? c : N - 1;
    UnitNear<T> near = {};
    if (f.bias) near.bias = f.bias[at];
    if (f.residual) near.residual = f.residual[r * f.ldr + at];
    return near;
}
template <typename T>
__device__ __forceinline__ void finish_near_by(const UnitNear<T>& near) {
    asm volatile("" :: "v"(near.bias), "v"(near.residual));
}
// step: mask_step(f.mask)
template <typename T, int ACT>
__device__ __forceinline__ void finish_unit(const MxFinish<T, ACT>& f, uint32_t step, int64_t r, int64_t c, int64_t N, const UnitInputs<T>& in,
                                            const float (&v)[8]) {
    float b[8], one[1][8];
    unpack(in.bias, in.back, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) one[0][i] = v[i] + b[i];
    if (f.pre) store_part<T, true>(f.pre + r * f.ldp + c, N - c, one[0]);
    finish_values<1>(f, step, c, [&](int) __attribute__((always_inline)) { return (uint32_t)r; }, one);
    if (f.residual) {
        float res[8];
        unpack(in.residual, in.back, res);
#pragma unroll
        for (int i = 0; i < 8; ++i) one[0][i] += res[i];
    }
    store_part<T, true>(f.y + r * f.ldy + c, N - c, one[0]);
}
template <typename T, int ACT>
__device__ __forceinline__ void finish_bias(const MxFinish<T, ACT>& f, int64_t c, int64_t N, float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if (f.bias && c < N) load_unit(f.bias + c, N - c, b);
}

// an element near row r0, which is uniform, by a 32-bit offset
template <typename T>
__device__ __forceinline__ T* narrow_at(T* p, int64_t ld, int64_t r0, uint32_t low, uint32_t c) {
    return in_global(reinterpret_cast<T*>((uintptr_t)(p + r0 * ld) + (low * (uint32_t)ld + c) * (uint32_t)sizeof(T)));
}
// What is computed from the epilogue's arguments is computed where it is used: the empty asm hides that they are the same for every tile of a
// persistent workgroup (kept over its products, the strides' multiples alone took the scalar registers, and vector registers after them).  The pointers are
// global memory's again behind it: flat instructions took 8192 x 8192 x 1024 in fp32 with a residual 149 us, these 132.
template <typename T, int ACT>
__device__ __forceinline__ MxFinish<T, ACT> finish_afresh(MxFinish<T, ACT> f) {
    asm volatile("" : "+s"(f.y), "+s"(f.ldy), "+s"(f.bias), "+s"(f.pre), "+s"(f.ldp), "+s"(f.residual), "+s"(f.ldr));
    asm volatile("" : "+s"(f.mask.seed), "+s"(f.mask.step), "+s"(f.mask.dropped), "+s"(f.mask.keep), "+s"(f.act));
    f.y = in_global(f.y);
    f.bias = in_global(f.bias);
    f.pre = in_global(f.pre);
    f.residual = in_global(f.residual);
    f.mask.step = in_global(f.mask.step);
    return f;
}
// A wave's TM x TN accumulator tiles, transposed (a lane holds runs of four columns of one row), through the epilogue.  32 rows of its columns at
// a time are staged at sm as fp32 (mx_wave_rows<float, TN> bytes), and a lane takes eight neighbouring columns of some of them: one block of the
// mask's numbers, and 16 bytes of every bf16 operand.  The residual's next 32 rows are on their way meanwhile.
template <bool WHOLE, bool PAST, int TM, int TN, typename T, int ACT>
__device__ __forceinline__ void mx_finish_rows(const float16_t (&acc)[TM][TN], uint8_t* sm, const MxFinish<T, ACT>& f, int64_t m0, int64_t n0, int64_t M,
                                               int64_t N, int lane) {
    constexpr int LROW = 32 * TN * 4 + 16, UNITS = 4 * TN, ROWS = 64 / UNITS, S = 32 / ROWS;
    const int li = lane & 31, half = lane >> 5, unit = lane % UNITS;
    const uint32_t low = (uint32_t)(lane / UNITS);
    const int64_t c = n0 + 8 * unit, n = N - c;
    const uint32_t step = mask_step(f.mask);
    float b[8];
    finish_bias(f, c, N, b);
    RawUnit<T> next[S];
    auto here = [&](int64_t r0) __attribute__((always_inline)) { return WHOLE || (r0 + low < M && n > 0); };
    auto fetch = [&](int i) __attribute__((always_inline)) {
        if (!f.residual) return;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t r0 = m0 + 32 * i + ROWS * s;
            if constexpr (WHOLE) load_whole(narrow_at(f.residual, f.ldr, r0, low, (uint32_t)c), next[s]);
            else if (here(r0)) load_raw(f.residual + (r0 + low) * f.ldr + c, n, next[s]);
        }
    };
    auto store = [&](T* p, int64_t ld, int64_t r0, const float (&v)[8]) __attribute__((always_inline)) {
        if constexpr (WHOLE) store_unit<PAST>(narrow_at(p, ld, r0, low, (uint32_t)c), 8, v);
        else store_part<T, true>(p + (r0 + low) * ld + c, n, v);
    };
    // The streamed kernel's fp32 instances (an activation of their own) have no registers for the next 32 rows beside these: 8192 x 8192 x 4096 with a
    // residual 261 us with them ahead, 231 without.  (They spill 80 to 106 registers, the bf16 ones 8 to 16, and no other instance more than 6.)
    constexpr bool AHEAD = sizeof(T) < 4 || TN < 2 || ACT == ACT_ANY;
    if (AHEAD) fetch(0);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        if (!AHEAD) fetch(i);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                mx_put4(reinterpret_cast<float*>(sm + li * LROW) + 32 * j + 2 * v + 4 * half, acc[i][j][v], acc[i][j][v + 1], acc[i][j][v + 2],
                        acc[i][j][v + 3]);
        gs_wave_order();
        RawUnit<T> res[S];
#pragma unroll
        for (int s = 0; s < S; ++s) res[s] = next[s];
        if (AHEAD && i + 1 < TM) fetch(i + 1);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t r0 = m0 + 32 * i + ROWS * s;
            if (!here(r0)) continue;
            float v[1][8];
            load_row(reinterpret_cast<const float*>(sm + (ROWS * s + low) * LROW + 32 * unit), v[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] += b[e];
            if (f.pre) store(f.pre, f.ldp, r0, v[0]);
            finish_values<1>(f, step, c, [&](int) __attribute__((always_inline)) { return (uint32_t)r0 + low; }, v);
            if (f.residual) {
                float x[8];
                unpack(res[s], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[0][e] += x[e];
            }
            store(f.y, f.ldy, r0, v[0]);
        }
        gs_wave_order();
    }
}
// The streamed kernel's bf16 outputs, where a row's 64 columns are a whole line, leave past the caches, which keep the operands: 16384 x 14336 x 4096 with gelu
// and pre 644 us, so 605; 16384 x 4096 x 14336 with a residual 518, so 501.  Parts of lines cost more than they spare: 3000 x 6001 x 1024 39, past the caches 46;
// fp32 (half a line a store) 8192 x 8192 x 4096 178, 222.  (Not a choice at each store: the branches took half of it back.)
template <int TM, int TN, typename T, int ACT>
__device__ __forceinline__ void mx_finish_wave(const float16_t (&acc)[TM][TN], uint8_t* sm, const MxFinish<T, ACT>& end, int64_t m0, int64_t n0, int64_t M,
                                               int64_t N, int lane) {
    const MxFinish<T, ACT> f = finish_afresh(end);
    constexpr bool LINES = sizeof(T) == 2 && ACT != ACT_ANY;
    if (!f.narrow || m0 + 32 * TM > M || n0 + 32 * TN > N) mx_finish_rows<false, false>(acc, sm, f, m0, n0, M, N, lane);
    else if (LINES && f.lines) mx_finish_rows<true, LINES>(acc, sm, f, m0, n0, M, N, lane);
    else mx_finish_rows<true, false>(acc, sm, f, m0, n0, M, N, lane);
}

}  // namespace
