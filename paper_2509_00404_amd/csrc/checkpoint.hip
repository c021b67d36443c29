// 8-bit checkpoints of activations, and the gated activation whose backward pass reads one.
#include <type_traits>
#include "elementwise.h"

namespace {

// Largest magnitude bits of the four lanes that hold a block of 32 between them (as unsigned numbers, so that NaN is above infinity)
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true);     // lanes 1 0 3 2
    m = m > o ? m : o;
    o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true);              // lanes 2 3 0 1
    return m > o ? m : o;
}

// The lane's 8 codes of a block, and the block's scale byte.  448 * 2^t = 1.75 * 2^(t + 8): from the exponent field e of the largest
// magnitude, t + 127 = e - 8, or e - 7 where its fraction is above 0.75; at least 0.
__device__ __forceinline__ ew_u2 mx8_encode(const float (&v)[8], uint32_t& byte) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        m = m > b ? m : b;
    }
    m = quad_max(m);
    const int e = (int)(m >> 23) - ((m & 0x7FFFFFu) > 0x600000u ? 7 : 8);
    byte = e > 0 ? (uint32_t)e : 0u;
    const float inv = __uint_as_float((254u - byte) << 23);                                  // 2^-t, exact
    int w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inv, v[4 * h + 1] * inv, 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inv, v[4 * h + 3] * inv, w[h], true);
    }
    if (m >= 0x7F800000u) {
        byte = 255u;
        w[0] = w[1] = 0x7F7F7F7F;
    }
    return ew_u2{(uint32_t)w[0], (uint32_t)w[1]};
}
__device__ __forceinline__ void mx8_decode(ew_u2 c, uint32_t byte, float (&v)[8]) {
    typedef float f2_t __attribute__((ext_vector_type(2)));
    const float s = __uint_as_float(byte << 23 | (byte == 0u || byte == 255u ? 0x400000u : 0u));     // 0: 2^-127, 255: NaN
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
        v[4 * h] = lo.x * s;
        v[4 * h + 1] = lo.y * s;
        v[4 * h + 2] = hi.x * s;
        v[4 * h + 3] = hi.y * s;
    }
}

// a lane per 8 elements, four lanes per block; `units` of 8 a row.  Memory bounds all four kernels here: 65536 x 1024 bf16 activations and their
// checkpoint (541 MB moved) take 94 us, the gradients (674 MB) 115, 5.8 TB/s.
template <typename T>
__global__ void __launch_bounds__(256)
k_quantize_mx8(const T* __restrict__ A, int64_t ld, uint64_t total, FastDiv units, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;                                               // total is a multiple of 4: whole blocks leave
    const uint64_t row = div_by(units, n), c = n - row * units.d;
    float v[8];
    load_row(A + row * ld + 8 * c, v);
    uint32_t byte;
    const ew_u2 w = mx8_encode(v, byte);
    *reinterpret_cast<ew_u2*>(codes + 8 * n) = w;
    if ((threadIdx.x & 3) == 0) scales[n >> 2] = (uint8_t)byte;
}

template <typename T>
__global__ void __launch_bounds__(256)
k_dequantize_mx8(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint64_t total, FastDiv units, T* __restrict__ A,
                 int64_t ld) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const uint64_t row = div_by(units, n), c = n - row * units.d;
    float v[8];
    mx8_decode(*reinterpret_cast<const ew_u2*>(codes + 8 * n), scales[n >> 2], v);
    store_row(A + row * ld + 8 * c, v);
}

// sigmoid: for bf16 results the hardware's exponential and reciprocal, one unit in the last place each, as against a rounding to 8 bits
template <typename T>
__device__ __forceinline__ float gate(float g) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
    else return 1.0f / (1.0f + expf(-g));
}

template <typename T, bool SAVE>
__global__ void __launch_bounds__(256)
k_swiglu(const T* __restrict__ gu, int64_t ldg, uint64_t total, FastDiv units, T* __restrict__ act, int64_t lda, uint8_t* __restrict__ codes,
         uint8_t* __restrict__ scales) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const uint64_t row = div_by(units, n), c = n - row * units.d, F = 8ull * units.d;
    float g[8], u[8], a[8];
    load_row(gu + row * ldg + 8 * c, g);
    load_row(gu + row * ldg + F + 8 * c, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = g[i] * gate<T>(g[i]) * u[i];
    store_row(act + row * lda + 8 * c, a);
    if constexpr (SAVE) {
        uint32_t bg, bu;
        const ew_u2 wg = mx8_encode(g, bg), wu = mx8_encode(u, bu);
        uint8_t* p = codes + row * 2 * F + 8 * c;
        *reinterpret_cast<ew_u2*>(p) = wg;
        *reinterpret_cast<ew_u2*>(p + F) = wu;
        if ((threadIdx.x & 3) == 0) {
            uint8_t* q = scales + row * (F / 16) + c / 4;
            q[0] = (uint8_t)bg;
            q[F / 32] = (uint8_t)bu;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
k_swiglu_grads(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, uint64_t total, FastDiv units,
               const T* __restrict__ dact, int64_t ldd, T* __restrict__ dgu, int64_t ldg, T* __restrict__ act, int64_t lda) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const uint64_t row = div_by(units, n), c = n - row * units.d, F = 8ull * units.d;
    const uint8_t* p = codes + row * 2 * F + 8 * c;
    const uint8_t* q = scales + row * (F / 16) + c / 4;
    float g[8], u[8], d[8], a[8];
    load_row(dact + row * ldd + 8 * c, d);
    mx8_decode(*reinterpret_cast<const ew_u2*>(p), q[0], g);
    mx8_decode(*reinterpret_cast<const ew_u2*>(p + F), q[F / 32], u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = gate<T>(g[i]), gs = g[i] * s;
        a[i] = gs * u[i];
        g[i] = d[i] * u[i] * (s * (1.0f + g[i] * (1.0f - s)));
        u[i] = d[i] * gs;
    }
    store_row(dgu + row * ldg + 8 * c, g);
    store_row(dgu + row * ldg + F + 8 * c, u);
    if (act) store_row(act + row * lda + 8 * c, a);
}

bool mx8_ok(const metis_mx8* q) { return q && q->codes && q->scales && q->rows >= 1 && q->cols >= 32 && q->cols % 32 == 0; }
// blocks of 32 of a row in one go: 16-byte loads of A, 8-byte loads of the codes; the units of a launch (a lane has one, or one of either half
// of the row) fit its grid
int mx8_status(const metis_mat* A, const metis_mx8* q, bool halves = false) {
    if (!mat_ok(A) || !mx8_ok(q)) return METIS_INVALID_ARG;
    if (A->rows != q->rows || A->cols != q->cols || A->ld < A->cols || !mat_aligned16(A) || (uintptr_t)q->codes % 8) return METIS_BAD_SHAPE;
    return units_status(q->rows, q->cols / (halves ? 16 : 8));
}
dim3 unit_grid(int64_t units) { return dim3((unsigned)ceil_div64(units, 256)); }

bool half_of(const metis_mat* a, const metis_mat* whole) {
    return a->dtype == whole->dtype && a->rows == whole->rows && 2 * a->cols == whole->cols && a->ld >= a->cols && mat_aligned16(a);
}

}  // namespace

extern "C" int metis_quantize_mx8(void* stream, const metis_mat* A, metis_mx8* out) {
    if (A && out && A->rows == 0 && out->rows == 0) return METIS_OK;
    const int st = mx8_status(A, out);
    if (st != METIS_OK) return st;
    const FastDiv units = fast_div((uint32_t)(A->cols / 8));
    const int64_t total = A->rows * (A->cols / 8);
    hipStream_t s = (hipStream_t)stream;
    if (A->dtype == METIS_BF16)
        hipLaunchKernelGGL(k_quantize_mx8<bf16_t>, unit_grid(total), dim3(256), 0, s, (const bf16_t*)A->ptr, A->ld, (uint64_t)total, units,
                           out->codes, out->scales);
    else
        hipLaunchKernelGGL(k_quantize_mx8<float>, unit_grid(total), dim3(256), 0, s, (const float*)A->ptr, A->ld, (uint64_t)total, units,
                           out->codes, out->scales);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" int metis_dequantize_mx8(void* stream, const metis_mx8* A, metis_mat* out) {
    if (A && out && A->rows == 0 && out->rows == 0) return METIS_OK;
    const int st = mx8_status(out, A);
    if (st != METIS_OK) return st;
    const FastDiv units = fast_div((uint32_t)(A->cols / 8));
    const int64_t total = A->rows * (A->cols / 8);
    hipStream_t s = (hipStream_t)stream;
    if (out->dtype == METIS_BF16)
        hipLaunchKernelGGL(k_dequantize_mx8<bf16_t>, unit_grid(total), dim3(256), 0, s, A->codes, A->scales, (uint64_t)total, units,
                           (bf16_t*)out->ptr, out->ld);
    else
        hipLaunchKernelGGL(k_dequantize_mx8<float>, unit_grid(total), dim3(256), 0, s, A->codes, A->scales, (uint64_t)total, units,
                           (float*)out->ptr, out->ld);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" int metis_swiglu(void* stream, const metis_mat* gate_up, metis_mat* act, metis_mx8* saved) {
    if (gate_up && act && gate_up->rows == 0 && act->rows == 0) return METIS_OK;
    if (!mat_ok(gate_up) || !mat_ok(act)) return METIS_INVALID_ARG;
    if (act->rows < 1 || act->cols < 32 || act->cols % 32 || gate_up->ld < gate_up->cols || !mat_aligned16(gate_up) || !half_of(act, gate_up))
        return METIS_BAD_SHAPE;
    if (saved) {
        const int st = mx8_status(gate_up, saved, true);
        if (st != METIS_OK) return st;
    }
    const int big = units_status(act->rows, act->cols / 8);
    if (big != METIS_OK) return big;
    const FastDiv units = fast_div((uint32_t)(act->cols / 8));
    const int64_t total = act->rows * (act->cols / 8);
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](auto kern, auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(kern, unit_grid(total), dim3(256), 0, s, (const T*)gate_up->ptr, gate_up->ld, (uint64_t)total, units, (T*)act->ptr,
                           act->ld, saved ? saved->codes : nullptr, saved ? saved->scales : nullptr);
    };
    if (act->dtype == METIS_BF16) saved ? launch(k_swiglu<bf16_t, true>, bf16_t()) : launch(k_swiglu<bf16_t, false>, bf16_t());
    else saved ? launch(k_swiglu<float, true>, float()) : launch(k_swiglu<float, false>, float());
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" int metis_swiglu_grads(void* stream, const metis_mx8* saved, const metis_mat* dact, metis_mat* dgate_up, metis_mat* act) {
    if (saved && dact && dgate_up && saved->rows == 0 && dact->rows == 0 && dgate_up->rows == 0) return METIS_OK;
    if (!mat_ok(dact) || (act && !mat_ok(act))) return METIS_INVALID_ARG;
    const int st = mx8_status(dgate_up, saved, true);
    if (st != METIS_OK) return st;
    if (dact->cols < 32 || dact->cols % 32 || !half_of(dact, dgate_up) || (act && !half_of(act, dgate_up))) return METIS_BAD_SHAPE;
    const FastDiv units = fast_div((uint32_t)(dact->cols / 8));
    const int64_t total = dact->rows * (dact->cols / 8);
    hipStream_t s = (hipStream_t)stream;
    if (dact->dtype == METIS_BF16)
        hipLaunchKernelGGL(k_swiglu_grads<bf16_t>, unit_grid(total), dim3(256), 0, s, saved->codes, saved->scales, (uint64_t)total, units,
                           (const bf16_t*)dact->ptr, dact->ld, (bf16_t*)dgate_up->ptr, dgate_up->ld, act ? (bf16_t*)act->ptr : nullptr,
                           act ? act->ld : 0);
    else
        hipLaunchKernelGGL(k_swiglu_grads<float>, unit_grid(total), dim3(256), 0, s, saved->codes, saved->scales, (uint64_t)total, units,
                           (const float*)dact->ptr, dact->ld, (float*)dgate_up->ptr, dgate_up->ld, act ? (float*)act->ptr : nullptr,
                           act ? act->ld : 0);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
