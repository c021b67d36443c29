// MXFP4 variant of the block-FP4 GEMM: the microscaling format that Sec. 2.3 names next to NVFP4
// (OCP MX v1.0: blocks of 32, one power-of-two E8M0 scale per block, E2M1 elements).  Its scales are
// exactly what gfx950's block-scaled matrix instruction applies in hardware, so the codes go from
// LDS straight into v_mfma_scale_f32_32x32x64_f8f6f4 with no expansion in the vector ALUs: this is
// the chip's FP4 rate, against which the NVFP4 path (E4M3 scales per 16, expanded to fp16) can be read.
#include "mx_gemm.h"

namespace {

// ---- quantizer: one lane per block of 32 consecutive elements of a row ----
// X = 2^(floor(log2 amax) - 2); elements round to the nearest E2M1 value of e / X, ties to the even code,
// magnitudes above 6 saturate (the packed converter does the rounding, saturation and nibble packing).
template <typename T>
__global__ void __launch_bounds__(256)
k_quantize_mx(const T* __restrict__ A, int64_t ld, int64_t M, int64_t nblk /* cols / 32 */, uint8_t* __restrict__ codes,
              uint8_t* __restrict__ scales) {
    const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (t >= M * nblk) return;
    const int64_t row = t / nblk, bc = t - row * nblk;
    float v[32];
    if constexpr (sizeof(T) == 2) {
        const uint4* src = reinterpret_cast<const uint4*>(A + row * ld + bc * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 a = src[i];
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * i + 2 * j] = bf16lo_to_f32(w[j]);
                v[8 * i + 2 * j + 1] = bf16hi_to_f32(w[j]);
            }
        }
    } else {
        const float4* src = reinterpret_cast<const float4*>(A + row * ld + bc * 32);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 a = src[i];
            v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
        }
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(v[i]));
    int sh = -127;
    if (amax > 0.0f) {
        sh = ilogbf(amax) - 2;
        sh = sh < -127 ? -127 : (sh > 127 ? 127 : sh);
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float y0 = ldexpf(v[8 * i + 2 * j], -sh), y1 = ldexpf(v[8 * i + 2 * j + 1], -sh);   // exact
            switch (j) {
                case 0: w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y0, y1, 1.0f, 0); break;
                case 1: w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y0, y1, 1.0f, 1); break;
                case 2: w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y0, y1, 1.0f, 2); break;
                default: w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[i], y0, y1, 1.0f, 3); break;
            }
        }
    }
    *reinterpret_cast<uint4*>(codes + t * 16) = make_uint4(w[0], w[1], w[2], w[3]);     // [M, cols/2] contiguous
    scales[t] = (uint8_t)(sh + 127);
}

}  // namespace

extern "C" int metis_quantize_mx(void* stream, const metis_mat* A, metis_mxfp4* out) {
    if (!A || !A->ptr || !mx_ok(out)) return METIS_INVALID_ARG;
    if (A->dtype != METIS_BF16 && A->dtype != METIS_F32) return METIS_INVALID_ARG;
    if (A->rows != out->rows || A->cols != out->cols || A->ld < A->cols) return METIS_BAD_SHAPE;
    const int64_t esz = A->dtype == METIS_BF16 ? 2 : 4;
    if ((A->ld * esz) % 16 || reinterpret_cast<uintptr_t>(A->ptr) % 16 || reinterpret_cast<uintptr_t>(out->codes) % 16)
        return METIS_BAD_SHAPE;                                       // 16-byte row loads and code stores
    const int64_t nblk = A->cols / 32, total = A->rows * nblk;
    hipStream_t s = (hipStream_t)stream;
    if (A->dtype == METIS_BF16)
        hipLaunchKernelGGL(k_quantize_mx<bf16_t>, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s,
                           (const bf16_t*)A->ptr, A->ld, A->rows, nblk, out->codes, out->scales);
    else
        hipLaunchKernelGGL(k_quantize_mx<float>, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s,
                           (const float*)A->ptr, A->ld, A->rows, nblk, out->codes, out->scales);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" int metis_mxfp4_gemm_nt(void* stream, const metis_mxfp4* A, const metis_mxfp4* B, metis_mat* C) {
    if (!mx_ok(A) || !mx_ok(B) || !C || !C->ptr) return METIS_INVALID_ARG;
    if (C->dtype != METIS_BF16 && C->dtype != METIS_F32) return METIS_INVALID_ARG;
    if (A->cols != B->cols || C->rows != A->rows || C->cols != B->rows || C->ld < C->cols) return METIS_BAD_SHAPE;
    const int64_t K = A->cols;
    const int st = mx_operands_status(A, B);
    if (st != METIS_OK) return st;
    const MxOperand a = {A->codes, A->scales, A->rows}, b = {B->codes, B->scales, B->rows};
    hipStream_t s = (hipStream_t)stream;
    if (C->dtype == METIS_F32) return launch_mx_gemm<float>(s, a, b, K, (float*)C->ptr, C->ld);
    return launch_mx_gemm<bf16_t>(s, a, b, K, (bf16_t*)C->ptr, C->ld);
}
