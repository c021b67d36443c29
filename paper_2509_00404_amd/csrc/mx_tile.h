// Pieces shared by the kernels on the block-scaled FP4 matrix instruction: its wrapper, the streamed unit's layout in LDS, and the way of a
// wave's accumulator tiles to memory.
#pragma once
#include "gemm_tile.h"
#include "stream_dev.h"

typedef uint32_t uvec4_t __attribute__((ext_vector_type(4)));   // a native vector: copies stay in registers
typedef uint32_t uvec2_t __attribute__((ext_vector_type(2)));

#define MX_KI 256                                        // contraction elements of a stage: 128 bytes of every row

namespace {

// four neighbouring outputs of a row
__device__ __forceinline__ void mx_put4(bf16_t* p, float x, float y, float z, float w) {
    typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
    typedef float f2_t __attribute__((ext_vector_type(2)));
    const f2_t lo = {x, y}, hi = {z, w};
    *reinterpret_cast<uvec2_t*>(p) = uvec2_t{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf2_t)),
                                             __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf2_t))};
}
__device__ __forceinline__ void mx_put4(float* p, float x, float y, float z, float w) {
    *reinterpret_cast<float4*>(p) = make_float4(x, y, z, w);
}

// A wave's TM x TN accumulator tiles to memory.  LINES: 32 rows of its columns at a time are staged at sm (mx_wave_rows bytes), else
// straight from the registers.  whole: the workgroup's tile is stored without looking at each element (mx_whole).
template <typename OUT, int TN>
constexpr int mx_wave_rows() { return 32 * (32 * TN * (int)sizeof(OUT) + 16); }
// A tile inside the matrix; by way of LDS C has to allow 16-byte stores too, as vec says.  (Straight from the registers it has not: asked
// for it all the same, fp32 rows off 16 bytes took 151 us for 8192 x 14336 x 512 and 353 for x 4096, 131 and 332 without.)
template <bool LINES>
__device__ __forceinline__ bool mx_whole(bool inside, bool vec) { return inside && (!LINES || vec); }
template <typename OUT, bool LINES, int TM, int TN>
__device__ __forceinline__ void mx_store_wave(const float16_t (&acc)[TM][TN], uint8_t* sm, OUT* __restrict__ C, int64_t ldc, int64_t m0,
                                              int64_t n0, int64_t M, int64_t N, bool vec, bool whole, int lane) {
    const int li = lane & 31, half = lane >> 5;
    if constexpr (!LINES) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t c = n0 + 32 * j + li;
                const int64_t rbase = m0 + 32 * i + 4 * half;
                if (whole) {
                    store_tile16<OUT>(C + rbase * ldc + c, ldc, acc[i][j], 1.0f);
                } else {
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int64_t r = rbase + 8 * (v >> 2) + (v & 3);
                        if (r < M && c < N) store_out<OUT>(C + r * ldc + c, acc[i][j][v]);
                    }
                }
            }
    } else {
        constexpr int E = 16 / (int)sizeof(OUT), LROW = 32 * TN * (int)sizeof(OUT) + 16, UNITS = 32 * TN / E, ROWS = 64 / UNITS;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; v += 4)
                    mx_put4(reinterpret_cast<OUT*>(sm + li * LROW) + 32 * j + 2 * v + 4 * half, acc[i][j][v], acc[i][j][v + 1],
                            acc[i][j][v + 2], acc[i][j][v + 3]);
            gs_wave_order();
#pragma unroll
            for (int t = 0; t < 32 / ROWS; ++t) {
                const int row = ROWS * t + lane / UNITS, unit = lane % UNITS;
                const uint8_t* q = sm + row * LROW + 16 * unit;
                const uvec4_t w = *reinterpret_cast<const uvec4_t*>(q);
                const int64_t r = m0 + 32 * i + row, c = n0 + E * unit;
                OUT* p = C + r * ldc + c;
                if (whole) {
                    *reinterpret_cast<uvec4_t*>(p) = w;
                } else if (r < M) {
                    const int64_t left = N - c;
                    if (vec && left >= E) {
                        *reinterpret_cast<uvec4_t*>(p) = w;
                    } else {
#pragma unroll 1
                        for (int e = 0; e < E && e < left; ++e) p[e] = reinterpret_cast<const OUT*>(q)[e];
                    }
                }
            }
            gs_wave_order();
        }
    }
}

// acc (+)= X Y^T, 32 x 32 over 64 columns, block scales in byte 0 (HI: 2) of xs and ys; the accumulator in the accumulation registers.
// In asm for its place and its registers.  What the compiler then does not see: an accumulator read by a vector
// instruction soon after (mxs_settle); operands come from LDS, scales are shifted a step ahead.
template <bool FIRST, bool HI>
__device__ __forceinline__ void mxs_mfma(float16_t& acc, const uvec4_t& x, const uvec4_t& y, uint32_t xs, uint32_t ys) {
    if constexpr (FIRST)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, 0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "=a"(acc) : "v"(x), "v"(y), "v"(xs), "v"(ys));
    else if constexpr (HI)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(x), "v"(y), "v"(xs), "v"(ys));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc) : "v"(x), "v"(y), "v"(xs), "v"(ys));
}
__device__ __forceinline__ void mxs_settle(float16_t (&a)[2]) {
    asm volatile("s_nop 15\n\ts_nop 15" : "+a"(a[0]), "+a"(a[1]));
}
// between a vector instruction's result and the matrix instruction that reads it
__device__ __forceinline__ void mxs_settle_scales(uint32_t (&x)[6]) {
    asm volatile("s_nop 1" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]));
}

// LDS: two buffers of a unit: A's and B's codes row by row, 128 bytes a row, its 16-byte segments permuted by their number xor row / 2 %
// 8 (a transfer's lanes land side by side, and this is what spreads sixteen rows' reads of one segment over the banks), then 8 scale
// bytes of every row of both.
#define MXS_CODES 32768
#define MXS_SCALES 2048
#define MXS_UNIT (2 * MXS_CODES + 2 * MXS_SCALES)
#define MXS_LDS (2 * MXS_UNIT)
#define MXS_DMA 10                                       // transfers a wave makes for a unit

}  // namespace
