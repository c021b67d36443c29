// A linear layer on MXFP4 operands whose epilogue adds a bias, applies an activation, drops elements and adds a residual; and the gradient of
// that epilogue.
#include "mx_gemm.h"
#include "linear.h"
#include "experts.h"
#include "column_sums.h"

namespace {

// ---- few rows: the weights stream through registers ----
// A workgroup has 16 OF outputs (the first operand of v_mfma_scale_f32_16x16x128_f8f6f4, so that a lane ends with four neighbouring outputs of a
// row) and all rows, up to 16 TG.  Its waves share the contraction: a run of 512 elements is 16 blocks of a row, 256 bytes, read 64 at a time by the four
// lanes that hold them; a wave takes every `waves`-th run, with the next one's weights on their way.  The waves' sums meet in LDS, added in their order, and
// eight neighbouring outputs of a row go through the epilogue together.
// FUSE (a type): the workgroup quantizes the rows itself, into LDS, while its first weights travel.
struct DenseRows {
    const void* ptr;
    int64_t ld;
};
typedef uint32_t lf_u4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef float lf_f4 __attribute__((ext_vector_type(4)));
typedef int lf_i8 __attribute__((ext_vector_type(8)));
#define FEW_ROWS 64
constexpr int few_waves(int tg, int of) { return tg * of <= 2 ? 16 : 8; }         // at most: more rows need more registers a wave
__host__ __device__ inline int few_runs(int nblk) { return (nblk + 15) / 16; }
__host__ __device__ inline int few_codes_row(int nblk) { return few_runs(nblk) * 256 + 16; }        // 16 more spread the rows over the banks
__host__ __device__ inline int few_scales_row(int nblk) { return few_runs(nblk) * 16; }
// The lane's blocks 4 i + g of run r (c[i]) with their scale bytes (s[i], the lowest).  Behind the row: its last block, zeros where ZERO (one
// operand's are enough).
template <bool ZERO>
__device__ __forceinline__ void run_load(const uint8_t* codes, const uint8_t* scales, int r, int nblk, int g, uvec4_t (&c)[4], uint32_t (&s)[4]) {
    const int b = 16 * r;
    if (b + 16 <= nblk) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = *reinterpret_cast<const uvec4_t*>(codes + 16 * (int64_t)(b + g) + 64 * i);
        const lf_u4_any w = *reinterpret_cast<const lf_u4_any*>(scales + b);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = w[i] >> (8 * g);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = b + 4 * i + g, at = x < nblk ? x : nblk - 1;
            c[i] = *reinterpret_cast<const uvec4_t*>(codes + 16 * (int64_t)at);
            s[i] = scales[at];
            if (ZERO && x >= nblk) c[i] = uvec4_t{0u, 0u, 0u, 0u};
        }
    }
}

template <typename OUT, int TG, int OF, typename T = void>
__global__ void __launch_bounds__(64 * few_waves(TG, OF))
k_linear_few(MxOperand X, DenseRows dense, MxOperand W, int nblk, MxFinish<OUT> f) {
    constexpr bool FUSE = !std::is_void<T>::value;
    constexpr int PROW = 16 * OF + 4;                    // floats of a row's sums of one wave
    extern __shared__ __attribute__((aligned(16))) uint8_t s_mem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int li = lane & 15, g = lane >> 4, rows = (int)X.rows, runs = few_runs(nblk);
    const int64_t N = W.rows, n0 = 16 * OF * (int64_t)blockIdx.x;
    const uint8_t *wc[OF], *wsc[OF];
#pragma unroll
    for (int o = 0; o < OF; ++o) {
        const int64_t n = n0 + 16 * o + li < N ? n0 + 16 * o + li : N - 1;
        wc[o] = W.codes + n * nblk * 16;
        wsc[o] = W.scales + n * nblk;
    }
    uvec4_t w[2][OF][4];
    uint32_t ws[2][OF][4];
    int r = wave;
    const int have = waves < runs ? waves : runs;        // waves with runs (FUSE: the others help to quantize)
    if (!FUSE || r < runs) {
#pragma unroll
        for (int o = 0; o < OF; ++o) run_load<false>(wc[o], wsc[o], r, nblk, g, w[0][o], ws[0][o]);
    }
    // what the epilogue reads for the thread's unit of eight outputs (the first, where few waves have more) is brought near behind the first weights
    const auto near = finish_near(f, (int)threadIdx.x / (2 * OF) < rows ? (int)threadIdx.x / (2 * OF) : 0, n0 + 8 * (threadIdx.x % (2 * OF)), N);
    const uint8_t *tc[TG], *tsc[TG];                     // this lane's rows
    if constexpr (FUSE) {
        uint8_t* s_scales = s_mem + rows * few_codes_row(nblk);
        const int per = runs * 64;                       // lanes a row: 8 elements each, four per block
        for (int i = threadIdx.x; i < rows * per; i += blockDim.x) {
            const int row = i / per, c = i - row * per;
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (c < 4 * nblk) load_row((const T*)dense.ptr + row * dense.ld + 8 * c, v);
            uint32_t byte;
            *reinterpret_cast<uint32_t*>(s_mem + row * few_codes_row(nblk) + 4 * c) = mx_quad(v, byte);
            if ((i & 3) == 0) s_scales[row * few_scales_row(nblk) + (c >> 2)] = (uint8_t)byte;
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < TG; ++t) {
        const int row = 16 * t + li < rows ? 16 * t + li : rows - 1;
        if constexpr (FUSE) {
            tc[t] = s_mem + row * few_codes_row(nblk);
            tsc[t] = s_mem + rows * few_codes_row(nblk) + row * few_scales_row(nblk);
        } else {
            tc[t] = X.codes + (int64_t)row * nblk * 16;
            tsc[t] = X.scales + (int64_t)row * nblk;
        }
    }
    lf_f4 acc[OF][TG];
#pragma unroll
    for (int o = 0; o < OF; ++o)
#pragma unroll
        for (int t = 0; t < TG; ++t) acc[o][t] = lf_f4{0.0f, 0.0f, 0.0f, 0.0f};
    auto run = [&](auto now_) __attribute__((always_inline)) {
        constexpr int now = decltype(now_)::value;
        if (r + waves < runs) {
#pragma unroll
            for (int o = 0; o < OF; ++o) run_load<false>(wc[o], wsc[o], r + waves, nblk, g, w[now ^ 1][o], ws[now ^ 1][o]);
        }
#pragma unroll
        for (int t = 0; t < TG; ++t) {
            uvec4_t x[4];
            uint32_t xs[4];
            if constexpr (FUSE) {                        // (in whole runs, zeros behind the row)
                const uvec4_t s = *reinterpret_cast<const uvec4_t*>(tsc[t] + 16 * r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = *reinterpret_cast<const uvec4_t*>(tc[t] + 256 * r + 64 * i + 16 * g);
                    xs[i] = s[i] >> (8 * g);
                }
            } else {
                run_load<true>(tc[t], tsc[t], r, nblk, g, x, xs);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const lf_i8 b = {(int)x[i].x, (int)x[i].y, (int)x[i].z, (int)x[i].w, 0, 0, 0, 0};
#pragma unroll
                for (int o = 0; o < OF; ++o) {
                    const uvec4_t y = w[now][o][i];
                    const lf_i8 a = {(int)y.x, (int)y.y, (int)y.z, (int)y.w, 0, 0, 0, 0};
                    acc[o][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[o][t], 4, 4, 0, (int)ws[now][o][i], 0, (int)xs[i]);
                }
            }
        }
        r += waves;
    };
#pragma unroll 1
    while (r < runs) {
        run(std::integral_constant<int, 0>{});
        if (r >= runs) break;
        run(std::integral_constant<int, 1>{});
    }
    if constexpr (FUSE) __syncthreads();                 // the sums take the rows' place
    float* s_part = reinterpret_cast<float*>(s_mem);
    if (wave < have) {
#pragma unroll
        for (int o = 0; o < OF; ++o)
#pragma unroll
            for (int t = 0; t < TG; ++t)
                *reinterpret_cast<lf_f4*>(s_part + ((wave * TG + t) * 16 + li) * PROW + 16 * o + 4 * g) = acc[o][t];
    }
    __syncthreads();
    const uint32_t step = mask_step(f.mask);
    finish_near_by(near);
    for (int u = threadIdx.x; u < rows * 2 * OF; u += blockDim.x) {
        const int row = u / (2 * OF), unit = u % (2 * OF);
        const int64_t c = n0 + 8 * unit;
        if (c >= N) continue;
        UnitInputs<OUT> in;
        finish_inputs(f, row, c, N, in);
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < have; ++p) {
            const lf_f4* q = reinterpret_cast<const lf_f4*>(s_part + (p * TG * 16 + row) * PROW + 8 * unit);
            const lf_f4 lo = q[0], hi = q[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] += lo[i];
                v[4 + i] += hi[i];
            }
        }
        finish_unit(f, step, row, c, N, in, v);
    }
}

// ---- few tiles ----
#include "mx_deep.h"

#define PARTS_MAX 16
// The parts' sums (fp32, rows of ld, a multiple of 8) added up in their order, through the epilogue.  A lane per eight outputs.
template <typename OUT>
__global__ void __launch_bounds__(256)
k_linear_join(const float* __restrict__ sums, int64_t ld, int64_t stride, int parts, uint64_t total, FastDiv units, int64_t N, MxFinish<OUT> f) {
    const uint64_t u = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= total) return;
    const int64_t r = (int64_t)div_by(units, u), c = 8 * (int64_t)(u - (uint64_t)r * units.d);
    const float* p = sums + r * ld + c;
    float v[8];
    UnitInputs<OUT> in;
    finish_inputs(f, r, c, N, in);
    load_row(p, v);
    int i = 1;
    for (; i + 3 < parts; i += 4) {
        float x[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k) load_row(p + (i + k) * stride, x[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += x[k][e];
    }
    for (; i < parts; ++i) {
        float x[8];
        load_row(p + i * stride, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
    finish_unit(f, mask_step(f.mask), r, c, N, in, v);
}

struct LinearParts {
    int count, units;                             // count 1: not cut
    int64_t ld, stride;                           // of the sums
};
// Cut where the units that a tile is spared (1.1 us each where the weights come from memory) outweigh the sums, written and read at some 450 outputs a ns,
// and the joining launch.  us without the quantizer, weights from memory, whole / cut in 2 / 4 / 8: 128 rows of 4096 x 14336 65.2 / 38.7 / 24.9 / 20.1, 256
// 64.2 / 39.2 / 27.3, 512 63.2 / 41.3; 128 of 14336 x 4096 22.3 / 20.7; of 4096 x 4096 21.0 / 16.8 / 15.3 / 18.5, 256 20.6 / 18.9 / 19.9, 512 20.5 / 23.2; of
// 1024 x 4096 15.7 / 12.3 / 10.6 / 10.3.
LinearParts linear_parts(int64_t rows, int64_t N, int64_t K) {
    const int64_t tiles = ceil_div64(rows, 128) * ceil_div64(N, 128), units = ceil_div64(K, MX_KI), ld = (N + 7) / 8 * 8;
    LinearParts p = {1, (int)units, ld, (rows * ld + 63) / 64 * 64};
    if (rows <= FEW_ROWS || tiles > 128) return p;
    double least = 1.1 * units;
    for (int64_t n = 2; n <= PARTS_MAX && n <= units / 2 && n * tiles <= 256; ++n) {       // (256: a CU each, and the same on any chip)
        const int64_t per = ceil_div64(units, n);
        const double t = 1.1 * per + 0.5 + n * rows * ld / 450e3;
        if (t >= least) continue;
        least = t;
        p.units = (int)per;
        p.count = (int)ceil_div64(units, per);
    }
    return p;
}
template <typename END>
int launch_deep(hipStream_t s, const MxOperand& x, const MxOperand& w, int64_t K, int parts, const END& end) {
    const int64_t tm = ceil_div64(x.rows, 128), tn = ceil_div64(w.rows, 128);
    const MxOrder order = mx_order(tm, tn, K, 128);
    const int nblk = (int)(K / 32);
    auto launch = [&](auto kern, int bytes, LdsLimitCache& lds_set) -> int {
        if (!ensure_dyn_lds((const void*)kern, bytes, lds_set)) return METIS_HIP_ERROR;
        hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn), (unsigned)parts), dim3(512), bytes, s, x, w, nblk, order, end);
        METIS_LAUNCH_CHECK();
        return METIS_OK;
    };
    static LdsLimitCache lds_set[3];
    if (nblk % 4 || (uintptr_t)x.scales % 4 || (uintptr_t)w.scales % 4) return launch(k_mxfp4_deep<true, true, END>, mxd_lds(true), lds_set[0]);
    if (nblk % 8) return launch(k_mxfp4_deep<false, true, END>, mxd_lds(false), lds_set[1]);
    return launch(k_mxfp4_deep<false, false, END>, mxd_lds(false), lds_set[2]);
}
template <typename T>
int launch_parts(hipStream_t s, const MxOperand& x, const MxOperand& w, int64_t K, const LinearParts& p, float* sums, const MxFinish<T>& f) {
    const int64_t units = p.ld / 8;
    const int us = units_status(x.rows, units);
    if (us != METIS_OK) return us;
    const int ds = launch_deep(s, x, w, K, p.count, MxParts{sums, p.ld, p.stride, p.units});
    if (ds != METIS_OK) return ds;
    const int64_t total = x.rows * units;
    hipLaunchKernelGGL(k_linear_join<T>, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s, sums, p.ld, p.stride, p.count, (uint64_t)total,
                       fast_div((uint32_t)units), w.rows, f);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
// Up to 448 tiles of 128 x 128 (beyond, tiles of 256 x 256 are as quick or quicker: 768 rows of 14336 x 4096, 672 tiles, 49.8 us for 49.7).
bool deep_tiles(int64_t rows, int64_t N) { return ceil_div64(rows, 128) * ceil_div64(N, 128) <= 448; }

struct LinearPlace {
    size_t scales, sums, bytes;                   // places of the rows' scales behind their codes and of the parts' sums, and the end
    LinearParts parts;
};
// dense: the rows' codes and scales have a place too
LinearPlace linear_place(int64_t rows, int64_t N, int64_t K, bool dense) {
    LinearPlace p;
    p.parts = linear_parts(rows, N, K);
    p.scales = dense ? align_up((size_t)rows * (K / 2), 256) : 0;
    p.sums = p.scales + (dense ? align_up((size_t)rows * (K / 32), 256) : 0);
    p.bytes = p.sums + (p.parts.count > 1 ? (size_t)p.parts.count * p.parts.stride * 4 : 0);
    return p;
}

// How few rows are shared out: 16 or 32 outputs a workgroup, and as many waves as let a CU hold its share of the workgroups at once (16 waves a CU, or 8
// where they need more registers; four at least).  us, 16 / 32 outputs: one row 14336 x 4096 11.6 / 10.3, 4096 x 14336 10.5 / 16.0; 64 rows 35.5 / 18.8,
// 23.3 / 27.6.  24 rows of 14336 x 4096 with four waves 13.2, with eight (half of the workgroups wait) 15.9.
struct FewShape {
    int tg, of, waves, fused;                     // waves where the rows are quantized already, and where they are not
};
FewShape few_shape(int64_t rows, int64_t N, int64_t K) {
    const int tg = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, of = N >= 8192 ? 2 : 1;
    const int64_t wgs = ceil_div64(N, 16 * of);
    // waves that a CU holds at once, over the workgroups that it has to hold
    const int64_t room = (tg == 1 ? 16 : tg == 2 && of == 1 ? 16 : 8) / ceil_div64(wgs, 256);
    const int64_t runs = few_runs((int)(K / 32));
    int64_t most = room < few_waves(tg, of) ? room : few_waves(tg, of);
    most = most < 4 ? 4 : most;
    const int64_t per = (runs + most - 1) / most;
    return {tg, of, (int)((runs + per - 1) / per), (int)(rows * runs < most ? rows * runs : most)};
}
// Quantized on the spot up to four eights of elements a thread.  us, with the quantizer's launch / on the spot: 14336 x 4096 (8 waves) one row 12.1 /
// 10.6, four 12.6 / 12.2, six 12.8 / 13.5; 4096 x 4096 (16 waves) one 7.5 / 6.0, eight 8.3 / 7.9, twelve 8.6 / 9.2; 4096 x 14336 two 12.4 / 11.9, three 12.7 /
// 13.1; 1024 x 1024 sixteen 5.6 / 4.6.
bool few_fused(int64_t rows, int64_t N, int64_t K) { return rows <= 16 && rows * few_runs((int)(K / 32)) <= 4 * few_shape(rows, N, K).fused; }
template <typename OUT, int TG, int OF, typename IN>
int launch_few(hipStream_t s, const MxOperand& x, const metis_mat* dense, const MxOperand& w, int64_t K, const MxFinish<OUT>& f, int waves) {
    constexpr bool FUSE = !std::is_void<IN>::value;
    const int nblk = (int)(K / 32);
    const size_t sums = (size_t)waves * TG * 16 * (16 * OF + 4) * 4, rows = FUSE ? (size_t)x.rows * (few_codes_row(nblk) + few_scales_row(nblk)) : 0;
    const size_t lds = sums > rows ? sums : rows;
    auto kern = k_linear_few<OUT, TG, OF, IN>;
    static LdsLimitCache lds_set;
    if (!ensure_dyn_lds((const void*)kern, lds, lds_set)) return METIS_HIP_ERROR;
    hipLaunchKernelGGL(kern, dim3((unsigned)ceil_div64(w.rows, 16 * OF)), dim3(64 * waves), lds, s, x,
                       DenseRows{FUSE ? dense->ptr : nullptr, FUSE ? dense->ld : 0}, w, nblk, f);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
// dense: rows that the kernel quantizes itself, or null
template <typename OUT>
int launch_few_shape(hipStream_t s, const MxOperand& x, const metis_mat* dense, const MxOperand& w, int64_t K, const MxFinish<OUT>& f) {
    const FewShape p = few_shape(x.rows, w.rows, K);
    auto by_type = [&](auto tg, auto of) {
        constexpr int TG = decltype(tg)::value, OF = decltype(of)::value;
        if (!dense) return launch_few<OUT, TG, OF, void>(s, x, dense, w, K, f, p.waves);
        if constexpr (TG == 1) return dense->dtype == METIS_BF16 ? launch_few<OUT, TG, OF, bf16_t>(s, x, dense, w, K, f, p.fused)
                                                                             : launch_few<OUT, TG, OF, float>(s, x, dense, w, K, f, p.fused);
        else return (int)METIS_INVALID_ARG;
    };
    auto by_of = [&](auto tg) {
        return p.of == 1 ? by_type(tg, std::integral_constant<int, 1>{}) : by_type(tg, std::integral_constant<int, 2>{});
    };
    return p.tg == 1 ? by_of(std::integral_constant<int, 1>{}) : p.tg == 2 ? by_of(std::integral_constant<int, 2>{}) : by_of(std::integral_constant<int, 4>{});
}

// ---- gradient of the epilogue ----
// dz = act'(pre) m dy, and the sum of its columns.  A lane has eight columns and goes down its rows with the next two on their way; the columns' sums stay in
// registers.  WIDE: the four waves of a workgroup lie side by side, 2048 columns, else they take neighbouring rows of 512 columns.  Workgroups take
// turns at the rows, so that what is read at any time lies together: with runs of rows of their own 16384 x 14336 bf16 takes 289 us (gelu) and 277
// (relu), so 269 and 245; BACK: the last unit of a row is short (see load_back; for rows of whole units as well, 265 for 256).  Memory bounds it: 1.41 GB
// in 250 us, 5.6 TB/s, with any activation.
template <typename T, int ACT, bool WIDE, bool PAST, bool BACK>
__global__ void __launch_bounds__(256)
k_linear_grads(const T* dy, int64_t ldd, const T* pre, int64_t ldp, T* dz, int64_t ldz, MaskKey mask, int64_t rows, int64_t cols,
               float* __restrict__ sums) {
    __shared__ float s_sum[WIDE ? 1 : 3 * 8 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t c = (WIDE ? 2048 * (int64_t)blockIdx.x + 512 * wave : 512 * (int64_t)blockIdx.x) + 8 * lane, n = cols - c;
    const int back = BACK ? unit_back(c, cols) : 0;
    const int64_t hop = WIDE ? gridDim.y : 4 * (int64_t)gridDim.y;
    const uint32_t step = mask_step(mask);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    int64_t r = WIDE ? blockIdx.y : 4 * (int64_t)blockIdx.y + wave;
    if (n > 0 && r < rows) {
        RawUnit<T> nd[2], np[2];
        auto fetch = [&](int64_t row, int k) __attribute__((always_inline)) {
            if constexpr (BACK) {
                load_back<PAST>(dy + row * ldd, c, back, cols, nd[k]);
                if (ACT != METIS_ACT_NONE) load_back<PAST>(pre + row * ldp, c, back, cols, np[k]);
            } else {
                load_whole<PAST>(dy + row * ldd + c, nd[k]);
                if (ACT != METIS_ACT_NONE) load_whole<PAST>(pre + row * ldp + c, np[k]);
            }
        };
        auto one = [&](int64_t row, int k) __attribute__((always_inline)) {
            float v[8], z[8];
            unpack(nd[k], back, v);
            if (ACT != METIS_ACT_NONE) unpack(np[k], back, z);
            fetch(row + 2 * hop < rows ? row + 2 * hop : row, k);
            if (ACT != METIS_ACT_NONE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= act_slope<sizeof(T) == 2>(ACT, z[i]);
            }
            // (the mask last: a dropped element is 0 whatever its slope is)
            if (mask.dropped) mask_apply(mask, step, (uint32_t)(c >> 3), (uint32_t)row, v);
            if (dz) store_unit<PAST>(dz + row * ldz + c, BACK ? n : 8, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        };
        fetch(r, 0);
        fetch(r + hop < rows ? r + hop : r, 1);
        for (; r < rows; r += 2 * hop) {
            one(r, 0);
            if (r + hop < rows) one(r + hop, 1);
        }
    }
    if (!sums) return;
    if constexpr (!WIDE) {
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s_sum[((wave - 1) * 8 + i) * 64 + lane] = sum[i];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += s_sum[(p * 8 + i) * 64 + lane];
    }
    if (n > 0) store_part<float, true>(sums + blockIdx.y * cols + c, n, sum);
}

// Past the caches from 128 MiB a matrix on, where the three do not fit the last-level cache: us, through / past, 16384 x 14336 283 / 269, 16384 x 4096 82 / 77,
// 4096 x 4096 23.8 / 27.4.
#define GRADS_PAST (128ll << 20)
// Few rows, one launch: a workgroup has 16 columns and all the rows, 128 at a time, two lanes a row.
template <typename T, int ACT>
__global__ void __launch_bounds__(256)
k_linear_grads_few(const T* dy, int64_t ldd, const T* pre, int64_t ldp, T* dz, int64_t ldz, MaskKey mask, int64_t rows, int64_t cols, float* dbias) {
    constexpr int W = 2, STEP = 256 / W;
    const uint32_t strip = xcd_strip(blockIdx.x, gridDim.x);
    __shared__ float s_sum[4 * 8 * W];
    const int64_t c = 8 * W * (int64_t)strip + 8 * (threadIdx.x % W), n = cols - c;
    const int back = unit_back(c, cols);
    const uint32_t step = mask_step(mask);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    int64_t r = threadIdx.x / W;
    if (n > 0 && r < rows) {
        RawUnit<T> nd, np;
        auto fetch = [&](int64_t row) __attribute__((always_inline)) {
            load_back(dy + row * ldd, c, back, cols, nd);
            if (ACT != METIS_ACT_NONE) load_back(pre + row * ldp, c, back, cols, np);
        };
        fetch(r);
        for (; r < rows; r += STEP) {
            float v[8], z[8];
            unpack(nd, back, v);
            if (ACT != METIS_ACT_NONE) unpack(np, back, z);
            fetch(r + STEP < rows ? r + STEP : r);
            if (ACT != METIS_ACT_NONE) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= act_slope<sizeof(T) == 2>(ACT, z[i]);
            }
            // (the mask last: a dropped element is 0 whatever its slope is)
            if (mask.dropped) mask_apply(mask, step, (uint32_t)(c >> 3), (uint32_t)r, v);
            if (dz) store_part<T, true>(dz + r * ldz + c, n, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
    }
    if (dbias) group_columns<4, W>(sum, s_sum, dbias, strip, cols);
}

bool grads_wide(int64_t cols) { return cols >= 2048; }
// us, bf16, gelu, rows in parts and a joining launch / k_linear_grads_few: 4 x 14336 6.9 / 4.5, 128 x 4096 8.1 / 5.0, 512 x 14336 16.6 / 14.7, 512 x 256
// 7.0 / 6.5, 700 x 4096 11.4 / 8.9, 1000 x 4096 12.0 / 10.5, 1000 x 256 9.6 / 9.4, 1111 x 1000 8.1 / 10.2, 1500 x 256 8.6 / 12.2.
bool grads_few(int64_t rows, int64_t cols) { return rows <= 768 && cols <= 65536; }
int64_t grads_strips(int64_t cols) { return ceil_div64(cols, grads_wide(cols) ? 2048 : 512); }
// Workgroups that share the rows of a strip, each of which leaves a row of partial sums: 1024 in all where each has eight rows or more, else 512 with two rows at
// least; the same on any chip so that the sums have the same order.  us, 512 / 1024 / 2048, gelu, bf16: 16384 x 14336 300 / 269 / 292, 16384 x 4096 87 / 77 /
// 86, 4096 x 4096 25.0 / 23.8 / 29.4, 1000 x 4096 11.6 / 14.7.
int64_t grads_parts(int64_t rows, int64_t cols) {
    if (grads_few(rows, cols)) return 1;
    const int64_t strips = grads_strips(cols), many = strips < 1024 ? 1024 / strips : 1, few = strips < 512 ? 512 / strips : 1;
    if (rows >= 8 * many) return many;
    const int64_t want = ceil_div64(rows, 2);
    return want < few ? want : few;
}

// whether two matrices of few rows have memory in common
bool share_memory(const metis_mat* a, const metis_mat* b) {
    auto row = [](const metis_mat* m, int64_t i) { return (uintptr_t)m->ptr + (uintptr_t)(i * m->ld * mat_size(m)); };
    auto meet = [](uintptr_t p, int64_t n, uintptr_t q, int64_t k) { return p < q + (uintptr_t)k && q < p + (uintptr_t)n; };
    const int64_t na = a->cols * mat_size(a), nb = b->cols * mat_size(b);
    if (!meet(row(a, 0), (int64_t)(row(a, a->rows - 1) - row(a, 0)) + na, row(b, 0), (int64_t)(row(b, b->rows - 1) - row(b, 0)) + nb)) return false;
    for (int64_t i = 0; i < a->rows; ++i)
        for (int64_t j = 0; j < b->rows; ++j)
            if (meet(row(a, i), na, row(b, j), nb)) return true;
    return false;
}
bool same_layout(const metis_mat* a, const metis_mat* b) { return a->rows == b->rows && a->cols == b->cols && a->ld >= a->cols; }

}  // namespace

static bool linear_sizes_ok(int64_t rows, int64_t N, int64_t K) {
    return rows >= 1 && N >= 1 && K >= 32 && K % 32 == 0 && rows <= 0xFFFFFFFFll / (K / 2) && N <= 0xFFFFFFFFll / (K / 2);
}
extern "C" size_t metis_mxfp4_linear_workspace_bytes(int64_t rows, int64_t N, int64_t K) {
    return !linear_sizes_ok(rows, N, K) || few_fused(rows, N, K) ? 0 : linear_place(rows, N, K, true).bytes;
}
extern "C" size_t metis_mxfp4_linear_quantized_workspace_bytes(int64_t rows, int64_t N, int64_t K) {
    return linear_sizes_ok(rows, N, K) ? linear_place(rows, N, K, false).bytes : 0;
}

extern "C" int metis_mxfp4_linear(void* stream, const metis_mat* X, const metis_mxfp4* Xq, const metis_mxfp4* W, const metis_epilogue* e,
                                  metis_mat* Y, void* workspace, size_t workspace_bytes) {
    if (!X == !Xq || !mx_ok(W) || !Y) return METIS_INVALID_ARG;
    const int64_t rows = X ? X->rows : Xq->rows, K = W->cols, N = W->rows;
    if (rows == 0 && Y->rows == 0) return METIS_OK;
    if (!mat_ok(Y) || (X ? !mat_ok(X) : !mx_ok(Xq)) || rows < 1) return METIS_INVALID_ARG;
    if (e && (!act_ok(e->act) || mask_status(e->mask) != METIS_OK || (e->pre && !mat_ok(e->pre)) || (e->residual && !mat_ok(e->residual)) ||
              (e->pre && e->pre->dtype != Y->dtype) || (e->residual && e->residual->dtype != Y->dtype) || (uintptr_t)e->bias % 4))
        return METIS_INVALID_ARG;
    if ((X ? X->cols : Xq->cols) != K || Y->rows != rows || Y->cols != N || Y->ld < N) return METIS_BAD_SHAPE;
    if (e && ((e->pre && !same_layout(e->pre, Y)) || (e->residual && !same_layout(e->residual, Y)))) return METIS_BAD_SHAPE;
    if (X && (X->ld < K || !mat_aligned16(X))) return METIS_BAD_SHAPE;
    uint8_t* ws = (uint8_t*)workspace;
    const LinearPlace place = linear_place(rows, N, K, X != nullptr);
    metis_mxfp4 q = X ? metis_mxfp4{ws, ws + place.scales, rows, K} : *Xq;
    const int st = mx_operands_status(X ? W : &q, W);
    if (st != METIS_OK) return st;
    const bool few = rows <= FEW_ROWS, fused = few && X && few_fused(rows, N, K);
    if (X) {
        if (rows * (K / 2) > 0xFFFFFFFFll) return METIS_UNSUPPORTED;
    }
    // (workgroups that are done store outputs while others still quantize X)
    if (fused && (share_memory(X, Y) || (e && e->pre && share_memory(X, e->pre)))) return METIS_INVALID_ARG;
    if (X && !fused) {
        if (!workspace || workspace_bytes < place.bytes) return METIS_WORKSPACE_TOO_SMALL;
        if ((uintptr_t)workspace % 256) return METIS_INVALID_ARG;
        const int qs = metis_quantize_mx(stream, X, &q);
        if (qs != METIS_OK) return qs;
    }
    const bool cut = place.parts.count > 1 && workspace && workspace_bytes >= place.bytes && (uintptr_t)workspace % 256 == 0;
    const int cus = device_cu_count();
    if (cus < 1) return METIS_HIP_ERROR;
    const MxOperand x = {q.codes, q.scales, rows}, w = {W->codes, W->scales, N};
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        const MxFinish<T> f = finish_of<T>(e, Y);
        if (few) return launch_few_shape<T>(s, x, fused ? X : nullptr, w, K, f);
        if (cut) return launch_parts<T>(s, x, w, K, place.parts, (float*)(ws + place.sums), f);
        if (deep_tiles(rows, N)) return launch_deep(s, x, w, K, 1, f);
        if (mx_streams(ceil_div64(rows, 256) * ceil_div64(N, 256), K, cus)) return linear_stream(s, &q, W, e, Y);
        return launch_mx_tile<T, 256>(s, x, w, K, f.y, f.ldy, f);
    };
    return Y->dtype == METIS_BF16 ? launch(bf16_t()) : launch(float());
}

extern "C" size_t metis_linear_grads_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || cols > (1 << 28) || rows > 0xFFFFFFFFll) return 0;
    const int64_t chunks = grads_parts(rows, cols);
    return chunks > 1 ? align_up((size_t)chunks * cols * 4, 256) : 0;
}

extern "C" int metis_linear_grads(void* stream, const metis_mat* dY, const metis_mat* pre, int act, const metis_dropout_mask* mask, metis_mat* dZ,
                                  float* dbias, void* workspace, size_t workspace_bytes) {
    if (!dY || !act_ok(act) || mask_status(mask) != METIS_OK || (uintptr_t)dbias % 4 || (!dZ && !dbias)) return METIS_INVALID_ARG;
    if (dY->rows != 0 && !mat_ok(dY)) return METIS_INVALID_ARG;
    if (act != METIS_ACT_NONE && !pre) return METIS_INVALID_ARG;
    if (act == METIS_ACT_NONE) pre = nullptr;
    if (dY->rows < 0 || dY->cols < 1 || dY->ld < dY->cols) return METIS_BAD_SHAPE;
    const int64_t rows = dY->rows, cols = dY->cols;
    if (cols > (1 << 28) || rows > 0xFFFFFFFFll) return METIS_UNSUPPORTED;
    hipStream_t s = (hipStream_t)stream;
    if ((pre && (pre->rows != rows || pre->cols != cols)) || (dZ && (dZ->rows != rows || dZ->cols != cols))) return METIS_BAD_SHAPE;
    if (rows == 0) return dbias ? launch_clear(s, dbias, cols) : METIS_OK;
    if ((pre && (!mat_ok(pre) || pre->dtype != dY->dtype)) || (dZ && (!mat_ok(dZ) || dZ->dtype != dY->dtype))) return METIS_INVALID_ARG;
    if ((pre && !same_layout(pre, dY)) || (dZ && !same_layout(dZ, dY))) return METIS_BAD_SHAPE;
    const bool few = grads_few(rows, cols);
    const int64_t chunks = grads_parts(rows, cols), strips = few ? ceil_div64(cols, 16) : grads_strips(cols);
    if (!grid_fits(strips, 256) || chunks > 65535) return METIS_UNSUPPORTED;
    const bool parts = dbias && chunks > 1;
    if (parts && (!workspace || workspace_bytes < metis_linear_grads_workspace_bytes(rows, cols))) return METIS_WORKSPACE_TOO_SMALL;
    if (parts && (uintptr_t)workspace % 256) return METIS_INVALID_ARG;
    float* sums = parts ? (float*)workspace : dbias;
    auto launch = [&](auto zero, auto a) {
        typedef decltype(zero) T;
        constexpr int ACT = decltype(a)::value;
        const bool past = rows * cols * mat_size(dY) >= GRADS_PAST;
        if (few) {
            hipLaunchKernelGGL((k_linear_grads_few<T, ACT>), dim3((unsigned)strips), dim3(256), 0, s, (const T*)dY->ptr, dY->ld,
                               pre ? (const T*)pre->ptr : nullptr, pre ? pre->ld : 0, dZ ? (T*)dZ->ptr : nullptr, dZ ? dZ->ld : 0, mask_key(mask),
                               rows, cols, dbias);
            return;
        }
        auto kern = k_linear_grads<T, ACT, false, false, true>;
        if (grads_wide(cols) && cols % 8) kern = past ? k_linear_grads<T, ACT, true, true, true> : k_linear_grads<T, ACT, true, false, true>;
        else if (grads_wide(cols)) kern = past ? k_linear_grads<T, ACT, true, true, false> : k_linear_grads<T, ACT, true, false, false>;
        hipLaunchKernelGGL(kern, dim3((unsigned)strips, (unsigned)chunks), dim3(256), 0, s, (const T*)dY->ptr, dY->ld,
                           pre ? (const T*)pre->ptr : nullptr, pre ? pre->ld : 0, dZ ? (T*)dZ->ptr : nullptr, dZ ? dZ->ld : 0, mask_key(mask),
                           rows, cols, sums);
    };
    auto by_act = [&](auto zero) {
        switch (act) {
            case METIS_ACT_RELU: launch(zero, std::integral_constant<int, METIS_ACT_RELU>{}); break;
            case METIS_ACT_GELU: launch(zero, std::integral_constant<int, METIS_ACT_GELU>{}); break;
            case METIS_ACT_GELU_TANH: launch(zero, std::integral_constant<int, METIS_ACT_GELU_TANH>{}); break;
            case METIS_ACT_SILU: launch(zero, std::integral_constant<int, METIS_ACT_SILU>{}); break;
            default: launch(zero, std::integral_constant<int, METIS_ACT_NONE>{}); break;
        }
    };
    if (dY->dtype == METIS_BF16) by_act(bf16_t());
    else by_act(float());
    METIS_LAUNCH_CHECK();
    return parts ? launch_join(s, sums, chunks, cols, dbias, cols, nullptr) : METIS_OK;
}
