// The experts' products in MXFP4: the slots' rows with their experts' weights, and the weights' gradients.
#include <type_traits>
#include "mx_tile.h"
#include "experts.h"

typedef int ex_i8 __attribute__((ext_vector_type(8)));
typedef float ex_f4 __attribute__((ext_vector_type(4)));
typedef uint32_t ex_u2_any __attribute__((ext_vector_type(2), aligned(1)));

namespace {

// Scales as the stream reads them, "in units": [units of 256 contraction elements][rows][8 bytes], so that a tile's 256 rows have theirs of
// a unit in 2 KB that lie together.  (Row by row, a unit's 8 bytes of every row cost as many cache lines as its codes: of 16384 tokens'
// four experts, 2048 x 4096 each, 409 us with the quantizers; 356 without their transfers.)

// ---- blocks along the rows: A^T quantized, segment by segment ----
// A segment's result is a matrix of its own, [cols, its rows], behind those of the segments before it.  A lane holds 32 rows of two
// neighbouring columns, all of them in flight together; a workgroup's 8 waves have 256 rows of 128 columns, which leave by way of LDS as
// whole lines.  With a plan the segments are the experts' slots, padded with zeros to a multiple of 64, in rows of whole units and with
// scales in units, and row s of the segment is A's row token[s] where they are gathered; else they are runs of `rows` rows.
// FLAT (a plan's segments, for the gradients of few slots): rows of whole 64 slots and scales row by row, as k_experts_short reads them; a
// workgroup has 64 rows of 512 columns, and its lanes store by themselves.
// What bounds it: vector issue, 0.94 of the clocks, and memory alike.  32768 x 4096 gathered rows, 339 MB to be moved, take 55 us, x 2048 by slot
// (170 MB) 36, both in one launch 80 (6.3 TB/s).  (Loads in branches, 16
// bytes of a column stored at a time and scales byte by byte: 140 and 103.)
// Both operands of a gradient go in one launch, side by side along the columns: every workgroup takes up one of the two, `side`.
struct TurnSide {
    const void* A;
    const int32_t* token;
    uint8_t* codes;
    uint8_t* scales;
    int64_t ld, arows, cols;
    uint32_t blocks;                          // workgroups along its columns
};
#define QT_ROW 144                            // a column's 8 blocks of 16 bytes, and 16 that spread the columns over the banks
template <typename T, bool FLAT>
__global__ void __launch_bounds__(512)
k_quantize_mx_t(TurnSide one, TurnSide two, const int32_t* __restrict__ offsets, int E, int64_t S, int64_t rows, int64_t units) {
    const bool other = blockIdx.x >= one.blocks;
    const T* __restrict__ A = (const T*)(other ? two.A : one.A);
    const int32_t* __restrict__ token = other ? two.token : one.token;
    uint8_t* __restrict__ codes = other ? two.codes : one.codes;
    uint8_t* __restrict__ scales = other ? two.scales : one.scales;
    const int64_t ld = other ? two.ld : one.ld, arows = other ? two.arows : one.arows, cols = other ? two.cols : one.cols;
    const uint32_t bx = other ? blockIdx.x - one.blocks : blockIdx.x;
    __shared__ __attribute__((aligned(16))) uint8_t s_codes[FLAT ? 16 : 128 * QT_ROW];
    __shared__ __attribute__((aligned(16))) uint8_t s_scales[FLAT ? 8 : 128 * 8];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t unit = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    if (unit >= units) return;            // gridDim.y and z multiply to more than there are
    int64_t begin, count, stride, written, base, first;   // the segment's rows, the length of its result's rows and what is written of them, its place; the unit's first row
    if (FLAT || offsets) {
        constexpr int UNIT = FLAT ? 64 : SLOT_ALIGN;
        const SlotUnit u = find_unit(offsets, E, S, UNIT, unit);
        if (u.expert < 0) return;
        begin = u.begin;
        count = u.end - u.begin;
        stride = (count + UNIT - 1) / UNIT * UNIT;
        written = (count + 63) / 64 * 64;
        base = (unit - u.local) * UNIT * cols;
        first = (int64_t)u.local * UNIT;
    } else {
        const int64_t per = (rows + SLOT_ALIGN - 1) / SLOT_ALIGN, g = unit / per;
        begin = g * rows;
        count = stride = written = rows;
        base = begin * cols;
        first = (unit - g * per) * SLOT_ALIGN;
    }
    const int64_t col0 = FLAT ? (int64_t)bx * 512 + 128 * (wave >> 1) : (int64_t)bx * 128, col = col0 + 2 * lane;
    const int64_t from = first + 32 * (FLAT ? wave & 1 : wave);
    if (FLAT && col0 >= cols) return;
    if (from < written) {
        const int left = (int)(count - from < 32 ? count - from : 32);        // may be 0 or less: zeros
        int64_t r = from + (lane & 31);
        r = begin + (r < count ? r : count - 1);
        if (token) r = token[r];
        int row = (uint64_t)r < (uint64_t)arows ? (int)r : 0;
        const T* p = A + (col < cols ? col : 0);
        float v[2][32];
        if constexpr (sizeof(T) == 2) {
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = *reinterpret_cast<const uint32_t*>(p + (int64_t)__builtin_amdgcn_readlane(row, i) * ld);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                v[0][i] = bf16lo_to_f32(w[i]);
                v[1][i] = bf16hi_to_f32(w[i]);
            }
        } else {
            float2 w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = *reinterpret_cast<const float2*>(p + (int64_t)__builtin_amdgcn_readlane(row, i) * ld);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                v[0][i] = w[i].x;
                v[1][i] = w[i].y;
            }
        }
        if (left < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                v[0][i] = i < left ? v[0][i] : 0.0f;
                v[1][i] = i < left ? v[1][i] : 0.0f;
            }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t byte;
            const ew_u4 w = mx_block(v[c], byte);
            if constexpr (FLAT) {
                if (col < cols) {
                    const int64_t at = base + (col + c) * stride + from;
                    *reinterpret_cast<ew_u4*>(codes + at / 2) = w;
                    scales[at / 32] = (uint8_t)byte;
                }
            } else {
                *reinterpret_cast<ew_u4*>(s_codes + (2 * lane + c) * QT_ROW + 16 * wave) = w;
                s_scales[(2 * lane + c) * 8 + wave] = (uint8_t)byte;
            }
        }
    }
    if constexpr (FLAT) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = 64 * i + (tid >> 3), b = tid & 7;
        if (col0 + c < cols && first + 32 * b < written)
            *reinterpret_cast<ew_u4*>(codes + (base + (col0 + c) * stride + first + 32 * b) / 2) =
                *reinterpret_cast<const ew_u4*>(s_codes + c * QT_ROW + 16 * b);
    }
    if (offsets) {
        if (tid < 128 && col0 + tid < cols)
            *reinterpret_cast<ew_u2*>(scales + base / 32 + (first / 256 * cols + col0 + tid) * 8) = *reinterpret_cast<const ew_u2*>(s_scales + 8 * tid);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = 64 * i + (tid >> 3), b = tid & 7;
            if (col0 + c < cols && first + 32 * b < written) scales[(base + (col0 + c) * stride + first) / 32 + b] = s_scales[8 * c + b];
        }
    }
}

// ---- products for few slots an expert: straight from memory ----
// What counts is that the weights stream: they pass through registers alone, and nothing waits for anybody.  A wave has 32 of the expert's N
// (the first operand, so that a lane ends with runs of four neighbouring outputs) and up to 32 slots, on v_mfma_scale_f32_32x32x64_f8f6f4:
// a lane's operand is the 32 codes (16 bytes) of row lane % 32 and one block of either half of the step.  Which blocks a step takes is free as
// long as both operands agree: over a run of 512 elements a lane takes the 8 blocks of its half one after the other, 128 bytes
// that lie together, and their 8 scale bytes.  The weights of the next run are on their way while one is multiplied.
// SPLIT: the workgroup's four waves share 32 outputs, take every fourth run, and add up in their order by way of LDS; else each has 32 of its own.
// FUSE: few elements a unit (a decode step).  The workgroup quantizes its slots' rows itself, into LDS, while its first weights travel; a launch
// of the row quantizer in front costs more (figures where it is chosen).
struct MxRows {
    const uint8_t* codes;
    const uint8_t* scales;
};
// Blocks r + 8 h .. r + 8 h + 7 of a row (h = lane / 32), r the run's first.  Of the last run, where it is short, what lies behind the row's
// nblk blocks is the last block once more under some scale, and zeros where ZERO: one operand's zeros are enough.
template <bool ZERO>
__device__ __forceinline__ void few_load(const uint8_t* codes, const uint8_t* scales, int r, int nblk, int half, ew_u4 (&c)[8], uint32_t (&sc)[2]) {
    const int b = r + 8 * half;
    if (r + 16 <= nblk) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = *reinterpret_cast<const ew_u4*>(codes + 16 * (int64_t)b + 16 * i);
        const ex_u2_any w = *reinterpret_cast<const ex_u2_any*>(scales + b);
        sc[0] = w[0];
        sc[1] = w[1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = *reinterpret_cast<const ew_u4*>(codes + 16 * (int64_t)(b + i < nblk ? b + i : nblk - 1));
        if (ZERO) {
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = b + i < nblk ? c[i] : ew_u4{0u, 0u, 0u, 0u};
        }
        uint64_t w = 0;
        if (nblk >= 8) {
            const int at = b + 8 < nblk ? b : nblk - 8, off = b - at;
            const ex_u2_any v = *reinterpret_cast<const ex_u2_any*>(scales + at);
            w = ((uint64_t)v[1] << 32 | v[0]) >> (8 * (off < 7 ? off : 7));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= (uint64_t)scales[b + i < nblk ? b + i : nblk - 1] << (8 * i);
        }
        sc[0] = (uint32_t)w;
        sc[1] = (uint32_t)(w >> 32);
    }
}
template <int I>
__device__ __forceinline__ void few_step(float16_t& acc, const ew_u4 (&w)[8], const uint32_t (&ws)[2], const ew_u4 (&t)[8], const uint32_t (&ts)[2]) {
    const ex_i8 a = {(int)w[I][0], (int)w[I][1], (int)w[I][2], (int)w[I][3], 0, 0, 0, 0};
    const ex_i8 b = {(int)t[I][0], (int)t[I][1], (int)t[I][2], (int)t[I][3], 0, 0, 0, 0};
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 4, I & 3, (int)ws[I >> 2], I & 3, (int)ts[I >> 2]);
}
// four neighbouring outputs of a row; vec: the row and the place allow one store
template <typename OUT>
__device__ __forceinline__ void put4(OUT* p, ex_f4 v, int64_t left, bool vec) {
    if (vec && left >= 4) {
        if constexpr (sizeof(OUT) == 2) *reinterpret_cast<ew_u2*>(p) = ew_u2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        else *reinterpret_cast<ex_f4*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) store_one(p + i, v[i]);
}

struct DenseRows {
    const void* ptr;
    int64_t ld;
};
// LDS of a quantized row: codes in whole runs and 16 bytes that spread the rows over the banks, then the scales
__host__ __device__ inline int few_code_row(int nblk) { return (nblk + 15) / 16 * 256 + 16; }
__host__ __device__ inline int few_scale_row(int nblk) { return (nblk + 15) / 16 * 16; }
// `rows` rows of A quantized to LDS, by all 256 threads; row_of(i): A's row
template <typename T, typename F>
__device__ __forceinline__ void few_quantize(const T* A, int64_t ld, int rows, int nblk, uint8_t* codes, uint8_t* scales, const F& row_of) {
    const int per = (nblk + 15) / 16 * 64;               // lanes a row: 8 elements each, four per block
    for (int i = threadIdx.x; i < rows * per; i += 256) {
        const int row = i / per, c = i - row * per;
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (c < 4 * nblk) load_row(A + row_of(row) * ld + 8 * c, v);
        uint32_t byte;
        const uint32_t w = mx_quad(v, byte);
        *reinterpret_cast<uint32_t*>(codes + row * few_code_row(nblk) + 4 * c) = w;
        if ((i & 3) == 0) scales[row * few_scale_row(nblk) + (c >> 2)] = (uint8_t)byte;
    }
}

template <typename OUT, bool SPLIT, typename T = void>
__global__ void __launch_bounds__(256, 2)
k_experts_few(MxRows A, DenseRows dense, int64_t arows, MxRows W, const int32_t* __restrict__ offsets, const int32_t* __restrict__ token, int E, int64_t S,
              int64_t N, int nblk, OUT* __restrict__ C, int64_t ldc, bool vec, uint32_t nblocks, uint32_t most) {
    constexpr bool FUSE = !std::is_void<T>::value;
    __shared__ float s_part[SPLIT ? 3 * 16 * 64 : 1];
    extern __shared__ __attribute__((aligned(16))) uint8_t s_rows[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), li = lane & 31, half = lane >> 5;
    const uint32_t ub = blockIdx.x / nblocks, nb = blockIdx.x - ub * nblocks;
    const SlotUnit u = find_unit(offsets, E, S, 32, ub);
    const int64_t n0 = SPLIT ? 32 * (int64_t)nb : 128 * (int64_t)nb + 32 * wave;
    if (u.expert < 0) {                                  // behind the last unit of slots the workgroups clear the unused ones
        const int64_t step = most - u.total, wide = SPLIT ? 32 : 128, c0 = wide * nb;
        for (int64_t s = u.used + ub - u.total; s < S; s += step)
            for (int64_t c = c0 + threadIdx.x; c < c0 + wide && c < N; c += 256) C[s * ldc + c] = OUT(0);
        return;
    }
    if (!FUSE && n0 >= N) return;                        // (SPLIT: not for some waves of a workgroup alone)
    const int64_t first = u.begin + 32 * (int64_t)u.local;
    const uint64_t n = (uint64_t)u.expert * N + (n0 + li < N ? n0 + li : N - 1);
    const uint8_t *wc = W.codes + n * nblk * 16, *wsc = W.scales + n * nblk;
    auto row_of = [&](int i) {                           // A's row of the unit's slot i
        const int64_t s = first + i, sr = s < u.end ? s : u.end - 1;
        const uint64_t row = token ? (uint64_t)(uint32_t)token[sr] : (uint64_t)sr;
        return (int64_t)(row < (uint64_t)arows ? row : (uint64_t)arows - 1);
    };
    const uint8_t *tc, *tsc;                             // this lane's slot's row
    float16_t acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
    constexpr int hop = SPLIT ? 64 : 16;
    ew_u4 w[2][8];
    uint32_t ws[2][2];
    int r = SPLIT ? 16 * wave : 0;
    if (r < nblk) few_load<false>(wc, wsc, r, nblk, half, w[0], ws[0]);
    if constexpr (FUSE) {
        const int rows = u.end - first < 32 ? (int)(u.end - first) : 32, mine = li < rows ? li : rows - 1;
        tc = s_rows + mine * few_code_row(nblk);
        tsc = s_rows + rows * few_code_row(nblk) + mine * few_scale_row(nblk);
        few_quantize((const T*)dense.ptr, dense.ld, rows, nblk, s_rows, s_rows + rows * few_code_row(nblk), row_of);
        __syncthreads();
        if (n0 >= N) return;
    } else {
        const int64_t row = row_of(li);
        tc = A.codes + row * nblk * 16;
        tsc = A.scales + row * nblk;
    }
    auto run = [&](auto now_) __attribute__((always_inline)) {
        constexpr int now = decltype(now_)::value;
        ew_u4 t[8];
        uint32_t ts[2];
        if constexpr (FUSE) {                            // (in whole runs, zeros behind the row)
            const int b = r + 8 * half;
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = *reinterpret_cast<const ew_u4*>(tc + 16 * (b + i));
            const ew_u2 x = *reinterpret_cast<const ew_u2*>(tsc + b);
            ts[0] = x[0];
            ts[1] = x[1];
        } else {
            few_load<true>(tc, tsc, r, nblk, half, t, ts);
        }
        if (r + hop < nblk) few_load<false>(wc, wsc, r + hop, nblk, half, w[now ^ 1], ws[now ^ 1]);
        few_step<0>(acc, w[now], ws[now], t, ts);
        few_step<1>(acc, w[now], ws[now], t, ts);
        few_step<2>(acc, w[now], ws[now], t, ts);
        few_step<3>(acc, w[now], ws[now], t, ts);
        few_step<4>(acc, w[now], ws[now], t, ts);
        few_step<5>(acc, w[now], ws[now], t, ts);
        few_step<6>(acc, w[now], ws[now], t, ts);
        few_step<7>(acc, w[now], ws[now], t, ts);
        r += hop;
    };
#pragma unroll 1
    while (r < nblk) {
        run(std::integral_constant<int, 0>{});
        if (r >= nblk) break;
        run(std::integral_constant<int, 1>{});
    }
    if constexpr (SPLIT) {
        if (wave > 0) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s_part[((wave - 1) * 16 + v) * 64 + lane] = acc[v];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[v] += s_part[(p * 16 + v) * 64 + lane];
    }
    const int64_t s = first + li;
    if (s >= u.end) return;
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
        const int64_t c = n0 + 2 * v + 4 * half;
        put4(C + s * ldc + c, ex_f4{acc[v], acc[v + 1], acc[v + 2], acc[v + 3]}, N - c, vec);
    }
}

#include "experts_stream.h"

// ---- gradients of few slots an expert ----
// dW is what is written and bounds it; the contraction is a step or two.  A wave has 128 x 64 outputs, a workgroup 128 x 256; operands come
// straight from memory and nothing waits for anybody, so that one wave's stores and another's loads overlap (on the stream, a tile of a single
// unit waits for its transfers, then for its stores).  Operands as the quantizer's FLAT form leaves them.
template <typename OUT, bool PAST>
__global__ void __launch_bounds__(256, 2)
k_experts_short(MxRows G, MxRows X, const int32_t* __restrict__ offsets, int E, int64_t S, int64_t N, int64_t K, OUT* __restrict__ dW, int64_t ldw,
                bool vec, uint32_t tiles_k) {
    constexpr bool LINES = sizeof(OUT) == 2;             // outputs by way of LDS, accumulator tiles transposed
    __shared__ __attribute__((aligned(16))) uint8_t s_stage[LINES ? 4 * EX_STAGE : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), li = lane & 31, half = lane >> 5;
    const int e = blockIdx.y;
    const uint32_t tn = blockIdx.x / tiles_k, tk = blockIdx.x - tn * tiles_k;
    const int64_t n0 = 128 * (int64_t)tn, k0 = 256 * (int64_t)tk + 64 * wave;
    if (k0 >= K) return;
    const ExpertSlots own = slots_of(offsets, E, S, 64, e);
    const int64_t before = own.units_before;
    const int steps = (int)((own.count + 63) >> 6);
    const int64_t len = 64 * (int64_t)steps;
    float16_t acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    int64_t at[6];                                       // of this lane's rows: 0 .. 3 of G, 4 and 5 of X
#pragma unroll
    for (int x = 0; x < 6; ++x) {
        const int64_t rows = x < 4 ? N : K, r = (x < 4 ? n0 + 32 * x : k0 + 32 * (x - 4)) + li;
        at[x] = 64 * before * rows + (r < rows ? r : rows - 1) * len + 32 * half;
    }
    for (int s = 0; s < steps; ++s) {
        ew_u4 f[6];
        int sc[6];
#pragma unroll
        for (int x = 0; x < 6; ++x) {
            const MxRows& m = x < 4 ? G : X;
            f[x] = *reinterpret_cast<const ew_u4*>(m.codes + at[x] / 2);
            sc[x] = m.scales[at[x] / 32];
            at[x] += 64;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n0 + 32 * i >= N) continue;
            const ex_i8 g = {(int)f[i][0], (int)f[i][1], (int)f[i][2], (int)f[i][3], 0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const ew_u4 y = f[4 + j];
                const ex_i8 x = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
                if constexpr (LINES) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, g, acc[i][j], 4, 4, 0, sc[4 + j], 0, sc[i]);
                else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(g, x, acc[i][j], 4, 4, 0, sc[i], 0, sc[4 + j]);
            }
        }
    }
    OUT* C = dW + (int64_t)e * N * ldw;
    const bool inside = n0 + 128 <= N && k0 + 64 <= K;
    if constexpr (LINES) ex_store_lines<PAST>(acc, s_stage + wave * EX_STAGE, C, ldw, n0, k0, N, K, vec, inside && vec, lane);
    else ex_store_plain<PAST>(acc, C, ldw, n0, k0, N, K, inside, lane);
}

// ---- rows quantized for the products ----
// [rows, K] -> codes, in rows of Kp elements (K filled up with zeros), and scales.  A lane per 8 elements, four lanes per block of 32.
// UNITS: Kp is a multiple of 256, and the scales go in units to the rows' slots: a lane of the 16 that hold four blocks writes their bytes for
// one choice.  The workgroups behind the rows' put the weights' scales in units.
struct RowScales {
    uint8_t* to;
    const int32_t* slot;                          // [rows, k]: the slots of a row; null: its own number
    int64_t S;
    int k;
};
struct WeightScales {
    const uint8_t* from;                          // [rows, have]
    uint8_t* to;
    int64_t rows;
    int have, units;
};
__device__ __forceinline__ void lay_scales(const WeightScales& w, int64_t block) {
    const int64_t row = block * 64 + (threadIdx.x & 63);
    if (row >= w.rows) return;
    const uint8_t* p = w.from + row * w.have;
    const int64_t left = (w.rows - row) * w.have;        // bytes that may be read from p on
    for (int u = threadIdx.x >> 6; u < w.units; u += 4) {
        const int n = w.have - 8 * u;                    // of the row's in this unit, 8 or more: all
        uint64_t v = 0;
        if (8 * u + 8 <= left) {
            const ex_u2_any x = *reinterpret_cast<const ex_u2_any*>(p + 8 * u);
            v = (uint64_t)x[1] << 32 | x[0];
        } else {
            for (int i = 0; i < n; ++i) v |= (uint64_t)p[8 * u + i] << (8 * i);
        }
        if (n < 8) v = (v & ~(~0ull << (8 * n))) | 0x7F7F7F7F7F7F7F7Full << (8 * n);
        *reinterpret_cast<uint64_t*>(w.to + (u * w.rows + row) * 8) = v;
    }
}
template <typename T, bool UNITS>
__global__ void __launch_bounds__(256)
k_quantize_rows(const T* __restrict__ A, int64_t ld, int64_t K, uint64_t total, FastDiv units, uint8_t* __restrict__ codes,
                RowScales rs, WeightScales ws, uint32_t row_blocks) {
    if (UNITS && blockIdx.x >= row_blocks) {
        lay_scales(ws, blockIdx.x - row_blocks);
        return;
    }
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;                                               // total is a multiple of 4 (UNITS: 32): whole blocks (units) leave
    const uint64_t row = div_by(units, n);
    const uint32_t unit = (uint32_t)(n - row * units.d);
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (8 * (int64_t)unit < K) load_row(A + row * ld + 8 * (int64_t)unit, v);
    uint32_t byte;
    *reinterpret_cast<uint32_t*>(codes + 4 * n) = mx_quad(v, byte);
    if constexpr (UNITS) {
        uint32_t w = byte << (8 * (threadIdx.x >> 2 & 3));
        w |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x124, 0xF, 0xF, true);         // around the 16 lanes by 4, then by 8
        w |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x128, 0xF, 0xF, true);
        const int j = threadIdx.x & 15;
        if (j < rs.k) {
            const int64_t s = rs.slot ? rs.slot[row * rs.k + j] : (int64_t)row;
            if ((uint64_t)s < (uint64_t)rs.S) *reinterpret_cast<uint32_t*>(rs.to + ((unit >> 5) * rs.S + s) * 8 + 4 * (unit >> 4 & 1)) = w;
        }
    } else {
        if ((threadIdx.x & 3) == 0) rs.to[n >> 2] = (uint8_t)byte;
    }
}

#define PARTS_MAX 8
// The parts of a contraction (sums of part p: rows p S and on of P, ld columns, a multiple of 4) added up in their order; slots from the end of
// the experts' on get zeros.
template <typename OUT>
__global__ void __launch_bounds__(256)
k_experts_join(const float* __restrict__ P, int64_t ld, int parts, const int32_t* __restrict__ offsets, int E, int64_t S, int64_t N, uint64_t total,
             FastDiv quads, OUT* __restrict__ C, int64_t ldc, bool vec) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const int64_t row = (int64_t)div_by(quads, n), c = 4 * (int64_t)(n - (uint64_t)row * quads.d);
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (row < held(offsets[E], S)) {
        const float* p = P + row * ld + c;
        ew_f4 x[PARTS_MAX] = {};
#pragma unroll
        for (int i = 0; i < PARTS_MAX; ++i, p += S * ld)
            if (i < parts) x[i] = *reinterpret_cast<const ew_f4*>(p);     // all on their way at once
#pragma unroll
        for (int i = 0; i < PARTS_MAX; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += x[i][j];
    }
    OUT* q = C + row * ldc + c;
    if (vec && c + 4 <= N) {
        mx_put4(q, v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < N) {
                if constexpr (sizeof(OUT) == 2) q[i] = (bf16_t)pack_bf16(v[i], 0.0f);
                else q[i] = v[i];
            }
    }
}

int experts_plan_status(const metis_expert_plan* p) {
    if (!p || !p->offsets || p->tokens < 0 || p->k < 1 || p->experts < 1) return METIS_INVALID_ARG;
    if (p->experts > EXPERTS_MAX || p->k > 16) return METIS_UNSUPPORTED;
    if (p->tokens > 0x7FFFFFFFll / p->k) return METIS_BAD_SHAPE;
    return METIS_OK;
}
// Gradients of few slots an expert go without the stream.  us with the quantizer, without / with it, by slots an expert:
//   bf16  64 experts of 1024 x 2048    31 67 / 72     100 77 / 73    160 86 / 77       64 of 1384 x 2456   31 148 / 155   126 175 / 151
//         128 of 80 x 3240             31 37 / 72     126 63 / 85    160 73 / 94       256 of 2464 x 400   31 185 / 254   126 269 / 282   160 302 / 296
//   fp32  64 of 1024 x 2048            31 100 / 111   62 101 / 111   100 108 / 113     64 of 1384 x 2456   31 258 / 252   62 259 / 251
//         128 of 80 x 3240             31 44 / 79     62 52 / 85     100 63 / 96       256 of 2464 x 400   31 261 / 334   62 262 / 335    100 286 / 342
//         64 of 1024 x 2040            31 176 / 155   62 178 / 154   100 184 / 159     64 of 512 x 1000    31 34 / 43     62 36 / 43      100 40 / 44
// The limits are between what gains and what loses: fp32 gradients of half a GB and more whose rows do not start on cache lines lose up to 15 %
// below theirs, others would gain as much above it.
bool wgrad_short(int64_t S, int E, int dtype) { return S < (dtype == METIS_BF16 ? 128 : 64) * (int64_t)E; }
// quantize A^T, and B^T of the same rows and type where there is a B, by segments of a plan (gathered where a token list is there) or of `rows` rows
TurnSide turn_side(const metis_mat* A, const int32_t* token, bool flat, uint8_t* codes, uint8_t* scales) {
    return {A->ptr, token, codes, scales, A->ld, A->rows, A->cols, (uint32_t)ceil_div64(A->cols, flat ? 512 : 128)};
}
int launch_quantize_mx_t(hipStream_t s, const TurnSide& one, const TurnSide& two, int dtype, const metis_expert_plan* p, bool flat, int64_t rows) {
    const int64_t S = p ? p->tokens * p->k : 0;
    const int64_t units = p ? most_units(S, p->experts, flat ? 64 : SLOT_ALIGN) : one.arows / rows * ceil_div64(rows, SLOT_ALIGN);
    const int64_t gy = units < 32768 ? units : 32768, gz = ceil_div64(units, gy);
    const dim3 grid(one.blocks + two.blocks, (unsigned)gy, (unsigned)gz);
    const int64_t blocks = ceil_div64(one.cols, flat ? 512 : 128) + ceil_div64(two.cols, flat ? 512 : 128);
    if (!grid_fits(blocks, 512) || gz > 65535 || one.arows > 0x7FFFFFFF || two.arows > 0x7FFFFFFF) return METIS_UNSUPPORTED;
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(512), 0, s, one, two, p ? p->offsets : nullptr, p ? p->experts : 0, S, rows, units); };
    if (dtype == METIS_BF16) flat ? launch(k_quantize_mx_t<bf16_t, true>) : launch(k_quantize_mx_t<bf16_t, false>);
    else flat ? launch(k_quantize_mx_t<float, true>) : launch(k_quantize_mx_t<float, false>);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
int64_t padded_slots(int64_t S, int E) { return most_units(S, E, SLOT_ALIGN) * SLOT_ALIGN; }
// (a tile reads the scales of 256 rows wherever its own end)
size_t mx_bytes(int64_t rows, int64_t cols) { return align_up((size_t)rows * cols / 2, 256) + align_up((size_t)rows * cols / 32, 256) + 2048; }

// The stream takes products of 16 slots an expert and more; what it cannot address, and fewer, goes straight from memory.  us, from memory /
// streamed, 2048 x 4096 with 64 experts of which a token takes four: 24 tokens 57 / 69 (4096 x 1024: 26 / 44), 64 66 / 73, 200 75 / 74, 250
// 81 / 75, 400 103 / 77, 1000 184 / 83.  The average decides: where all tokens share one expert beside their others, 100 tokens 73 / 72, 200 84 / 76.
// And so do products of less than 2^20 outputs and 2^31 multiplications, which end before the stream has begun in earnest: from memory / streamed, 64
// experts of 136 x 5376, 35 slots each 20 / 27; 8 of 1024 x 4096, 40 slots 18 / 24; 2 of 512 x 8192, 150 slots 18 / 26; 1 of 256 x 2048, 2000 slots
// 18 / 25; 96 of 72 x 800, 92 slots 18 / 21; and beyond: 2.0 M outputs of 992 22 / 21, 8.2 M of 256 31 / 20; 2048 x 7168, 40 slots 35 / 30 (24 slots
// 22 / 29, streamed all the same).
bool product_streams(int64_t S, int E, int64_t N, int64_t arows, int64_t K) {
    const int64_t Kp = (K + 255) / 256 * 256;
    if (arows * (Kp / 2) > 0xFFFFFFFFll || K > (1 << 24) || most_units(S, E, 256) * ceil_div64(N, 256) > 0x3FFFFFFF) return false;
    return S >= 16 * (int64_t)E && (S * N >= (1 << 20) || S * N >= (1ll << 31) / K);
}
// A streamed product whose tiles (as many as evenly filled experts have) fill half the chip or less has its contraction cut into parts, where
// the units that a tile is spared (1.1 us each, 1.6 where all CUs fetch other weights) outweigh the launch that joins them (5 us) and what
// the sums are written and read at.  us, cut / whole: 4 experts of 4096 x 14336, 64 slots each 44 / 79; 8 of 512 x 8192, 350 slots
// 39 / 64; 64 of 128 x 7520, 114 slots 40 / 60; 16 of 1024 x 4096, 64 slots 28 / 32; 8 of 1384 x 5312, 345 slots 47 / 51; and those left whole:
// 4 of 1024 x 4096, 1500 slots 48 / 43; 8 of 1024 x 2048, 150 slots 27 / 24.  Parts of 3 and 6 units at least: as 4; 1 to 2 us slower.
#define PART_LEAST 4                              // units
#define PART_TILES 256                            // tiles of all parts: a CU each, and the same on any chip, so that results are the same
int64_t parts_ld(int64_t N) { return (N + 3) / 4 * 4; }
struct Parts {
    int count, units;                             // count 1: not cut
};
Parts product_parts(int64_t S, int E, int64_t N, int64_t K) {
    const int64_t units = (K + 255) / 256, tiles = E * ceil_div64(S, 256 * (int64_t)E) * ceil_div64(N, 256);
    const int64_t room = PART_TILES / tiles, most = units / PART_LEAST, want = room < most ? room : most;
    if (want < 2) return {1, (int)units};
    const int64_t per = ceil_div64(units, want < PARTS_MAX ? want : PARTS_MAX);
    const int64_t count = ceil_div64(units, per);
    if (2 * (units - per - 6) < (count * S * N) >> 20) return {1, (int)units};
    return {(int)count, (int)per};
}
struct ProductPlace {
    int64_t Kp;                                   // K as the quantized rows have it
    size_t scales, wscales, parts, bytes;         // places of the rows' scales, of the weights' and of the parts' sums, and the end
    Parts cut;
};
// (a tile reads the scales of 256 rows wherever its own end)
ProductPlace product_place(bool stream, int64_t rows, int64_t S, int E, int64_t N, int64_t K) {
    const int64_t Kp = stream ? (K + 255) / 256 * 256 : K;
    ProductPlace p = {Kp, align_up((size_t)rows * Kp / 2, 256), 0, 0, 0, {1, 0}};
    p.wscales = p.bytes = p.scales + align_up((size_t)(stream ? S : rows) * Kp / 32, 256);
    if (stream) {
        p.cut = product_parts(S, E, N, K);
        p.parts = p.bytes = p.wscales + 2048 + align_up((size_t)E * N * Kp / 32, 256) + 2048;
        if (p.cut.count > 1) p.bytes += (size_t)p.cut.count * S * parts_ld(N) * 4;
    }
    return p;
}
template <bool UNITS>
int launch_quantize_rows(hipStream_t s, const metis_mat* A, int64_t Kp, uint8_t* codes, const RowScales& rs, const WeightScales& ws) {
    const int st = units_status(A->rows, Kp / 8);
    if (st != METIS_OK) return st;
    const int64_t total = A->rows * (Kp / 8), blocks = ceil_div64(total, 256), more = UNITS ? ceil_div64(ws.rows, 64) : 0;
    if (!grid_fits(blocks + more, 256)) return METIS_UNSUPPORTED;
    const FastDiv units = fast_div((uint32_t)(Kp / 8));
    auto launch = [&](auto kern, auto zero) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(blocks + more)), dim3(256), 0, s, (const decltype(zero)*)A->ptr, A->ld, A->cols, (uint64_t)total,
                           units, codes, rs, ws, (uint32_t)blocks);
    };
    if (A->dtype == METIS_BF16) launch(k_quantize_rows<bf16_t, UNITS>, bf16_t());
    else launch(k_quantize_rows<float, UNITS>, float());
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
template <typename OUT, int MODE>
int launch_stream(hipStream_t s, const ExStream& a, int64_t tiles, metis_mat* C, bool past) {
    const int cus = device_cu_count();
    if (cus < 1) return METIS_HIP_ERROR;
    auto launch = [&](auto kern, LdsLimitCache& lds_set) -> int {
        if (!ensure_dyn_lds((const void*)kern, EX_LDS, lds_set)) return METIS_HIP_ERROR;
        hipLaunchKernelGGL(kern, dim3((unsigned)(tiles < cus ? tiles : cus)), dim3(512), EX_LDS, s, a, (OUT*)C->ptr, C->ld, mat_aligned16(C));
        METIS_LAUNCH_CHECK();
        return METIS_OK;
    };
    static LdsLimitCache lds_set[2];
    if constexpr (MODE != EX_PRODUCT)
        if (!past) return launch(k_experts_stream<OUT, MODE, false>, lds_set[0]);
    if constexpr (MODE != EX_PARTS) return launch(k_experts_stream<OUT, MODE, true>, lds_set[1]);
    return METIS_INVALID_ARG;
}

}  // namespace

extern "C" int metis_quantize_mx_t(void* stream, const metis_mat* A, int groups, metis_mxfp4* out) {
    if (!mat_ok(A) || !out || !out->codes || !out->scales || groups < 1 || A->rows < 1 || A->cols < 1) return METIS_INVALID_ARG;
    if (A->cols >= 1ll << 30) return METIS_UNSUPPORTED;
    if (A->rows % groups || A->rows / groups % 32 || A->cols % 8 || A->ld < A->cols || !mat_aligned16(A) || (uintptr_t)out->codes % 16 ||
        out->rows != groups * A->cols || out->cols != A->rows / groups)
        return METIS_BAD_SHAPE;
    return launch_quantize_mx_t((hipStream_t)stream, turn_side(A, nullptr, false, out->codes, out->scales), {}, A->dtype, nullptr, false,
                                A->rows / groups);
}

extern "C" size_t metis_experts_workspace_bytes(int64_t rows, int64_t slots, int experts, int64_t N, int64_t K) {
    if (rows < 1 || slots < 1 || experts < 1 || experts > EXPERTS_MAX || N < 1 || N > (1ll << 40) || K < 32 || K % 32 || K > (1 << 28)) return 0;
    return product_place(product_streams(slots, experts, N, rows, K), rows, slots, experts, N, K).bytes;
}

extern "C" int metis_experts_product(void* stream, const metis_mat* A, const metis_mxfp4* W, const metis_expert_plan* plan, int gather,
                                     metis_mat* C, void* workspace, size_t workspace_bytes) {
    const int st = experts_plan_status(plan);
    if (st != METIS_OK) return st;
    if (plan->tokens == 0) return METIS_OK;
    if (!mat_ok(A) || !W || !W->codes || !W->scales || !mat_ok(C) || (gather && (!plan->token || !plan->slot))) return METIS_INVALID_ARG;
    const int64_t S = plan->tokens * plan->k, K = W->cols, N = W->rows / plan->experts;
    const int E = plan->experts;
    if (K < 32 || K % 32 || W->rows < 1 || W->rows % E || A->cols != K || A->ld < K || A->rows != (gather ? plan->tokens : S) ||
        C->rows != S || C->cols != N || C->ld < N || !mat_aligned16(A) || (uintptr_t)W->codes % 16 || (uintptr_t)W->scales % 8)
        return METIS_BAD_SHAPE;
    if (K > (1 << 28) || N > (1ll << 40)) return METIS_UNSUPPORTED;
    if (!workspace || workspace_bytes < metis_experts_workspace_bytes(A->rows, S, E, N, K)) return METIS_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace % 256) return METIS_INVALID_ARG;
    const bool streams = product_streams(S, E, N, A->rows, K);
    const ProductPlace place = product_place(streams, A->rows, S, E, N, K);
    uint8_t* ws = (uint8_t*)workspace;
    hipStream_t s = (hipStream_t)stream;
    if (streams) {
        const int us = place.cut.count > 1 ? units_status(S, parts_ld(N) / 4) : METIS_OK;
        if (us != METIS_OK) return us;
        const int qs = launch_quantize_rows<true>(s, A, place.Kp, ws, {ws + place.scales, gather ? plan->slot : nullptr, S, gather ? plan->k : 1},
                                                  {W->scales, ws + place.wscales + 2048, W->rows, (int)(K / 32), (int)(place.Kp / 256)});
        if (qs != METIS_OK) return qs;
        const int tn = (int)ceil_div64(N, 256);
        const ExStream a = {{ws, ws + place.scales}, {W->codes, ws + place.wscales + 2048}, plan->offsets, gather ? plan->token : nullptr, S,
                            A->rows, N, K, (uint32_t)(place.Kp / 2), 8 * S, 8 * W->rows, E, 0, tn, place.cut.count, place.cut.units};
        const int64_t tiles = most_units(S, E, 256) * tn * place.cut.count;
        if (place.cut.count > 1) {
            const int64_t ld = parts_ld(N), total = S * (ld / 4);
            float* const sums = (float*)(ws + place.parts);
            metis_mat P = *C;
            P.ptr = sums;
            P.ld = ld;
            const int ss = launch_stream<float, EX_PARTS>(s, a, tiles, &P, false);
            if (ss != METIS_OK) return ss;
            auto join = [&](auto zero) {
                typedef decltype(zero) OUT;
                hipLaunchKernelGGL(k_experts_join<OUT>, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s, sums, ld, place.cut.count,
                                   plan->offsets, E, S, N, (uint64_t)total, fast_div((uint32_t)(ld / 4)), (OUT*)C->ptr, C->ld,
                                   (uintptr_t)C->ptr % (4 * sizeof(OUT)) == 0 && C->ld % 4 == 0);
            };
            if (C->dtype == METIS_BF16) join(bf16_t());
            else join(float());
            METIS_LAUNCH_CHECK();
            return METIS_OK;
        }
        return C->dtype == METIS_BF16 ? launch_stream<bf16_t, EX_PRODUCT>(s, a, tiles, C, true) : launch_stream<float, EX_PRODUCT>(s, a, tiles, C, true);
    }
    const int nblk = (int)(K / 32);
    const int64_t most = most_units(S, E, 32) + 1;
    // The contraction is split where there are few waves (not counting that a unit may not exist).  us, split / not, 8 experts of 2048 x 7168,
    // two a token: one token 13.7 / 19.7, 8 18.2 / 29.0, 64 20.4 / 32.7; 64 of 2048 x 4096, four a token: 2 tokens 13.9 / 15.5, 8 29.1 /
    // 29.2, 16 45.9 / 41.8, 24 58.3 / 56.5, 200 83.4 / 74.1; 4096 x 1024, 24 tokens 44.2 / 26.6; and 128 of 1024 x 2048, eight a token, where it
    // loses a little: 8 tokens 23.4 / 19.0.
    const bool split = most * ceil_div64(N, 32) < 4096;
    const int64_t nb = ceil_div64(N, split ? 32 : 128);
    if (!grid_fits(most * nb, 256)) return METIS_UNSUPPORTED;
    const size_t row_lds = (size_t)few_code_row(nblk) + few_scale_row(nblk), lds = row_lds * (S < 32 ? S : 32);
    // Quantized on the spot where an expert has 8192 elements or fewer on average, and the rows of a full unit leave room for four
    // workgroups a CU.  us, with the quantizer's launch / on the spot, 2048 x 4096 with 64 experts of which a token takes four: one token
    // 18.7 / 16.9, two 19.0 / 15.5, 64 64.0 / 68.6, 200 74.3 / 97.9; 4096 x 1024, 24 tokens 27.3 / 24.7.  Rows of 70 KB, 8 tokens: 25.7 / 43.0.
    const bool fuse = S * K <= 8192 * (S < E ? S : E) && lds <= 24 * 1024;
    if (!fuse) {
        const int qs = launch_quantize_rows<false>(s, A, K, ws, {ws + place.scales, nullptr, 0, 0}, {});
        if (qs != METIS_OK) return qs;
    }
    const int64_t size = mat_size(C);
    const bool vec = (uintptr_t)C->ptr % (4 * size) == 0 && C->ld % 4 == 0;
    auto launch = [&](auto kern, auto zero, size_t dyn) {
        hipLaunchKernelGGL(kern, dim3((unsigned)(most * nb)), dim3(256), dyn, s, MxRows{ws, ws + place.scales}, DenseRows{A->ptr, A->ld}, A->rows,
                           MxRows{W->codes, W->scales}, plan->offsets, gather ? plan->token : nullptr, E, S, N, nblk, (decltype(zero)*)C->ptr,
                           C->ld, vec, (uint32_t)nb, (uint32_t)most);
    };
    auto fused = [&](auto zero, auto in, auto split_) {
        typedef decltype(in) T;
        auto kern = k_experts_few<decltype(zero), decltype(split_)::value, T>;
        launch(kern, zero, lds);
    };
    auto by_shape = [&](auto zero) {
        typedef decltype(zero) OUT;
        if (fuse) {
            const bool bf = A->dtype == METIS_BF16;
            if (split) bf ? fused(zero, bf16_t(), std::true_type{}) : fused(zero, float(), std::true_type{});
            else bf ? fused(zero, bf16_t(), std::false_type{}) : fused(zero, float(), std::false_type{});
        } else {
            split ? launch(k_experts_few<OUT, true>, zero, 0) : launch(k_experts_few<OUT, false>, zero, 0);
        }
    };
    if (C->dtype == METIS_BF16) by_shape(bf16_t());
    else by_shape(float());
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" size_t metis_experts_wgrad_workspace_bytes(int64_t slots, int experts, int64_t N, int64_t K) {
    if (slots < 1 || slots > (1 << 25) || experts < 1 || experts > EXPERTS_MAX || N < 1 || N > (1 << 28) || K < 1 || K > (1 << 28)) return 0;
    const int64_t P = padded_slots(slots, experts);
    return mx_bytes(N, P) + mx_bytes(K, P);
}

extern "C" int metis_experts_wgrad(void* stream, const metis_mat* G, const metis_mat* X, const metis_expert_plan* plan, int gather,
                                   metis_mat* dW, void* workspace, size_t workspace_bytes) {
    const int st = experts_plan_status(plan);
    if (st != METIS_OK) return st;
    const int64_t S = plan->tokens * plan->k, E = plan->experts;
    if (!G || !X || !mat_ok(dW) || (S > 0 && (!mat_ok(G) || !mat_ok(X) || (gather && !plan->token)))) return METIS_INVALID_ARG;
    const int64_t N = G->cols, K = X->cols;
    if (N < 1 || K < 1 || N % 8 || K % 8 || G->rows != S || X->rows != (gather ? plan->tokens : S) || dW->rows != E * N || dW->cols != K ||
        dW->ld < K)
        return METIS_BAD_SHAPE;
    if (S > 0 && (G->ld < N || X->ld < K || !mat_aligned16(G) || !mat_aligned16(X))) return METIS_BAD_SHAPE;
    if (S > (1 << 25) || N > (1 << 28) || K > (1 << 28)) return METIS_UNSUPPORTED;
    const int64_t tm = ceil_div64(N, 256), tn = ceil_div64(K, 256), tiles = E * tm * tn;
    const bool brief = wgrad_short(S, (int)E, dW->dtype);
    if (tiles > 0x3FFFFFFF || (brief && !grid_fits(ceil_div64(N, 128) * tn, 256))) return METIS_UNSUPPORTED;
    const size_t need = metis_experts_wgrad_workspace_bytes(S, (int)E, N, K);
    if (workspace_bytes < need || (need && !workspace)) return METIS_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace % 256) return METIS_INVALID_ARG;
    const int64_t P = S > 0 ? padded_slots(S, (int)E) : 0;
    uint8_t* w = (uint8_t*)workspace;
    const MxRows g = {w, w + align_up((size_t)N * P / 2, 256)};
    w += mx_bytes(N, P);
    const MxRows x = {w, w + align_up((size_t)K * P / 2, 256)};
    hipStream_t s = (hipStream_t)stream;
    if (S > 0) {
        const TurnSide sg = turn_side(G, nullptr, brief, (uint8_t*)g.codes, (uint8_t*)g.scales);
        const TurnSide sx = turn_side(X, gather ? plan->token : nullptr, brief, (uint8_t*)x.codes, (uint8_t*)x.scales);
        const bool same = G->dtype == X->dtype;
        int r = launch_quantize_mx_t(s, sg, same ? sx : TurnSide{}, G->dtype, plan, brief, 0);
        if (r == METIS_OK && !same) r = launch_quantize_mx_t(s, sx, {}, X->dtype, plan, brief, 0);
        if (r != METIS_OK) return r;
    }
    const bool past = (uintptr_t)dW->ptr % 128 == 0 && dW->ld * mat_size(dW) % 128 == 0;
    if (brief) {
        const int64_t sn = ceil_div64(N, 128), sk = ceil_div64(K, 256);
        auto launch = [&](auto kern, auto zero) {
            hipLaunchKernelGGL(kern, dim3((unsigned)(sn * sk), (unsigned)E), dim3(256), 0, s, g, x, plan->offsets, (int)E, S, N, K,
                               (decltype(zero)*)dW->ptr, dW->ld, mat_aligned16(dW), (uint32_t)sk);
        };
        if (dW->dtype == METIS_BF16) past ? launch(k_experts_short<bf16_t, true>, bf16_t()) : launch(k_experts_short<bf16_t, false>, bf16_t());
        else past ? launch(k_experts_short<float, true>, float()) : launch(k_experts_short<float, false>, float());
        METIS_LAUNCH_CHECK();
        return METIS_OK;
    }
    const ExStream a = {g, x, plan->offsets, nullptr, S, 0, N, K, 0, 8 * N, 8 * K, (int)E, (int)tm, (int)tn};
    return dW->dtype == METIS_BF16 ? launch_stream<bf16_t, EX_WGRAD>(s, a, tiles, dW, past) : launch_stream<float, EX_WGRAD>(s, a, tiles, dW, past);
}
