// Layer norm of rows, and its gradients.
#include "column_sums.h"

namespace {

// A row belongs to RT threads, each of which holds U units of eight neighbouring elements in registers: unit u of thread t starts at column
// 8 (t + RT u).  RT 64: a workgroup of 256 has four rows, else one.  Workgroups go through the rows with the weights in registers and the next row
// on its way.  Whole vectors everywhere: a row's last unit, where it is short, lies at the row's end and has its first elements in common with the unit
// before it, and units behind the row are that unit once more.  What a thread has twice (`twice` elements of a unit, the first ones) stays out of
// the sums, and is stored twice with the same bits.  No load or store in the loops is under a condition: the wait for the next row would wait for
// this row's stores too, which come behind it in the queue, where the compiler cannot count them.  Rows of fewer than eight elements go to the kernels for long ones, which look at each.
template <int RT>
struct RowGroup {
    static constexpr int THREADS = RT < 256 ? 256 : RT, ROWS = THREADS / RT, WAVES = RT / 64;
};
// the wave's sum, the same in all lanes: within each 16 lanes by swaps, then the four in their order
__device__ __forceinline__ float wave_sum(float v) {
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
        v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    add(std::integral_constant<int, 0xB1>{});                     // lanes 1 0 3 2
    add(std::integral_constant<int, 0x4E>{});                     // 2 3 0 1
    add(std::integral_constant<int, 0x141>{});                    // halves of eight mirrored
    add(std::integral_constant<int, 0x140>{});                    // sixteen mirrored
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) s += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 16 * i + 15));
    return s;
}
// the sum of each 16 lanes, the same in all of them
__device__ __forceinline__ double sixteen_sum(double v) {
    auto half = [&](uint32_t h, auto ctrl) __attribute__((always_inline)) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)h, decltype(ctrl)::value, 0xF, 0xF, true);
    };
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
        const uint64_t w = __builtin_bit_cast(uint64_t, v);
        v += __builtin_bit_cast(double, (uint64_t)half((uint32_t)(w >> 32), ctrl) << 32 | half((uint32_t)w, ctrl));
    };
    add(std::integral_constant<int, 0xB1>{});
    add(std::integral_constant<int, 0x4E>{});
    add(std::integral_constant<int, 0x141>{});
    add(std::integral_constant<int, 0x140>{});
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, sixteen_sum(v));
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)w, 16 * i + 15);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(w >> 32), 16 * i + 15);
        s += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    return s;
}
// Sums of N values over a row's threads.  slot: LDS of N * WAVES values, not written again before the workgroup has met once more.
template <int RT, int N, typename V>
__device__ __forceinline__ void row_sums(V (&v)[N], V* slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (RT > 64) {
        constexpr int W = RT / 64;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) slot[i * W + wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (W == 16 && sizeof(V) == 8) {                // (sixteen reads and additions one behind the other take longer)
                v[i] = sixteen_sum(slot[i * W + (threadIdx.x & 15)]);
                continue;
            }
            V s = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) s += slot[i * W + w];
            v[i] = s;
        }
    }
}
// A row's mean, from a sum in 64 bits, as two fp32 numbers: elements near each other keep all of their differences to it, however far from zero they are.  A row of
// equal elements has that element as its mean, and no lower part: the sum is exact, and the quotient is once it is corrected.  variance: from the sum of
// (v - hi)^2, of whose mean lo^2 is at most half.
struct RowLength {
    double n, inverse;
    __device__ __forceinline__ RowLength(int64_t cols) : n((double)cols), inverse(1.0 / n) {}
};
struct RowMean {
    float hi, lo;
    __device__ __forceinline__ RowMean(double sum, const RowLength& row) {
        const double near = sum * row.inverse, mean = fma(fma(-near, row.n, sum), row.inverse, near);
        hi = (float)(mean == mean ? mean : near);                     // (infinite sums)
        lo = (float)(mean - (double)hi);
    }
    __device__ __forceinline__ float variance(double squares, const RowLength& row) const { return fmaf(-lo, lo, (float)(squares * row.inverse)); }
};
// The sum of a unit's elements.  bf16: in fp32, which loses nothing unless they are more than 2^13 times apart (8 bits each), and is then off by
// 2^-24 of the largest; an eighth of it, which is in fp32's range where they are.
template <typename T>
__device__ __forceinline__ double unit_sum(const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        float s = v[0] * 0.125f;
#pragma unroll
        for (int i = 1; i < 8; ++i) s = fmaf(v[i], 0.125f, s);
        return 8.0 * s;
    } else {
        double s = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) s += v[i];
        return s;
    }
}
__device__ __forceinline__ float unit_squares(const float (&v)[8]) {
    float s = v[0] * v[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) s = fmaf(v[i], v[i], s);
    return s;
}
// v, zeros in place of the first `twice`
__device__ __forceinline__ void unit_own(const float (&v)[8], int twice, float (&own)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) own[i] = i >= twice ? v[i] : 0.0f;
}
// Nothing is on its way into a loop from before it: what the loop waits for is then counted from its own loads and stores alone.
__device__ __forceinline__ void loads_arrived() { __builtin_amdgcn_s_waitcnt(0xF70); }     // vmcnt(0)
struct UnitPlace {
    int64_t c;
    int twice;                                // 8: a unit behind the row
};
template <int RT>
__device__ __forceinline__ UnitPlace unit_place(int t, int u, int64_t cols) {
    const int64_t c = 8 * (int64_t)(t + RT * u), last = cols - 8;
    return c <= last ? UnitPlace{c, 0} : UnitPlace{last, c - last < 8 ? (int)(c - last) : 8};
}
__device__ __forceinline__ void load_factors(const float* p, float none, float (&v)[8]) {
    if (p) {
        load_row<true>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
    }
}

// Two passes over what the registers hold, mean first (RowMean), so that a mean far from zero costs neither the variance nor the results anything.
// Memory bounds it: 16384 x 4096 bf16 (268 MB) takes 43.6 us, 6.2 TB/s (part of the rows is still in the last-level cache).
template <typename T, int RT, int U>
__global__ void __launch_bounds__(RowGroup<RT>::THREADS)
k_layernorm(const T* x, int64_t ldx, T* y, int64_t ldy, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
            float2* __restrict__ stats, int64_t rows, int64_t cols) {
    typedef RowGroup<RT> G;
    __shared__ double s_mean[G::WAVES];
    __shared__ float s_var[G::WAVES];
    const int t = RT == 64 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
    const int own = RT == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
    const RowLength length(cols);
    const bool units = cols % 8 == 0;                            // (nothing is held twice but whole units: no element is looked at)
    float w[U][8], b[U][8];
    UnitPlace at[U];
    RawUnit<T> next[U];
    const int64_t hop = (int64_t)gridDim.x * G::ROWS;
    int64_t r = (int64_t)blockIdx.x * G::ROWS + own;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = unit_place<RT>(t, u, cols);
        if (r < rows) load_whole(x + r * ldx + at[u].c, next[u]);
        load_factors(weight ? weight + at[u].c : nullptr, 1.0f, w[u]);
        load_factors(bias ? bias + at[u].c : nullptr, 0.0f, b[u]);
    }
    loads_arrived();
    for (; r < rows; r += hop) {
        float v[U][8], sum[1] = {0.0f};
        double whole[1] = {0.0};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unpack(next[u], v[u]);
            load_whole(x + (r + hop < rows ? r + hop : r) * ldx + at[u].c, next[u]);
            float own[8];
            if (!units) unit_own(v[u], at[u].twice, own);
            const double s = units ? unit_sum<T>(v[u]) : unit_sum<T>(own);
            whole[0] += at[u].twice < 8 ? s : 0.0;
        }
        row_sums<RT>(whole, s_mean);
        const RowMean mean(whole[0], length);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] -= mean.hi;
            float own[8];
            if (!units) unit_own(v[u], at[u].twice, own);
            const float s = units ? unit_squares(v[u]) : unit_squares(own);
            sum[0] += at[u].twice < 8 ? s : 0.0f;
        }
        row_sums<RT>(sum, s_var);
        const float rstd = 1.0f / sqrtf(mean.variance(sum[0], length) + eps), low = -mean.lo * rstd;
        if (stats && t == 0) stats[r] = make_float2(mean.hi, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[u][i] = fmaf(fmaf(v[u][i], rstd, low), w[u][i], b[u][i]);
            store_row<true>(y + r * ldy + at[u].c, v[u]);
        }
    }
}

// Rows longer than what registers hold: three passes over the row, which stays in the caches.  Sums in 64 bits: a thread has up to 2^18 of their terms.
template <typename T>
__global__ void __launch_bounds__(1024)
k_layernorm_long(const T* x, int64_t ldx, T* y, int64_t ldy, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
                 float2* __restrict__ stats, int64_t rows, int64_t cols) {
    __shared__ double s_mean[16], s_var[16];
    const RowLength length(cols);
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        double sum[1] = {0.0};
        float v[8];
        auto each = [&](auto f) __attribute__((always_inline)) {
            for (int64_t c = 8 * (int64_t)threadIdx.x; c < cols; c += 8192) {
                load_unit(x + r * ldx + c, cols - c, v);
                f(c);
            }
        };
        each([&](int64_t) { sum[0] += unit_sum<T>(v); });
        row_sums<1024>(sum, s_mean);
        const RowMean mean(sum[0], length);
        sum[0] = 0.0;
        each([&](int64_t c) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = c + i < cols ? v[i] - mean.hi : 0.0f;
            sum[0] += unit_squares(d);
        });
        row_sums<1024>(sum, s_var);
        const float rstd = 1.0f / sqrtf(mean.variance(sum[0], length) + eps), low = -mean.lo * rstd;
        if (stats && threadIdx.x == 0) stats[r] = make_float2(mean.hi, rstd);
        each([&](int64_t c) {
            float w[8] = {1, 1, 1, 1, 1, 1, 1, 1}, b[8] = {};
            if (weight) load_unit(weight + c, cols - c, w);
            if (bias) load_unit(bias + c, cols - c, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(fmaf(v[i] - mean.hi, rstd, low), w[i], b[i]);
            store_part<T, true>(y + r * ldy + c, cols - c, v);
        });
    }
}

// ---- gradients ----
// xh = (x - mean) rstd, g = dy w:  dx = add + rstd (g - mean of g - xh * mean of g xh).  Both means come from one pass over what the registers
// hold; the columns' sums of dy xh and dy stay in registers over all the rows of a workgroup, and leave as one row of `sums` [gridDim.x, 2 cols].
// Memory bounds it: 16384 x 4096 bf16 with `add` (537 MB) takes 93 us, 5.8 TB/s, and the sums' join 2.4 (with the rows' loads where they are used, not a
// row ahead, 160).
template <typename T, int RT, int U, bool ADD>
__device__ __forceinline__ void norm_grads_rows(const T* dy, int64_t ldd, const T* x, int64_t ldx, const float2* __restrict__ stats,
                                                const float* __restrict__ weight, const T* add, int64_t lda, T* dx, int64_t ldo, int64_t rows,
                                                int64_t cols, float* __restrict__ sums, uint32_t block, uint32_t blocks) {
    typedef RowGroup<RT> G;
    constexpr bool AHEAD = RT * U <= 1024;               // (of 16384 columns a thread has no registers for the next row and the weights)
    __shared__ float s_sum[2][2 * G::WAVES], s_join[RT == 64 ? 3 * 512 : 1];
    const int t = RT == 64 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
    const int own = RT == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
    const float n = (float)cols;
    float w[U][8], dw[U][8], db[U][8];
    UnitPlace at[U];
    RawUnit<T> nx[U], nd[U], na[U];
    float2 nst = make_float2(0.0f, 0.0f);
    const int64_t hop = (int64_t)blocks * G::ROWS;
    int64_t r = (int64_t)block * G::ROWS + own;
    auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        nst = stats[row];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            load_whole(x + row * ldx + at[u].c, nx[u]);
            load_whole(dy + row * ldd + at[u].c, nd[u]);
            if (ADD) load_whole(add + row * lda + at[u].c, na[u]);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = unit_place<RT>(t, u, cols);
    if (AHEAD && r < rows) fetch(r);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (AHEAD) load_factors(weight ? weight + at[u].c : nullptr, 1.0f, w[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[u][i] = db[u][i] = 0.0f;
    }
    loads_arrived();
    for (int turn = 0; r < rows; r += hop, turn ^= 1) {
        float xh[U][8], g[U][8], sum[2] = {0.0f, 0.0f};
        RawUnit<T> plus[U];
        if (!AHEAD) fetch(r);
        const float2 st = nst;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unpack(nx[u], xh[u]);
            unpack(nd[u], g[u]);
            plus[u] = na[u];
        }
        if (AHEAD) fetch(r + hop < rows ? r + hop : r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!AHEAD) load_factors(weight ? weight + at[u].c : nullptr, 1.0f, w[u]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                xh[u][i] = (xh[u][i] - st.x) * st.y;
                dw[u][i] = fmaf(g[u][i], xh[u][i], dw[u][i]);
                db[u][i] += g[u][i];
                g[u][i] *= w[u][i];
                sum[0] += i >= at[u].twice ? g[u][i] : 0.0f;
                sum[1] = i >= at[u].twice ? fmaf(g[u][i], xh[u][i], sum[1]) : sum[1];
            }
        }
        row_sums<RT>(sum, s_sum[turn]);
        const float mg = sum[0] / n, mx = sum[1] / n;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float a[8] = {};
            if (ADD) unpack(plus[u], a);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = fmaf(st.y, g[u][i] - mg - xh[u][i] * mx, a[i]);
            store_row<true>(dx + r * ldo + at[u].c, a);
        }
    }
    if (!sums) return;
    float* out = sums + (int64_t)block * 2 * cols;
    auto leave = [&](float (&s)[U][8], float* to) __attribute__((always_inline)) {
        if constexpr (RT == 64) {                                                     // the four waves' sums in their order
            __syncthreads();
            if (own > 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s_join[(own - 1) * 512 + 64 * i + t] = s[0][i];
            }
            __syncthreads();
            if (own > 0) return;
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0][i] += s_join[p * 512 + 64 * i + t];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (at[u].twice < 8) store_row<true>(to + at[u].c, s[u]);
    };
    leave(dw, out);
    leave(db, out + cols);
}

template <typename T, int RT, int U, bool ADD>
__global__ void __launch_bounds__(RowGroup<RT>::THREADS)
k_layernorm_grads(const T* dy, int64_t ldd, const T* x, int64_t ldx, const float2* __restrict__ stats, const float* __restrict__ weight,
                  const T* add, int64_t lda, T* dx, int64_t ldo, int64_t rows, int64_t cols, float* __restrict__ sums) {
    norm_grads_rows<T, RT, U, ADD>(dy, ldd, x, ldx, stats, weight, add, lda, dx, ldo, rows, cols, sums, blockIdx.x, gridDim.x);
}

// Few rows, one launch: the first `strips` workgroups have 8 W columns each, 16 or, of longer rows, 64, and go down all the rows, 128 at a time,
// for the columns' sums; the others have rows.  (Both read x and dy: where dx takes the place of one, the rows follow in a launch of their own.)
template <typename T, int RT, int U, bool ADD>
__global__ void __launch_bounds__(RowGroup<RT>::THREADS)
k_layernorm_grads_few(const T* dy, int64_t ldd, const T* x, int64_t ldx, const float2* __restrict__ stats, const float* __restrict__ weight,
                      const T* add, int64_t lda, T* dx, int64_t ldo, int64_t rows, int64_t cols, float* dweight, float* dbias, uint32_t strips) {
    constexpr int WAVES = RowGroup<RT>::THREADS / 64, STEP = 128, W = RowGroup<RT>::THREADS / STEP;
    if (blockIdx.x >= strips) {
        norm_grads_rows<T, RT, U, ADD>(dy, ldd, x, ldx, stats, weight, add, lda, dx, ldo, rows, cols, nullptr, blockIdx.x - strips, gridDim.x - strips);
        return;
    }
    const uint32_t strip = xcd_strip(blockIdx.x, strips);
    __shared__ float s_columns[2 * 8 * W * WAVES];
    const int64_t c = 8 * W * (int64_t)strip + 8 * (threadIdx.x % W);
    const int back = unit_back(c, cols);
    float dw[8] = {}, db[8] = {};
    int64_t r = threadIdx.x / W;
    if (c < cols && r < rows) {
        RawUnit<T> nx, nd;
        float2 nst;
        auto fetch = [&](int64_t row) __attribute__((always_inline)) {
            nst = stats[row];
            load_whole(x + row * ldx + (c - back), nx);
            load_whole(dy + row * ldd + (c - back), nd);
        };
        fetch(r);
        for (; r < rows; r += STEP) {
            float v[8], g[8];
            const float2 st = nst;
            unpack(nx, back, v);
            unpack(nd, back, g);
            fetch(r + STEP < rows ? r + STEP : r);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[i] = fmaf(g[i], (v[i] - st.x) * st.y, dw[i]);
                db[i] += g[i];
            }
        }
    }
    if (dweight) group_columns<WAVES, W>(dw, s_columns, dweight, strip, cols);
    if (dbias) group_columns<WAVES, W>(db, s_columns + 8 * W * WAVES, dbias, strip, cols);
}

// Long rows: two passes over a row for its gradient, and the columns' sums by a kernel that goes down the columns.
template <typename T>
__global__ void __launch_bounds__(1024)
k_layernorm_grads_long(const T* dy, int64_t ldd, const T* x, int64_t ldx, const float2* __restrict__ stats, const float* __restrict__ weight,
                       const T* add, int64_t lda, T* dx, int64_t ldo, int64_t rows, int64_t cols) {
    __shared__ float s_sum[2][32];
    const float n = (float)cols;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x, turn ^= 1) {
        const float2 st = stats[r];
        float sum[2] = {0.0f, 0.0f}, xh[8], g[8];
        auto each = [&](auto f) __attribute__((always_inline)) {
            for (int64_t c = 8 * (int64_t)threadIdx.x; c < cols; c += 8192) {
                float w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
                load_unit(x + r * ldx + c, cols - c, xh);
                load_unit(dy + r * ldd + c, cols - c, g);                   // (zeros behind the row)
                if (weight) load_unit(weight + c, cols - c, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    xh[i] = (xh[i] - st.x) * st.y;
                    g[i] = c + i < cols ? g[i] * w[i] : 0.0f;
                }
                f(c);
            }
        };
        each([&](int64_t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum[0] += g[i];
                sum[1] = fmaf(g[i], xh[i], sum[1]);
            }
        });
        row_sums<1024>(sum, s_sum[turn]);
        const float mg = sum[0] / n, mx = sum[1] / n;
        each([&](int64_t c) {
            float a[8] = {};
            if (add) load_unit(add + r * lda + c, cols - c, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = fmaf(st.y, g[i] - mg - xh[i] * mx, a[i]);
            store_part<T, true>(dx + r * ldo + c, cols - c, a);
        });
    }
}
// a workgroup has 512 columns of `chunk` rows
template <typename T>
__global__ void __launch_bounds__(256)
k_layernorm_columns(const T* __restrict__ dy, int64_t ldd, const T* __restrict__ x, int64_t ldx, const float2* __restrict__ stats, int64_t rows,
                    int64_t cols, int64_t chunk, float* __restrict__ sums) {
    __shared__ float s_join[2 * 3 * 512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t c = 512 * (int64_t)blockIdx.x + 8 * lane, n = cols - c;
    const int64_t first = chunk * blockIdx.y, end = first + chunk < rows ? first + chunk : rows;
    float s[2][8] = {};
    if (n > 0) {
        for (int64_t r = first + wave; r < end; r += 4) {
            const float2 st = stats[r];
            float v[8], g[8];
            load_unit(x + r * ldx + c, n, v);
            load_unit(dy + r * ldd + c, n, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[0][i] = fmaf(g[i], (v[i] - st.x) * st.y, s[0][i]);
                s[1][i] += g[i];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (wave > 0) s_join[(3 * k + wave - 1) * 512 + 64 * i + lane] = s[k][i];
    __syncthreads();
    if (wave > 0 || n <= 0) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[k][i] += s_join[(3 * k + p) * 512 + 64 * i + lane];
        store_part<float, true>(sums + (blockIdx.y * 2 + k) * cols + c, n, s[k]);
    }
}

#define NORM_REGS 16384                           // longest row that a workgroup keeps, with its columns' sums, in registers
// Workgroups of the gradients' kernel at most, each of which leaves a row of partial sums: one a CU, and the same on any chip so that the sums have the
// same order.  More lose what their partial sums cost: 16384 x 4096 bf16 with `add`, us: 192 113, 256 97, 384 108, 512 108, 1024 119; 1111 x 2057 fp32:
// 128 15.3, 256 13.5, 512 16.0.
#define NORM_PARTS 256

bool in_registers(int64_t cols) { return cols >= 8 && cols <= NORM_REGS; }
int64_t norm_rows(int64_t cols) { return cols <= 512 ? 4 : 1; }          // rows of a workgroup at a time
int64_t norm_parts(int64_t rows, int64_t cols) {
    const int64_t groups = ceil_div64(rows, norm_rows(cols));
    return groups < NORM_PARTS ? groups : NORM_PARTS;
}
int64_t column_chunk(int64_t rows, int64_t cols) {                       // rows of a workgroup of k_layernorm_columns
    const int64_t chunks = ceil_div64(2048, ceil_div64(cols, 512)), chunk = ceil_div64(rows, chunks);
    return chunk < 32 ? 32 : chunk;
}
int64_t sum_rows(int64_t rows, int64_t cols) {
    return in_registers(cols) ? norm_parts(rows, cols) : ceil_div64(rows, column_chunk(rows, cols));
}
// Few rows: one launch.  us, two launches / one, fp32: 128 x 4096 9.3 / 5.2, 512 x 4096 13.9 / 9.0, 700 x 4096 14.6 / 12.3, 1000 x 4096 16.2 / 17.5,
// 512 x 14336 29.8 / 28.2, 1000 x 256 8.8 / 6.6, 1111 x 2057 13.7 / 12.4, 1500 x 1000 10.9 / 12.0, 2000 x 256 7.4 / 9.0; bf16: 4 x 4096 6.7 / 4.7,
// 512 x 14336 23.4 / 17.5, 1000 x 6000 17.6 / 13.9.
bool norm_few(int64_t rows, int64_t cols, int64_t size) {
    return in_registers(cols) && (rows <= 512 || (rows <= 1280 && rows * cols * size <= 12 << 20));
}
// the threads of a row and the units of a thread: f(threads, units)
template <typename F>
void by_length(int64_t cols, F f) {
    if (cols <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    else if (cols <= 2048) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
    else if (cols <= 4096) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    else if (cols <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
    else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}
bool norm_mat(const metis_mat* m, const metis_mat* like) {
    return m->rows == like->rows && m->cols == like->cols && m->ld >= m->cols;
}
int norm_limits(int64_t rows, int64_t cols) { return cols > (1 << 28) || rows > 0xFFFFFFFFll ? METIS_UNSUPPORTED : METIS_OK; }

}  // namespace

extern "C" int metis_layernorm(void* stream, const metis_mat* x, const float* weight, const float* bias, float eps, metis_mat* y, float* stats) {
    if (!x || !y || !(eps >= 0.0f) || (uintptr_t)weight % 4 || (uintptr_t)bias % 4 || (uintptr_t)stats % 8) return METIS_INVALID_ARG;
    if (x->rows == 0 && y->rows == 0) return METIS_OK;
    if (!mat_ok(x) || !mat_ok(y) || x->dtype != y->dtype) return METIS_INVALID_ARG;
    if (x->rows < 1 || x->cols < 1 || !norm_mat(x, x) || !norm_mat(y, x)) return METIS_BAD_SHAPE;
    const int64_t rows = x->rows, cols = x->cols;
    const int st = norm_limits(rows, cols);
    if (st != METIS_OK) return st;
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        auto go = [&](auto kern, int threads, int64_t groups, int64_t most) {
            hipLaunchKernelGGL(kern, dim3((unsigned)(groups < most ? groups : most)), dim3(threads), 0, s, (const T*)x->ptr, x->ld, (T*)y->ptr,
                               y->ld, weight, bias, eps, (float2*)stats, rows, cols);
        };
        if (!in_registers(cols)) return go(k_layernorm_long<T>, 1024, rows, 512);
        by_length(cols, [&](auto rt, auto u) {
            constexpr int RT = decltype(rt)::value;
            go(k_layernorm<T, RT, decltype(u)::value>, RowGroup<RT>::THREADS, ceil_div64(rows, RowGroup<RT>::ROWS), RT == 1024 ? 512 : 2048);
        });
    };
    if (x->dtype == METIS_BF16) launch(bf16_t());
    else launch(float());
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

extern "C" size_t metis_layernorm_grads_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || norm_limits(rows, cols) != METIS_OK) return 0;
    if (norm_few(rows, cols, 4)) return 0;                // (of either type)
    return align_up((size_t)sum_rows(rows, cols) * 2 * cols * 4, 256);
}

extern "C" int metis_layernorm_grads(void* stream, const metis_mat* dy, const metis_mat* x, const float* stats, const float* weight,
                                     const metis_mat* add, metis_mat* dx, float* dweight, float* dbias, void* workspace, size_t workspace_bytes) {
    if (!dy || !x || !dx || (uintptr_t)weight % 4 || (uintptr_t)dweight % 4 || (uintptr_t)dbias % 4 || (uintptr_t)stats % 8) return METIS_INVALID_ARG;
    const int64_t rows = x->rows, cols = x->cols;
    const bool columns = dweight || dbias;
    hipStream_t s = (hipStream_t)stream;
    if (rows == 0 && dy->rows == 0 && dx->rows == 0) {
        if (cols < 1 || cols > (1 << 28)) return cols < 1 ? METIS_BAD_SHAPE : METIS_UNSUPPORTED;
        int r = dweight ? launch_clear(s, dweight, cols) : METIS_OK;
        if (r == METIS_OK && dbias) r = launch_clear(s, dbias, cols);
        return r;
    }
    if (!mat_ok(x) || !mat_ok(dy) || !mat_ok(dx) || !stats || (add && !mat_ok(add)) || x->dtype != dy->dtype || x->dtype != dx->dtype ||
        (add && add->dtype != x->dtype))
        return METIS_INVALID_ARG;
    if (rows < 1 || cols < 1 || !norm_mat(x, x) || !norm_mat(dy, x) || !norm_mat(dx, x) || (add && !norm_mat(add, x))) return METIS_BAD_SHAPE;
    const int st = norm_limits(rows, cols);
    if (st != METIS_OK) return st;
    const bool few = columns && norm_few(rows, cols, mat_size(x));
    if (columns && !few && (!workspace || workspace_bytes < metis_layernorm_grads_workspace_bytes(rows, cols))) return METIS_WORKSPACE_TOO_SMALL;
    if (columns && !few && (uintptr_t)workspace % 256) return METIS_INVALID_ARG;
    float* sums = columns && !few ? (float*)workspace : nullptr;
    auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        const T *pd = (const T*)dy->ptr, *px = (const T*)x->ptr, *pa = add ? (const T*)add->ptr : nullptr;
        const int64_t la = add ? add->ld : 0;
        if (!in_registers(cols)) {
            if (columns) {
                const int64_t chunk = column_chunk(rows, cols);
                hipLaunchKernelGGL(k_layernorm_columns<T>, dim3((unsigned)ceil_div64(cols, 512), (unsigned)ceil_div64(rows, chunk)), dim3(256), 0, s,
                                   pd, dy->ld, px, x->ld, (const float2*)stats, rows, cols, chunk, sums);
                if (hipGetLastError() != hipSuccess) return METIS_HIP_ERROR;
            }
            hipLaunchKernelGGL(k_layernorm_grads_long<T>, dim3((unsigned)(rows < 512 ? rows : 512)), dim3(1024), 0, s, pd, dy->ld, px, x->ld,
                               (const float2*)stats, weight, pa, la, (T*)dx->ptr, dx->ld, rows, cols);
        } else {
            by_length(cols, [&](auto rt, auto u) {
                constexpr int RT = decltype(rt)::value;
                constexpr int U = decltype(u)::value;
                if (few) {
                    const unsigned strips = (unsigned)ceil_div64(cols, RowGroup<RT>::THREADS / 16), groups = (unsigned)ceil_div64(rows, RowGroup<RT>::ROWS);
                    const bool over = dx->ptr == x->ptr || dx->ptr == dy->ptr;
                    auto kern = add ? k_layernorm_grads_few<T, RT, U, true> : k_layernorm_grads_few<T, RT, U, false>;
                    hipLaunchKernelGGL(kern, dim3(over ? strips : strips + groups), dim3(RowGroup<RT>::THREADS), 0, s, pd, dy->ld, px, x->ld,
                                       (const float2*)stats, weight, pa, la, (T*)dx->ptr, dx->ld, rows, cols, dweight, dbias, strips);
                    if (!over) return;
                }
                auto kern = add ? k_layernorm_grads<T, RT, U, true> : k_layernorm_grads<T, RT, U, false>;
                hipLaunchKernelGGL(kern, dim3((unsigned)norm_parts(rows, cols)), dim3(RowGroup<RT>::THREADS), 0, s, pd, dy->ld, px, x->ld,
                                   (const float2*)stats, weight, pa, la, (T*)dx->ptr, dx->ld, rows, cols, sums);
            });
        }
        return hipGetLastError() == hipSuccess ? METIS_OK : METIS_HIP_ERROR;
    };
    const int ls = x->dtype == METIS_BF16 ? launch(bf16_t()) : launch(float());
    if (ls != METIS_OK || !columns || few) return ls;
    return launch_join(s, sums, sum_rows(rows, cols), 2 * cols, dweight, cols, dbias);
}
