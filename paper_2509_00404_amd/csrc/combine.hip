// The experts' rows back to their tokens, and the gradients of that.
#include <type_traits>
#include "elementwise.h"

#define COMBINE_MAX_K 16

namespace {

// A lane per eight columns of a token, its choices' rows in flight together.  ANY: rows of any length and alignment.  Memory: 16384 tokens' four
// rows of 4096 bf16 (672 MB) 126 us, 5.3 TB/s; 3668 tokens' seven rows of 1388 22 us (82 MB; a column a lane 49).
template <typename T, typename O, bool ANY>
__global__ void __launch_bounds__(256)
k_combine(const T* __restrict__ rows, int64_t ldr, int64_t S, int64_t cols, const int32_t* __restrict__ slot, const float* __restrict__ weights,
          int k, O* __restrict__ y, int64_t ldy, uint64_t total, FastDiv units) {
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const uint64_t t = div_by(units, n), c = 8 * (n - t * units.d);
    const int64_t left = cols - (int64_t)c;
    float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int j = 0; j < k; ++j) {
        const int32_t s = slot[t * k + j];
        if ((uint32_t)s >= (uint64_t)S) continue;
        const float w = weights ? weights[t * k + j] : 1.0f;
        float v[8];
        load_part<T, ANY>(rows + s * ldr + c, left, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = fmaf(w, v[i], acc[i]);
    }
    store_part<O, ANY>(y + t * ldy + c, left, acc);
}

// A workgroup per token: its gradient row is read once for all its choices.  The products with the rows are added up per lane, then over
// the wave, then over the waves, always in the same order.  Memory: 8192 tokens' four rows of 4096 bf16 (604 MB) 126 us, 4.8 TB/s.
template <typename T, typename D, bool ANY, int K>
__global__ void __launch_bounds__(256)
k_combine_grads(const D* __restrict__ dy, int64_t ldy, const T* __restrict__ rows, int64_t ldr, int64_t S, int64_t cols,
                const int32_t* __restrict__ offsets, int E, const int32_t* __restrict__ slot, const float* __restrict__ weights, int k,
                T* __restrict__ drows, int64_t ldd, float* __restrict__ dweights) {
    __shared__ float s_part[4][K];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t s[K];
    float w[K], dot[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        s[j] = j < k ? slot[t * k + j] : -1;
        if ((uint32_t)s[j] >= (uint64_t)S) s[j] = -1;
        w[j] = s[j] >= 0 ? weights[t * k + j] : 0.0f;
        dot[j] = 0.0f;
    }
    for (int64_t c = (int64_t)threadIdx.x * 8; c < cols; c += (int64_t)blockDim.x * 8) {
        const int64_t left = cols - c;
        float d[8];
        load_part<D, ANY>(dy + t * ldy + c, left, d);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (s[j] < 0) continue;
            float v[8];
            load_part<T, ANY>(rows + s[j] * ldr + c, left, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dot[j] = fmaf(d[i], v[i], dot[j]);
                v[i] = w[j] * d[i];
            }
            store_part<T, ANY>(drows + s[j] * ldd + c, left, v);
        }
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) dot[j] += __shfl_xor(dot[j], m);
        if (lane == 0) s_part[wave][j] = dot[j];
    }
    __syncthreads();
    if ((int)threadIdx.x < k) {
        float sum = 0.0f;
        for (int v = 0; v < (int)blockDim.x / 64; ++v) sum += s_part[v][threadIdx.x];
        dweights[t * k + threadIdx.x] = sum;
    }
    // the slots that serve no choice
    const float zero[8] = {};
    const int64_t used = offsets[E] > 0 ? offsets[E] : 0;
    for (int64_t r = used + t; r < S; r += gridDim.x)
        for (int64_t c = (int64_t)threadIdx.x * 8; c < cols; c += (int64_t)blockDim.x * 8) store_part<T, ANY>(drows + r * ldd + c, cols - c, zero);
}

int plan_rows_status(const metis_mat* rows, const metis_expert_plan* p) {
    if (!mat_ok(rows) || !p || !p->slot || p->tokens < 1 || p->k < 1 || p->experts < 1) return METIS_INVALID_ARG;
    if (p->k > COMBINE_MAX_K) return METIS_UNSUPPORTED;
    if (p->tokens > 0x7FFFFFFFll / p->k || rows->rows != p->tokens * p->k || rows->cols < 1 || rows->cols > 0x7FFFFFFF || rows->ld < rows->cols)
        return METIS_BAD_SHAPE;
    return METIS_OK;
}

template <typename T, typename O>
int launch_combine(hipStream_t s, const metis_mat* rows, const metis_expert_plan* p, const float* weights, metis_mat* y) {
    const bool whole = rows->cols % 8 == 0 && mat_aligned16(rows) && mat_aligned16(y);
    const int64_t units = ceil_div64(rows->cols, 8), total = p->tokens * units;
    const int st = units_status(p->tokens, units);
    if (st != METIS_OK) return st;
    auto kern = whole ? k_combine<T, O, false> : k_combine<T, O, true>;
    hipLaunchKernelGGL(kern, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s, (const T*)rows->ptr, rows->ld, rows->rows, rows->cols,
                       p->slot, weights, p->k, (O*)y->ptr, y->ld, (uint64_t)total, fast_div((uint32_t)units));
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

template <typename T, typename D, int K>
int launch_combine_grads(hipStream_t s, const metis_mat* dy, const metis_mat* rows, const metis_expert_plan* p, const float* weights,
                         metis_mat* drows, float* dweights) {
    const bool whole = rows->cols % 8 == 0 && mat_aligned16(rows) && mat_aligned16(drows) && mat_aligned16(dy);
    const int64_t units = ceil_div64(rows->cols, 8);
    const int threads = units <= 64 ? 64 : units <= 128 ? 128 : 256;
    if (!grid_fits(p->tokens, threads)) return METIS_UNSUPPORTED;
    auto kern = whole ? k_combine_grads<T, D, false, K> : k_combine_grads<T, D, true, K>;
    hipLaunchKernelGGL(kern, dim3((unsigned)p->tokens), dim3(threads), 0, s, (const D*)dy->ptr, dy->ld,
                       (const T*)rows->ptr, rows->ld, rows->rows, rows->cols, p->offsets, p->experts, p->slot, weights, p->k, (T*)drows->ptr,
                       drows->ld, dweights);
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}

}  // namespace

extern "C" int metis_combine(void* stream, const metis_mat* rows, const metis_expert_plan* plan, const float* weights, metis_mat* y) {
    if (plan && plan->tokens == 0) return METIS_OK;
    const int st = plan_rows_status(rows, plan);
    if (st != METIS_OK) return st;
    if (!mat_ok(y)) return METIS_INVALID_ARG;
    if (y->rows != plan->tokens || y->cols != rows->cols || y->ld < y->cols) return METIS_BAD_SHAPE;
    hipStream_t s = (hipStream_t)stream;
    if (rows->dtype == METIS_BF16)
        return y->dtype == METIS_BF16 ? launch_combine<bf16_t, bf16_t>(s, rows, plan, weights, y) : launch_combine<bf16_t, float>(s, rows, plan, weights, y);
    return y->dtype == METIS_BF16 ? launch_combine<float, bf16_t>(s, rows, plan, weights, y) : launch_combine<float, float>(s, rows, plan, weights, y);
}

extern "C" int metis_combine_grads(void* stream, const metis_mat* dy, const metis_mat* rows, const metis_expert_plan* plan, const float* weights,
                                   metis_mat* drows, float* dweights) {
    if (plan && plan->tokens == 0) return METIS_OK;
    const int st = plan_rows_status(rows, plan);
    if (st != METIS_OK) return st;
    if (!plan->offsets || !mat_ok(dy) || !mat_ok(drows) || !weights || !dweights || drows->dtype != rows->dtype) return METIS_INVALID_ARG;
    if (dy->rows != plan->tokens || dy->cols != rows->cols || dy->ld < dy->cols) return METIS_BAD_SHAPE;
    if (drows->rows != rows->rows || drows->cols != rows->cols || drows->ld < drows->cols) return METIS_BAD_SHAPE;
    hipStream_t s = (hipStream_t)stream;
    auto by_k = [&](auto t, auto d) -> int {
        typedef decltype(t) T;
        typedef decltype(d) D;
        if (plan->k <= 4) return launch_combine_grads<T, D, 4>(s, dy, rows, plan, weights, drows, dweights);
        if (plan->k <= 8) return launch_combine_grads<T, D, 8>(s, dy, rows, plan, weights, drows, dweights);
        return launch_combine_grads<T, D, 16>(s, dy, rows, plan, weights, drows, dweights);
    };
    if (rows->dtype == METIS_BF16) return dy->dtype == METIS_BF16 ? by_k(bf16_t(), bf16_t()) : by_k(bf16_t(), float());
    return dy->dtype == METIS_BF16 ? by_k(float(), bf16_t()) : by_k(float(), float());
}
