// A linear layer on MXFP4 operands whose epilogue adds a bias, applies an activation, drops elements and adds a residual; and the gradient of
// that epilogue.
#include "mx_gemm.h"
#include "column_sums.h"

namespace {

struct LinearPlace {
    size_t scales, bytes;                         // place of the rows' scales behind their codes, and the end
};
LinearPlace linear_place(int64_t rows, int64_t K) {
    const size_t scales = align_up((size_t)rows * (K / 2), 256);
    return {scales, scales + align_up((size_t)rows * (K / 32), 256)};
}

template <typename T>
int launch_linear(hipStream_t s, const MxOperand& x, const MxOperand& w, int64_t K, const metis_epilogue* e, const metis_mat* Y) {
    const MxFinish<T> f = {(T*)Y->ptr,
                           Y->ld,
                           e ? e->bias : nullptr,
                           e && e->pre ? (T*)e->pre->ptr : nullptr,
                           e && e->pre ? e->pre->ld : 0,
                           e && e->residual ? (const T*)e->residual->ptr : nullptr,
                           e && e->residual ? e->residual->ld : 0,
                           mask_key(e ? e->mask : nullptr),
                           e ? e->act : METIS_ACT_NONE};
    return launch_mx_gemm<T>(s, x, w, K, f.y, f.ldy, f);
}

// ---- gradient of the epilogue ----
// dz = act'(pre) m dy, and the sum of its columns.  A workgroup has 512 columns, a lane eight of them, and its four waves take every fourth of
// its rows: the columns' sums stay in registers.
template <typename T>
__global__ void __launch_bounds__(256)
k_linear_grads(const T* dy, int64_t ldd, const T* pre, int64_t ldp, T* dz, int64_t ldz, int act, MaskKey mask, int64_t rows, int64_t cols,
               int64_t chunk, float* __restrict__ sums) {
    __shared__ float s_sum[3 * 8 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t c = 512 * (int64_t)blockIdx.x + 8 * lane, n = cols - c;
    const int64_t first = chunk * blockIdx.y, end = first + chunk < rows ? first + chunk : rows;
    const uint32_t step = mask_step(mask);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    if (n > 0) {
#pragma unroll 2
        for (int64_t r = first + wave; r < end; r += 4) {
            float v[8], z[8];
            load_part<T, true>(dy + r * ldd + c, n, v);
            if (pre) load_part<T, true>(pre + r * ldp + c, n, z);
            if (mask.dropped) mask_apply(mask, step, (uint32_t)(c >> 3), (uint32_t)r, v);
            if (pre) {
                auto all = [&](int a) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= act_slope<sizeof(T) == 2>(a, z[i]);
                };
                switch (act) {
                    case METIS_ACT_RELU: all(METIS_ACT_RELU); break;
                    case METIS_ACT_GELU: all(METIS_ACT_GELU); break;
                    case METIS_ACT_GELU_TANH: all(METIS_ACT_GELU_TANH); break;
                    case METIS_ACT_SILU: all(METIS_ACT_SILU); break;
                    default: break;
                }
            }
            if (dz) store_part<T, true>(dz + r * ldz + c, n, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
    }
    if (!sums) return;
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_sum[((wave - 1) * 8 + i) * 64 + lane] = sum[i];
    }
    __syncthreads();
    if (wave > 0 || n <= 0) return;
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += s_sum[(p * 8 + i) * 64 + lane];
    store_part<float, true>(sums + blockIdx.y * cols + c, n, sum);
}

// Rows of a workgroup: some 2048 workgroups in all, 32 rows each at least, the same on any chip so that the sums have the same order.
int64_t grads_chunk(int64_t rows, int64_t cols) {
    const int64_t strips = ceil_div64(cols, 512), chunks = ceil_div64(2048, strips);
    const int64_t chunk = ceil_div64(rows, chunks);
    return chunk < 32 ? 32 : chunk;
}

bool same_layout(const metis_mat* a, const metis_mat* b) { return a->rows == b->rows && a->cols == b->cols && a->ld >= a->cols; }

}  // namespace

extern "C" size_t metis_mxfp4_linear_workspace_bytes(int64_t rows, int64_t N, int64_t K) {
    if (rows < 1 || N < 1 || K < 32 || K % 32 || rows > 0xFFFFFFFFll / (K / 2) || N > 0xFFFFFFFFll / (K / 2)) return 0;
    return linear_place(rows, K).bytes;
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
    const LinearPlace place = linear_place(rows, K);
    metis_mxfp4 q = X ? metis_mxfp4{ws, ws + place.scales, rows, K} : *Xq;
    const int st = mx_operands_status(X ? W : &q, W);
    if (st != METIS_OK) return st;
    if (X) {
        if (rows * (K / 2) > 0xFFFFFFFFll) return METIS_UNSUPPORTED;
        if (!workspace || workspace_bytes < place.bytes) return METIS_WORKSPACE_TOO_SMALL;
        if ((uintptr_t)workspace % 256) return METIS_INVALID_ARG;
        const int qs = metis_quantize_mx(stream, X, &q);
        if (qs != METIS_OK) return qs;
    }
    const MxOperand x = {q.codes, q.scales, rows}, w = {W->codes, W->scales, N};
    hipStream_t s = (hipStream_t)stream;
    return Y->dtype == METIS_BF16 ? launch_linear<bf16_t>(s, x, w, K, e, Y) : launch_linear<float>(s, x, w, K, e, Y);
}

extern "C" size_t metis_linear_grads_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1 || cols > (1 << 28) || rows > 0xFFFFFFFFll) return 0;
    const int64_t chunks = ceil_div64(rows, grads_chunk(rows, cols));
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
    const int64_t chunk = grads_chunk(rows, cols), chunks = ceil_div64(rows, chunk), strips = ceil_div64(cols, 512);
    if (!grid_fits(strips, 256) || chunks > 65535) return METIS_UNSUPPORTED;
    const bool parts = dbias && chunks > 1;
    if (parts && (!workspace || workspace_bytes < metis_linear_grads_workspace_bytes(rows, cols))) return METIS_WORKSPACE_TOO_SMALL;
    if (parts && (uintptr_t)workspace % 256) return METIS_INVALID_ARG;
    float* sums = parts ? (float*)workspace : dbias;
    auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(k_linear_grads<T>, dim3((unsigned)strips, (unsigned)chunks), dim3(256), 0, s, (const T*)dY->ptr, dY->ld,
                           pre ? (const T*)pre->ptr : nullptr, pre ? pre->ld : 0, dZ ? (T*)dZ->ptr : nullptr, dZ ? dZ->ld : 0, act,
                           mask_key(mask), rows, cols, chunk, sums);
    };
    if (dY->dtype == METIS_BF16) launch(bf16_t());
    else launch(float());
    METIS_LAUNCH_CHECK();
    return parts ? launch_join(s, sums, chunks, cols, dbias, cols, nullptr) : METIS_OK;
}
