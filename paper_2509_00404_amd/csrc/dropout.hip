// Dropout whose mask is computed wherever it is needed and never stored.
#include "epilogue.h"

namespace {

// A lane per eight elements of a row: one block of the generator, 16 bytes of a bf16 operand.  Memory bounds it: 16384 x 4096 bf16 39.7 us (268 MB), with
// a residual 71.2 (403 MB, 5.7 TB/s); the generator's 20 multiplications take half of the clocks beside it.
template <typename T>
__global__ void __launch_bounds__(256)
k_dropout(const T* x, int64_t ldx, const T* residual, int64_t ldr, T* y, int64_t ldy, MaskKey mask, uint64_t total, FastDiv units, int64_t cols) {
    const uint64_t u = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= total) return;
    const uint64_t r = div_by(units, u), unit = u - r * units.d;
    const int64_t c = 8 * (int64_t)unit, n = cols - c;
    float v[8], res[8];
    load_part<T, true>(x + r * ldx + c, n, v);
    if (residual) load_part<T, true>(residual + r * ldr + c, n, res);
    if (mask.dropped) mask_apply(mask, mask_step(mask), (uint32_t)unit, (uint32_t)r, v);
    if (residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += res[i];
    }
    store_part<T, true>(y + r * ldy + c, n, v);
}

}  // namespace

extern "C" int metis_dropout(void* stream, const metis_mat* x, const metis_dropout_mask* mask, const metis_mat* residual, metis_mat* y) {
    if (!x || !y || !mask || mask_status(mask) != METIS_OK) return METIS_INVALID_ARG;
    if (x->rows == 0 && y->rows == 0) return METIS_OK;
    if (!mat_ok(x) || !mat_ok(y) || (residual && !mat_ok(residual)) || x->dtype != y->dtype || (residual && residual->dtype != y->dtype))
        return METIS_INVALID_ARG;
    auto fits = [&](const metis_mat* m) { return m->rows == y->rows && m->cols == y->cols && m->ld >= m->cols; };
    if (y->rows < 1 || y->cols < 1 || !fits(x) || !fits(y) || (residual && !fits(residual))) return METIS_BAD_SHAPE;
    const int64_t units = ceil_div64(y->cols, 8);
    const int st = units_status(y->rows, units);
    if (st != METIS_OK) return st;
    const int64_t total = y->rows * units;
    hipStream_t s = (hipStream_t)stream;
    auto launch = [&](auto zero) {
        typedef decltype(zero) T;
        hipLaunchKernelGGL(k_dropout<T>, dim3((unsigned)ceil_div64(total, 256)), dim3(256), 0, s, (const T*)x->ptr, x->ld,
                           residual ? (const T*)residual->ptr : nullptr, residual ? residual->ld : 0, (T*)y->ptr, y->ld, mask_key(mask),
                           (uint64_t)total, fast_div((uint32_t)units), y->cols);
    };
    if (y->dtype == METIS_BF16) launch(bf16_t());
    else launch(float());
    METIS_LAUNCH_CHECK();
    return METIS_OK;
}
