// What the files of the linear layer with an epilogue share.
#pragma once
#include "epilogue.h"

namespace {

inline bool near_rows(const metis_mat* m) { return !m || m->ld <= (1 << 24); }          // 16 of them, and their columns, within 2^31 bytes
inline bool whole_lines(const metis_mat* m) { return !m || ((uintptr_t)m->ptr % 128 == 0 && m->ld * mat_size(m) % 128 == 0); }
template <typename T, int ACT = ACT_ANY>
MxFinish<T, ACT> finish_of(const metis_epilogue* e, const metis_mat* Y) {
    return {(T*)Y->ptr,
            Y->ld,
            e ? e->bias : nullptr,
            e && e->pre ? (T*)e->pre->ptr : nullptr,
            e && e->pre ? e->pre->ld : 0,
            e && e->residual ? (const T*)e->residual->ptr : nullptr,
            e && e->residual ? e->residual->ld : 0,
            mask_key(e ? e->mask : nullptr),
            e ? e->act : METIS_ACT_NONE,
            near_rows(Y) && near_rows(e ? e->pre : nullptr) && near_rows(e ? e->residual : nullptr),
            whole_lines(Y) && whole_lines(e ? e->pre : nullptr)};
}

}  // namespace

// The streaming kernel (mx_stream.h) with the epilogue's activation built in: csrc/linear_stream.hip.  Arguments are checked already.
int linear_stream(hipStream_t s, const metis_mxfp4* X, const metis_mxfp4* W, const metis_epilogue* e, const metis_mat* Y);
