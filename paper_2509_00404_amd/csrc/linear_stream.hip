// Large products with an epilogue, on the streaming kernel.  An instance for every activation: with all of them in one, a step of the epilogue waits
// for its instructions (16384 x 14336 x 4096 without an activation 551 us, so 523; the product alone takes 498).  With the epilogue a wave's rows pass
// through LDS as fp32, all waves at once and with the matrix pipe idle; an activation adds its vector instructions (gelu 7 us a round of tiles), `pre`
// and the residual their memory time (16384 x 14336: 32 and 60 us; the residual's rows fetched where they are used, 137).
#include "mx_gemm.h"
#include "linear.h"

namespace {

template <typename T, int ACT>
int stream_act(hipStream_t s, const metis_mxfp4* X, const metis_mxfp4* W, const metis_epilogue* e, const metis_mat* Y) {
    const MxFinish<T, ACT> f = finish_of<T, ACT>(e, Y);
    return launch_mx_stream<T>(s, MxOperand{X->codes, X->scales, X->rows}, MxOperand{W->codes, W->scales, W->rows}, W->cols, f.y, f.ldy, f);
}
template <typename T>
int stream_type(hipStream_t s, const metis_mxfp4* X, const metis_mxfp4* W, const metis_epilogue* e, const metis_mat* Y) {
    switch (e ? e->act : METIS_ACT_NONE) {
        case METIS_ACT_RELU: return stream_act<T, METIS_ACT_RELU>(s, X, W, e, Y);
        case METIS_ACT_GELU: return stream_act<T, METIS_ACT_GELU>(s, X, W, e, Y);
        case METIS_ACT_GELU_TANH: return stream_act<T, METIS_ACT_GELU_TANH>(s, X, W, e, Y);
        case METIS_ACT_SILU: return stream_act<T, METIS_ACT_SILU>(s, X, W, e, Y);
        default: return stream_act<T, METIS_ACT_NONE>(s, X, W, e, Y);
    }
}

}  // namespace

int linear_stream(hipStream_t s, const metis_mxfp4* X, const metis_mxfp4* W, const metis_epilogue* e, const metis_mat* Y) {
    return Y->dtype == METIS_BF16 ? stream_type<bf16_t>(s, X, W, e, Y) : stream_type<float>(s, X, W, e, Y);
}
