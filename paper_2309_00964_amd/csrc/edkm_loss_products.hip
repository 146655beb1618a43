// The cross entropy's two gradient products, for gfx950 (MI355X).

#include "edkm_loss.h"

namespace edkm {

template <int F>
static hipError_t sum_f(const LossArgs& a, int opa, const LossPlan& q, hipStream_t s) {
    return opa == OP_ROWS ? loss_tiled<F, OP_ROWS, OP_DEPTH, LossSum<F>>(a, q, s) : loss_tiled<F, OP_DEPTH, OP_DEPTH, LossSum<F>>(a, q, s);
}

hipError_t launch_loss_sum(const LossArgs& a, int fmt, int opa, const LossPlan& q, hipStream_t s) {
    return fmt == FMT_BF16 ? sum_f<FMT_BF16>(a, opa, q, s) : sum_f<FMT_FP16>(a, opa, q, s);
}

}  // namespace edkm
