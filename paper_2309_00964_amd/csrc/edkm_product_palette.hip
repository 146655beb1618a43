// Products of some hundred tokens with palettized weights, for gfx950 (MI355X): the tiled
// product with a palette in the weights' place, decoded on the way into LDS.

#include "edkm_tiled.h"

namespace edkm {

template <int F>
static hipError_t palette_f(const ProductArgs& p, const ProductPlan& q, hipStream_t s) {
    switch (p.bits) {
    case 1: return tiled<F, OP_ROWS, OP_ROWS, 128, 2, 2, true, 1>(p, q, s);
    case 2: return tiled<F, OP_ROWS, OP_ROWS, 128, 2, 2, true, 2>(p, q, s);
    case 3: return tiled<F, OP_ROWS, OP_ROWS, 128, 2, 2, true, 3>(p, q, s);
    default: return tiled<F, OP_ROWS, OP_ROWS, 128, 2, 2, true, 4>(p, q, s);
    }
}

hipError_t launch_tiled_palette(ProductArgs p, int fmt, float* part, hipStream_t s) {
    const ProductPlan q = product_plan(p, OP_ROWS, OP_PALETTE);
    p.split_steps = q.split_steps;
    p.part = q.splits > 1 ? part : nullptr;
    return fmt == FMT_BF16 ? palette_f<FMT_BF16>(p, q, s) : palette_f<FMT_FP16>(p, q, s);
}

}  // namespace edkm
