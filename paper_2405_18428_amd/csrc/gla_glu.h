// Gated feed-forward product (host + gfx950 device code): parameters and launchers.
#pragma once
#include "gla_common.h"

namespace gla {

struct GluCall {
    const void *x, *w_gate, *w_up;      // [M, K], [F, K]: rows of ld_x, ld_w elements, beginning at 16 bytes
    const void *d_out;                  // [M, F], dense
    int M, K, F, ld_x, ld_w;
    int dtype, act;
    // backward
    void *dg[2], *du[2];                // [M, ld_f]: gradients of the two products, rows beginning at 16 bytes; bf16: what they are rounded to, and
                                        // what is left of them (null: not taken along)
    int ld_f;
    float *part;                        // glu_part_bytes()
    constexpr bool split() const { return dg[1] != nullptr; }
};
// y = act(x Wg^T) * (x Wu^T) -> out [M, F], and the two products to pre [2, M, F] if that is given
hipError_t launch_glu_fwd(const GluCall &c, void *out, int out_dtype, float *pre, hipStream_t stream);
// dg, du from the two products, which are formed again if pre is null
hipError_t launch_glu_slopes(const GluCall &c, const float *pre, hipStream_t stream);
hipError_t launch_glu_dx(const GluCall &c, void *dx, hipStream_t stream);
hipError_t launch_glu_dw(const GluCall &c, void *dw_gate, void *dw_up, hipStream_t stream);
// room for the parts that dx's and dW's sums are taken in, one after the other
size_t glu_part_bytes(int M, int K, int F, int dtype, bool split);
// x and the weights -> c.x, c.w_gate, c.w_up, whose rows have c.ld_x elements, zeros behind K
hipError_t launch_glu_pad(const GluCall &c, const void *x, const void *w_gate, const void *w_up, hipStream_t stream);

}  // namespace gla
