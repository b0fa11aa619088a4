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
    void *dg, *du;                      // [M, ld_f]: gradients of the two products, rows beginning at 16 bytes
    int ld_f;
    float *part;                        // [splits, M, K]
    int splits;
};
// y = act(x Wg^T) * (x Wu^T) -> out [M, F], and the two products to pre [2, M, F] if that is given
hipError_t launch_glu_fwd(const GluCall &c, void *out, int out_dtype, float *pre, hipStream_t stream);
// dg, du from the two products, which are formed again if pre is null
hipError_t launch_glu_slopes(const GluCall &c, const float *pre, hipStream_t stream);
hipError_t launch_glu_dx(const GluCall &c, void *dx, hipStream_t stream);
hipError_t launch_glu_dw(const GluCall &c, void *dw_gate, void *dw_up, hipStream_t stream);
// parts that dx's sum over 2 F products is taken in
int glu_splits(int M, int K, int F, int dtype);
// [rows, cols] -> rows of `ld` elements, zeros behind
hipError_t launch_glu_pad(const void *from, void *to, int rows, int cols, int ld, int dtype, hipStream_t stream);

}  // namespace gla
