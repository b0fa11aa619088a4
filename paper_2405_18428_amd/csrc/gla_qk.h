// Norm and rotation of queries and keys (host + gfx950 device code): parameters and launchers.
#pragma once
#include "gla_ops.h"

namespace gla {

// One of the two tensors.  Rows are `d` channels in a row, those of a batch, a head and a token `stride` elements apart
struct QkSide {
    const void *x;                      // null: no such tensor
    long long sb, sh, st;
    const float *weight;                // [d] or null: ones
    int heads;
    void *out;                          // forward: y, backward: dx; dense in `layout`
    const void *d_out;                  // backward: dense in `layout`
    float *part;                        // backward: [slots, d] sums for the weight's gradient, or null: not wanted
    float *dweight;
};
struct QkParams {
    QkSide side[2];                     // queries, keys
    RopeParams rope;                    // positions, frequencies, sections, B, T, d, grid, layout; rope.pairs 0: no rotation
    float eps;
    int out_dtype;
    int slots;                          // work-groups of the backward pass
};
// work-groups of the backward pass, and so partial sums a tensor
int qk_slots(int B, int T);
hipError_t launch_qk_fwd(const QkParams &p, int dtype, hipStream_t stream);
hipError_t launch_qk_bwd(const QkParams &p, int dtype, hipStream_t stream);

}  // namespace gla
