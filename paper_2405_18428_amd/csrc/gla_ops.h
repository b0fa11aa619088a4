// Layer norm and rotary positions (host + gfx950 device code): parameters and launchers.
#pragma once
#include "gla_common.h"

namespace gla {

constexpr int kNormMaxD = 8192;
constexpr int kRopeMaxD = 256, kRopeMaxAxes = 4;

// Rows of [B, H, T, D] or [B, T, H, D]; weight and bias [H, D]
struct NormParams {
    const void *x, *r_pre, *d_out;      // r_pre may be null: no gate
    const float *weight, *bias;         // null: ones, zeros
    void *out;                          // forward
    void *dx, *dr;                      // backward
    float *part;                        // [2, norm_partial_rows(), H, D]: sums for dweight and dbias, or null: not wanted
    float eps;
    int B, H, T, D, layout, out_dtype;
    int slots;                          // row groups that a head's rows are dealt to
};
// the backward pass's slots, and the partial sums of each head that these leave
int norm_slots(int B, int H, int T, int D, int layout);
int norm_partial_rows(int B, int H, int T, int D, int layout);
hipError_t launch_norm_fwd(const NormParams &p, int dtype, hipStream_t stream);
hipError_t launch_norm_bwd(const NormParams &p, int dtype, float *dweight, float *dbias, hipStream_t stream);

struct RopeParams {
    const void *x[2];                   // q, k (k may be null)
    void *y[2];
    const int *positions;               // [B, T, axes] or null: from the grid
    // of each pair, full turns a position: `turns` has 21 bits, so that its product with a position of 32 is exact, `rest` what is missing
    double turns[kRopeMaxD / 2], rest[kRopeMaxD / 2];
    int first[kRopeMaxAxes], pairs_end[kRopeMaxAxes], half[kRopeMaxAxes];   // of each section: first channel, pairs up to its end, its pairs
    int axes, pairs, adjacent, inverse;
    int B, H, T, d, grid_h, grid_w, layout;
    int heads_each;                     // heads a thread turns by one angle
};
// Checks and fills in what sections, base and grid say; a status of the C ABI
int rope_turns(RopeParams &p, const int *positions, const int *sections, int axes, float base, int T, int d, int grid_h, int grid_w);
hipError_t launch_rope(const RopeParams &p, int dtype, hipStream_t stream);

}  // namespace gla
