// Gated recurrence of channels, h_t = a_t h_{t-1} + u_t (host + gfx950 device code): parameters and launchers.
#pragma once
#include "gla_common.h"
#include "gla_recur_plan.h"

namespace gla {

// Steps of a work-group's round: 8 waves of 8 steps; units of the backward pass are rounds, those of the forward pass two
constexpr int kRecurSteps = 8, kRecurWaves = 8, kRecurRound = kRecurSteps * kRecurWaves, kRecurChain = 2 * kRecurRound, kRecurChainWaves = 8;
constexpr int kRecurBlock = 16;         // units that look back over each other

struct RecurCall {
    const void *x, *gate;               // [B, T, D]
    const int *seq_lens;                // [B] or null: all T
    int B, T, D, grid_h, grid_w, scan_dir;
    long long step, wrap;               // elements from one scan step's row to the next, and at the end of a column
    int dtype, kind, rest;              // element type of x (and of pre-activations), a gla_gate_kind, u = (1 - a) x
    float inv_tau;
    int unit, nunits;                   // steps of a unit, and how many there are
};
// Forward: words that units and blocks of units publish (see the kernel), recur_chain_columns() of each, the second array right behind the first
struct RecurChain {
    unsigned long long *local;          // [nunits, columns]
    uint32_t *after, *ticket;           // [blocks, columns]
    int looks;                          // of a wait, or kRecurNoEnd
};
long long recur_chain_columns(const RecurCall &c);
// work-groups that a launch has for each unit of steps
long long recur_groups(const RecurCall &c);
// of 4 bytes, a column
inline long long recur_chain_words(const RecurCall &c) { return 2LL * c.nunits + (c.nunits + kRecurBlock - 1) / kRecurBlock; }
// Backward, per unit and channel, [B, nunits, D]: log2 of its decay, its state from zero and its adjoint from zero at its first step, the gate
// included; the latter two replaced by what enters the unit (from behind, for the adjoint)
struct RecurUnits {
    float *decay, *state, *adjoint;
};
hipError_t launch_recur_units(const RecurCall &c, const void *d_out, const RecurUnits &u, hipStream_t stream);
// Chains the units: `first` [B, D] enters the first (null: zero), `last` the last one from behind; the adjoint that leaves the first unit goes to
// d_first if that is given
hipError_t launch_recur_carry(const RecurCall &c, const RecurUnits &u, const float *first, const float *last, float *d_first, hipStream_t stream);
// Outputs, a work-group for the whole sequence, or in units
hipError_t launch_recur_walk(const RecurCall &c, const float *first, void *out, int out_dtype, float *final_state, hipStream_t stream);
hipError_t launch_recur_chain(const RecurCall &c, const RecurChain &ch, const float *first, void *out, int out_dtype, float *final_state, hipStream_t stream);
// Gradients, unit = kRecurRound.  One unit: `first` and `last` enter it, d_first leaves it
hipError_t launch_recur_back(const RecurCall &c, const void *d_out, const RecurUnits &u, const float *first, const float *last, void *dx,
                             void *dgate, int grad_dtype, float *d_first, hipStream_t stream);
hipError_t launch_recur_step(const RecurCall &c, const float *state, float *state_out, void *out, int out_dtype, hipStream_t stream);

}  // namespace gla
