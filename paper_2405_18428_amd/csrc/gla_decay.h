// Linear attention with one decay a head (host + gfx950 device code): parameters of its kernels and their launchers.
//
//   S_t = a_t S_{t-1} + k_t^T v_t ,   o_t = q_t S_t ,   a_t = exp(log_decay) one number for a (head) or a (batch, head, token)
//
// in chunks of C steps (Sec. 3.5 of the DiG paper with a scalar in place of the gate row).  With b_i the sum of the gates
// up to and with step i of a chunk that the state S enters:
//   o_i = exp(b_i) q_i S + sum over j <= i of exp(b_i - b_j) (q_i k_j) v_j ,
//   S'  = exp(b_last) S + sum over j of exp(b_last - b_j) k_j^T v_j .
// Only differences of b with a non-positive value are exponentiated, so any gates do, down to exp(log_decay) = 0.
//
// The backward pass is the same recurrence three times: with the adjoint state G_t = q_t^T dO_t + a_{t+1} G_{t+1},
//   dq_t = S_t dO_t^T  is the recurrence of (dO, v, k) from the transposed state, and read backwards, where step t meets the
//   gate of step t + 1,  dv_t = k_t G_t  that of (k, q, dO) and  dk_t = G_t v_t^T  that of (v, dO, q).
// What a log_decay changes is what flows from the state before step t into all that comes after,
//   dL/dlog a_t = <a_t S_{t-1}, G_t> = sum over s >= t of (q_s dq_s - k_s dk_s) + <S_T, dS_T> .
// Both dot products hold the step's own (q_s k_s)(v_s dO_s), which no gate scales: it is left out of both (dq_s - (v_s dO_s) k_s in place of
// dq_s, dk_s - (v_s dO_s) q_s in place of dk_s), as what its rounding left would bury the gradients of strong gates, which vanish
// with a_t.  The sum's terms cancel to a small rest when it runs far, so it runs to the end of a block of kFlowBlock steps only, and
// what flows across the block's end is the product of the state and the adjoint state there.
#pragma once
#include "gla_common.h"

namespace gla {

constexpr int kDecayMaxD = 128;
constexpr int kFlowBlock = 256;      // steps between two states that the backward pass keeps for the gates' gradient

enum DecayKind : int { kDecayHead = 0, kDecayToken = 1 };   // log_decay [H], or one for each token

// What calls on bf16 rows carry in three bf16 numbers instead of two (gla_decay_util.h)
enum DecayDigits : int {
    kDigitsRows = 0,                    // nothing: rows come out, or the gradients of tokens' gates
    kDigitsStates = 1,                  // what states take up: a state comes out
    kDigitsAll = 2                      // everything: the gradient of heads' gates comes out
};

// What all walks of one call share.
struct DecayCall {
    const float *log_decay;
    const int *seq_lens;                // [B] or null: all T steps
    int kind;                           // DecayKind
    int B, H, T, dk, dv, grid_h, grid_w, scan_dir;
    int layout;                         // gla_layout
    int digits;                         // bf16 calls: DecayDigits
    int fast;                           // rows through 32-bit views (gla_decay_util.h)
    int nspans, span_len;               // spans a sequence is walked in, steps in each (a multiple of 64)
};

// The states that enter the spans: `first` [B*H, dk, dv] (or null: zero) the first span walked; behind it, with `local` [B*H, nspans, dk, dv] and
// the base-2 logs of the spans' decays, what the walk chains for itself from the local states of the spans before its own, or
// with `chained` entry sp of `local` as it is.
struct DecayEntry {
    const float *first, *local, *decay;
    int chained;
};

// One walk: the recurrence of (x, y, z) in place of (q, k, v).  x and y are dk or dv wide (m), z is the other or the same (n);
// the state is [m, n].
struct DecayRole {
    const void *x, *y, *z;
    void *out;                          // n wide
    const void *dot;                    // rows of width n, or null: flow[row] = out row . dot row (in 32 bits, unrounded)
    float *flow;                        // [B*H, T] in scan steps
    int m, n;
};

struct DecayWalk {
    DecayCall c;
    DecayRole r;
    // states lie as [.., dk, dv]; with state_t a walk whose m is dv reads and writes them transposed
    DecayEntry in;
    float *state_out;                   // [B*H, dk, dv] after the last step, or null
    float *anchors;                     // [B*H, blocks, dk, dv] or null: the state at the end of each block of kFlowBlock steps
    int anchor_last;                    // the last block's too
    float *local, *decay;               // state walks: [B*H, nspans, dk, dv] state of a span from zero, [B*H, nspans] log2 of its decay
    int state_t;
    int out_dtype;
    int grad;                           // 1: a walk of the backward pass, with dots and anchors, which clears the rows behind a sequence's
                                        // end; 0: these rows stay as they are
};

// The reversed walk: dv (role a) and dk (role b) from one reading of q, k, v, dO.
struct DecayBack {
    DecayCall c;
    const void *q, *k, *v, *d_out;
    void *dk_grad, *dv_grad;
    DecayEntry in;                      // adjoint states, from behind
    float *d_initial;                   // [B*H, dk, dv] or null
    const float *anchors;               // what the walk for dq left, or null: no gate gradient
    int anchor_last;
    float *meet;                        // [B*H, blocks]: <S, G> at the end of each block, G before it decays past it
    float *flow_k;                      // [B*H, T]: k_s dk_s
    int grad_dtype;
};

struct DecayGate {
    DecayCall c;
    const float *flow_q, *flow_k, *meet;
    int anchor_last;
    float *dlog;                        // [H] or a token
    double *part;                       // [B*H, blocks] (heads)
};

__host__ __device__ inline int decay_blocks(int T) { return (T + kFlowBlock - 1) / kFlowBlock; }

hipError_t launch_decay_walk(const DecayWalk &w, int dtype, hipStream_t stream);
// local states of every span but the last one walked: of (k, v) to w.local and, with `back`, of the reversed (q, dO) to back->local
hipError_t launch_decay_states(const DecayWalk &w, const DecayWalk *back, int dtype, hipStream_t stream);
// chains local states in place: entry sp of `local` becomes the state that enters span sp, from `first` [B*H, dk, dv] or zero; `reversed`: the
// last span comes first
struct DecayChain {
    const float *first;
    float *local;
    const float *decay;
    int nspans, reversed;
};
hipError_t launch_decay_carry(const DecayCall &c, const DecayChain &chain, const DecayChain *other, hipStream_t stream);
hipError_t launch_decay_back(const DecayBack &w, int dtype, hipStream_t stream);
hipError_t launch_decay_gate(const DecayGate &w, hipStream_t stream);
hipError_t launch_decay_step(const void *q, const void *k, const void *v, const float *log_decay, int kind, int B, int H, int dk, int dv,
                             int dtype, int out_dtype, const float *state, float *state_out, void *out, hipStream_t stream);

}  // namespace gla
