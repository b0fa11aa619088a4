// Host side of the C ABI for what stands around the mixer in a block: the gated recurrence of channels, the norm and rotation of queries and
// keys, the gated feed-forward product.  Argument checks, plans, workspaces.
#include <math.h>

#include "gla_glu.h"
#include "gla_qk.h"
#include "gla_recur.h"

namespace gla {
namespace {

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
template <typename... P>
bool any_misaligned(P... p) { return (misaligned(p) || ...); }
bool off_element(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == GLA_DT_BF16 ? 1u : 3u)) != 0; }
bool bad_dtype(int d) { return d != GLA_DT_F32 && d != GLA_DT_BF16; }
size_t size_of(int dtype) { return dtype == GLA_DT_BF16 ? 2 : 4; }
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// A tensor's place in memory (null: none)
struct Span {
    const void *p;
    size_t bytes;
};
bool touch(Span a, Span b) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
    return p != 0 && q != 0 && p < q + b.bytes && q < p + a.bytes;
}
// whether one of some tensors shares memory with another one of them or with one of `others`
template <size_t N, size_t M>
bool any_touch(const Span (&mine)[N], const Span (&others)[M]) {
    for (size_t i = 0; i < N; ++i) {
        for (size_t j = 0; j < i; ++j)
            if (touch(mine[i], mine[j])) return true;
        for (size_t j = 0; j < M; ++j)
            if (touch(mine[i], others[j])) return true;
    }
    return false;
}

// --- gated recurrence of channels ---

// (e^-z is lost below 2^-126, which is 2^-62 of a gate's logarithm from 1 / tau = 2^64 on; an infinite reciprocal would make NaN of a gate of one)
bool bad_tau(float tau) { return !(tau >= 0x1p-64f) || isinf(tau); }

// Forward: the sequence in units, or walked by one work-group, where there are many of those or few units.  bf16, 2048 channels, walked and in
// units: 4096 steps of 64 groups of 128 channels 151 us and 49, of 128 groups 154 and 106, of 192 groups 154 and 136, of 256 groups 160 and 193 (1024 steps 43 and
// 46, 512 steps 24 and 29); 512 steps of 128 groups 22.6 and 20.4, 256 steps 12.3 and 12.9, of 64 groups 11.7 and 10.6, 160 steps 9.3 and 10.9.
// Odd D, whose groups have 64 channels and loads half as wide: 256 groups of 2047 channels, 300 steps 14 us and 23, 768 29 and 38, 1024 38 and 45, 1500 55 and
// 59, 2048 73 and 73, 4096 146 and 148; 512 groups 21 and 36, 50 and 58, 67 and 72, 95 and 98, 153 and 153, 302 and 271; 320 groups, the least fit for a walk,
// 20 and 27, 43 and 42, 56 and 52, 83 and 69, 110 and 86, 239 and 167.
constexpr int kWalkGroups = 256, kWalkUnits = 2, kWalkOddSteps = 1024;
constexpr long long kMostGroups = 1LL << 23;         // work-groups of 512 threads: fewer than 2^32 threads in a launch
void plan_forward(RecurCall &c) {
    const bool odd = c.D % 2 != 0;
    const long long units = (c.T + kRecurChain - 1) / kRecurChain, groups = ((long long)c.B * c.D + (odd ? 63 : 127)) / (odd ? 64 : 128);
    const bool walks = c.T <= kWalkUnits * kRecurChain || (groups >= kWalkGroups && (!odd || c.T <= kWalkOddSteps || recur_groups(c) >= kMostGroups / units));
    c.unit = walks ? c.T : kRecurChain;
    c.nunits = walks ? 1 : (int)units;
}
void plan_backward(RecurCall &c) {
    c.unit = kRecurRound;
    c.nunits = (c.T + kRecurRound - 1) / kRecurRound;
}
// The words that units publish, and the ticket
size_t chain_bytes(const RecurCall &c) { return c.nunits > 1 ? align_up((size_t)(recur_chain_columns(c) * recur_chain_words(c)) * 4) + 256 : 0; }
RecurChain chain_in(const RecurCall &c, void *workspace, bool in_place) {
    char *p = static_cast<char *>(workspace);
    RecurChain r;
    r.local = reinterpret_cast<unsigned long long *>(p);
    r.after = reinterpret_cast<uint32_t *>(p + (size_t)recur_chain_columns(c) * c.nunits * 8);
    r.ticket = reinterpret_cast<uint32_t *>(p + chain_bytes(c) - 256);
    r.looks = in_place ? kRecurNoEnd : gla_get_option(GLA_OPT_LOOK_BACK_POLLS);
    return r;
}
size_t units_bytes(const RecurCall &c) { return c.nunits > 1 ? 3 * align_up((size_t)c.B * c.nunits * c.D * sizeof(float)) : 0; }
RecurUnits units_in(const RecurCall &c, void *workspace) {
    const size_t each = align_up((size_t)c.B * c.nunits * c.D * sizeof(float));
    char *p = static_cast<char *>(workspace);
    return {reinterpret_cast<float *>(p), reinterpret_cast<float *>(p + each), reinterpret_cast<float *>(p + 2 * each)};
}

// (backward also the chain's work-groups, of 1024 threads for each 64 channels of a sequence)
bool fits(const RecurCall &c, bool back) {
    const long long groups = recur_groups(c);
    return groups < kMostGroups && groups * c.nunits < kMostGroups && (!back || c.nunits == 1 || (long long)c.B * ((c.D + 63) / 64) < (1LL << 22));
}

int check_recur(RecurCall &c, bool back, const void *x, const void *gate, int kind, float tau, int complement, const int *seq_lens, int B, int T, int D,
                int grid_h, int grid_w, int scan_dir, int dtype, int other_dtype) {
    if (B <= 0 || T <= 0 || D <= 0 || grid_h <= 0 || grid_w <= 0) return GLA_ERR_SHAPE;
    if ((long long)grid_h * grid_w != T || scan_dir < 0 || scan_dir > 3) return GLA_ERR_SHAPE;
    if (bad_dtype(dtype) || bad_dtype(other_dtype) || (kind != GLA_GATE_LOG && kind != GLA_GATE_PRE)) return GLA_ERR_SHAPE;
    if (kind == GLA_GATE_PRE && bad_tau(tau)) return GLA_ERR_SHAPE;
    if (seq_lens != nullptr && scan_dir > GLA_SCAN_ROW_REV) return GLA_ERR_UNSUPPORTED;
    // (steps and what lies behind the last unit as int; a row's channels as 32-bit byte offsets)
    if (T > (1 << 30) || D > (1 << 26)) return GLA_ERR_UNSUPPORTED;
    c = {};
    c.B = B;
    c.T = T;
    c.D = D;
    back ? plan_backward(c) : plan_forward(c);
    if (!fits(c, back)) return GLA_ERR_UNSUPPORTED;
    if (any_misaligned(x, gate) || (reinterpret_cast<uintptr_t>(seq_lens) & 3u) != 0) return GLA_ERR_ALIGN;
    c.x = x;
    c.gate = gate;
    c.seq_lens = seq_lens;
    c.grid_h = grid_h;
    c.grid_w = grid_w;
    c.scan_dir = scan_dir;
    const long long onward = scan_dir & 1 ? -D : D;
    c.step = (scan_dir >= GLA_SCAN_COL_FWD ? (long long)grid_w : 1) * onward;
    c.wrap = (1 - (long long)(grid_h - 1) * grid_w) * onward;
    c.dtype = dtype;
    c.kind = kind;
    c.rest = complement != 0;
    c.inv_tau = kind == GLA_GATE_PRE ? 1.f / tau : 1.f;
    return GLA_OK;
}
bool sized_recur(RecurCall &c, bool back, int B, int T, int D) {
    return check_recur(c, back, nullptr, nullptr, GLA_GATE_LOG, 1.f, 0, nullptr, B, T, D, 1, T, 0, GLA_DT_F32, GLA_DT_F32) == GLA_OK;
}

// --- norm and rotation of queries and keys ---

// Bytes from the first element of a tensor's first row to behind the last of its last
size_t reach(const QkSide &s, int B, int T, int d, int dtype) {
    return (size_t)((B - 1) * s.sb + (s.heads - 1) * s.sh + (T - 1) * s.st + d) * size_of(dtype);
}
int side_in(QkSide &s, const void *x, const long long *strides, const float *weight, int B, int heads, int T, int d, int layout) {
    s.x = x;
    s.weight = weight;
    s.heads = x != nullptr ? heads : 0;
    if (strides != nullptr) {
        s.sb = strides[0];
        s.sh = strides[1];
        s.st = strides[2];
        // (elements to the last batch, head and token: what they add up to has to be an address)
        const long long strides_of[] = {s.sb, s.sh, s.st}, counts[] = {B, heads, T};
        for (int i = 0; i < 3; ++i)
            if (strides_of[i] < 0 || strides_of[i] > (1LL << 40) / (counts[i] > 1 ? counts[i] - 1 : 1)) return GLA_ERR_SHAPE;
    } else {
        s.sb = (long long)heads * T * d;
        s.sh = layout == GLA_LAYOUT_BHTD ? (long long)T * d : d;
        s.st = layout == GLA_LAYOUT_BHTD ? d : (long long)heads * d;
    }
    return GLA_OK;
}
int check_qk(QkParams &p, const void *q, const long long *q_strides, int H, const void *k, const long long *k_strides, int Hk, const float *q_weight,
             const float *k_weight, float eps, const int *positions, const int *sections, int axes, float base, int pairing, int B, int T, int d, int grid_h,
             int grid_w, int dtype, int other_dtype, int layout) {
    if (!q || (axes > 0 && !sections) || (!k && k_weight)) return GLA_ERR_NULL;
    if (B <= 0 || H <= 0 || T <= 0 || d <= 0 || (k && Hk <= 0) || axes < 0 || bad_dtype(dtype) || bad_dtype(other_dtype) ||
        (layout != GLA_LAYOUT_BHTD && layout != GLA_LAYOUT_BTHD) || (pairing != GLA_ROPE_ADJACENT && pairing != GLA_ROPE_HALVES) || !(eps >= 0.f) || isinf(eps))
        return GLA_ERR_SHAPE;
    if (axes > 0 && (!(base > 0.f) || isinf(base))) return GLA_ERR_SHAPE;
    if (axes > kRopeMaxAxes || d > kRopeMaxD) return GLA_ERR_UNSUPPORTED;
    p = {};
    if (axes > 0) {
        const int st = rope_turns(p.rope, positions, sections, axes, base, T, d, grid_h, grid_w);
        if (st != GLA_OK) return st;
    }
    // 32-bit numbers of tokens and heads
    if ((long long)B * T >= (1LL << 31) || H > (1 << 20) || Hk > (1 << 20)) return GLA_ERR_UNSUPPORTED;
    int st = side_in(p.side[0], q, q_strides, q_weight, B, H, T, d, layout);
    if (st == GLA_OK) st = side_in(p.side[1], k, k_strides, k_weight, B, Hk, T, d, layout);
    if (st != GLA_OK) return st;
    if (off_element(q, dtype) || off_element(k, dtype) || any_misaligned((const void *)q_weight, (const void *)k_weight) ||
        (reinterpret_cast<uintptr_t>(positions) & 3u) != 0)
        return GLA_ERR_ALIGN;
    p.rope.B = B;
    p.rope.T = T;
    p.rope.d = d;
    p.rope.layout = layout;
    p.rope.adjacent = pairing == GLA_ROPE_ADJACENT;
    p.eps = eps;
    p.out_dtype = other_dtype;
    return GLA_OK;
}
// whether a tensor of rows lies dense in the layout's order
bool dense(const QkSide &s, int B, int T, int d, int layout) {
    return (B == 1 || s.sb == (long long)s.heads * T * d) && (s.heads == 1 || s.sh == (layout == GLA_LAYOUT_BHTD ? (long long)T * d : d)) &&
           (T == 1 || s.st == (layout == GLA_LAYOUT_BHTD ? d : (long long)s.heads * d));
}

// --- gated feed-forward product ---

constexpr int kGluMost = 1 << 20;       // columns: rows of a tile in 32-bit offsets
int whole_pieces(int n, int dtype) {    // elements of rows in pieces of 16 bytes
    const int each = 16 / (int)size_of(dtype);
    return (n + each - 1) / each * each;
}
// Copies of operands whose rows are no whole pieces, and the backward pass's arrays, in a workspace (null: it only counts)
struct GluRoom {
    char *x, *w_gate, *w_up, *dg[2], *du[2];
    float *part;
    size_t bytes;
};
GluRoom glu_room(void *workspace, int M, int K, int F, int dtype, bool back, bool split) {
    GluRoom r = {};
    char *base = static_cast<char *>(workspace);
    auto take = [&](size_t rows, size_t cols, size_t each) {
        char *p = base == nullptr ? nullptr : base + r.bytes;
        r.bytes += align_up(rows * cols * each);
        return p;
    };
    const int ld = whole_pieces(K, dtype);
    if (ld != K) {
        r.x = take(M, ld, size_of(dtype));
        r.w_gate = take(F, ld, size_of(dtype));
        r.w_up = take(F, ld, size_of(dtype));
    }
    if (back) {
        for (int i = 0; i < (split ? 2 : 1); ++i) {
            r.dg[i] = take(M, whole_pieces(F, dtype), size_of(dtype));
            r.du[i] = take(M, whole_pieces(F, dtype), size_of(dtype));
        }
        r.part = reinterpret_cast<float *>(take(1, glu_part_bytes(M, K, F, dtype, split), 1));
    }
    return r;
}
bool glu_split(int dtype) { return dtype == GLA_DT_BF16 && gla_get_option(GLA_OPT_GLU_SPLIT) != 0; }
int check_glu(const void *x, const void *w_gate, const void *w_up, int M, int K, int F, int act, int dtype, int other_dtype) {
    if (M <= 0 || K <= 0 || F <= 0 || bad_dtype(dtype) || bad_dtype(other_dtype) || act < GLA_ACT_SILU || act > GLA_ACT_GELU_TANH) return GLA_ERR_SHAPE;
    // (tiles of 128 rows and columns, and four columns a thread, in launches of fewer than 2^32 threads)
    const long long most = K > F ? K : F;
    if (K > kGluMost || F > kGluMost || M > (1 << 28) || M * (most + 8) >= (1LL << 34) || F * (long long)(K + 8) >= (1LL << 32)) return GLA_ERR_UNSUPPORTED;
    return any_misaligned(x, w_gate, w_up) ? GLA_ERR_ALIGN : GLA_OK;
}
// The call's operands, copied where their rows are no whole pieces
int glu_operands(GluCall &c, const GluRoom &room, const void *x, const void *w_gate, const void *w_up, int M, int K, int F, int act, int dtype, hipStream_t stream) {
    c = {};
    c.M = M;
    c.K = K;
    c.F = F;
    c.dtype = dtype;
    c.act = act;
    c.ld_x = c.ld_w = whole_pieces(K, dtype);
    c.ld_f = whole_pieces(F, dtype);
    const bool copied = room.x != nullptr;
    c.x = copied ? room.x : x;
    c.w_gate = copied ? room.w_gate : w_gate;
    c.w_up = copied ? room.w_up : w_up;
    return !copied || launch_glu_pad(c, x, w_gate, w_up, stream) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

}  // namespace
}  // namespace gla

using namespace gla;

extern "C" {

size_t gla_recur_fwd_workspace_bytes(int B, int T, int D) {
    RecurCall c;
    if (!sized_recur(c, false, B, T, D)) return 0;
    return chain_bytes(c);
}
size_t gla_recur_bwd_workspace_bytes(int B, int T, int D) {
    RecurCall c;
    if (!sized_recur(c, true, B, T, D)) return 0;
    return units_bytes(c);
}

int gla_recur_fwd(const void *x, const void *gate, int gate_kind, float tau, int complement, const int *seq_lens, int B, int T, int D,
                  int grid_h, int grid_w, int scan_dir, int x_dtype, int out_dtype, const float *initial_state, void *out, float *final_state,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream_) {
    if (!x || !gate || !out) return GLA_ERR_NULL;
    RecurCall c;
    const int st = check_recur(c, false, x, gate, gate_kind, tau, complement, seq_lens, B, T, D, grid_h, grid_w, scan_dir, x_dtype, out_dtype);
    if (st != GLA_OK) return st;
    if (any_misaligned((const void *)initial_state, (const void *)out, (const void *)final_state)) return GLA_ERR_ALIGN;
    const int gate_dtype = gate_kind == GLA_GATE_LOG ? GLA_DT_F32 : x_dtype;
    const size_t n = (size_t)B * T * D, state_bytes = (size_t)B * D * sizeof(float);
    const Span xs = {x, n * size_of(x_dtype)}, gs = {gate, n * size_of(gate_dtype)}, os = {out, n * size_of(out_dtype)};
    const Span first = {initial_state, state_bytes}, last = {final_state, state_bytes};
    // (in place is each element's own place: a wave has read its rows before it writes them)
    const bool in_place = touch(os, xs) || touch(os, gs) || touch(first, last);
    if (touch(os, xs) && (out != x || out_dtype != x_dtype)) return GLA_ERR_SHAPE;
    if (touch(os, gs) && (out != gate || out_dtype != gate_dtype)) return GLA_ERR_SHAPE;
    if (touch(os, first) || touch(os, last) || touch(last, xs) || touch(last, gs) || (touch(first, last) && initial_state != final_state)) return GLA_ERR_SHAPE;
    if (chain_bytes(c) > 0 && (!workspace || misaligned(workspace) || workspace_bytes < chain_bytes(c))) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    const hipError_t e = c.nunits == 1 ? launch_recur_walk(c, initial_state, out, out_dtype, final_state, stream)
                                       : launch_recur_chain(c, chain_in(c, workspace, in_place), initial_state, out, out_dtype, final_state, stream);
    return e == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_recur_bwd(const void *x, const void *gate, int gate_kind, float tau, int complement, const int *seq_lens, const void *d_out,
                  const float *initial_state, const float *d_final_state, int B, int T, int D, int grid_h, int grid_w, int scan_dir, int x_dtype,
                  int grad_dtype, void *dx, void *d_gate, float *d_initial_state, void *workspace, size_t workspace_bytes, gla_stream_t stream_) {
    if (!x || !gate || !d_out || !dx || !d_gate) return GLA_ERR_NULL;
    RecurCall c;
    const int st = check_recur(c, true, x, gate, gate_kind, tau, complement, seq_lens, B, T, D, grid_h, grid_w, scan_dir, x_dtype, grad_dtype);
    if (st != GLA_OK) return st;
    if (any_misaligned(d_out, (const void *)initial_state, (const void *)d_final_state, (const void *)dx, (const void *)d_gate, (const void *)d_initial_state))
        return GLA_ERR_ALIGN;
    const size_t n = (size_t)B * T * D, state_bytes = (size_t)B * D * sizeof(float);
    const Span outs[] = {{dx, n * size_of(grad_dtype)}, {d_gate, n * size_of(grad_dtype)}, {d_initial_state, state_bytes}};
    const Span ins[] = {{x, n * size_of(x_dtype)}, {gate, n * size_of(gate_kind == GLA_GATE_LOG ? GLA_DT_F32 : x_dtype)}, {d_out, n * size_of(x_dtype)},
                        {initial_state, state_bytes}, {d_final_state, state_bytes}};
    if (any_touch(outs, ins)) return GLA_ERR_SHAPE;
    if (units_bytes(c) > 0 && (!workspace || misaligned(workspace) || workspace_bytes < units_bytes(c))) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    const RecurUnits u = c.nunits > 1 ? units_in(c, workspace) : RecurUnits{};
    if (c.nunits > 1) {
        if (launch_recur_units(c, d_out, u, stream) != hipSuccess) return GLA_ERR_HIP;
        if (launch_recur_carry(c, u, initial_state, d_final_state, d_initial_state, stream) != hipSuccess) return GLA_ERR_HIP;
    }
    return launch_recur_back(c, d_out, u, initial_state, d_final_state, dx, d_gate, grad_dtype, d_initial_state, stream) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_recur_step(const void *x, const void *gate, int gate_kind, float tau, int complement, int B, int D, int x_dtype, int out_dtype,
                   const float *state, float *state_out, void *out, gla_stream_t stream) {
    if (!x || !gate || !state || !state_out || !out) return GLA_ERR_NULL;
    if (B <= 0 || D <= 0 || bad_dtype(x_dtype) || bad_dtype(out_dtype) || (gate_kind != GLA_GATE_LOG && gate_kind != GLA_GATE_PRE)) return GLA_ERR_SHAPE;
    if (gate_kind == GLA_GATE_PRE && bad_tau(tau)) return GLA_ERR_SHAPE;
    if ((long long)B * D >= (1LL << 31)) return GLA_ERR_UNSUPPORTED;
    const int gate_dtype = gate_kind == GLA_GATE_LOG ? GLA_DT_F32 : x_dtype;
    if (any_misaligned((const void *)state, (const void *)state_out) || off_element(x, x_dtype) || off_element(gate, gate_dtype) || off_element(out, out_dtype))
        return GLA_ERR_ALIGN;
    const size_t n = (size_t)B * D;
    const Span outs[] = {{out, n * size_of(out_dtype)}};
    const Span others[] = {{x, n * size_of(x_dtype)}, {gate, n * size_of(gate_dtype)}, {state, n * 4}, {state_out, n * 4}};
    if (any_touch(outs, others)) return GLA_ERR_SHAPE;
    if (touch(others[2], others[3]) && state != state_out) return GLA_ERR_SHAPE;
    if (touch(others[3], others[0]) || touch(others[3], others[1])) return GLA_ERR_SHAPE;
    RecurCall c = {};
    c.x = x;
    c.gate = gate;
    c.B = B;
    c.T = 1;
    c.D = D;
    c.dtype = x_dtype;
    c.kind = gate_kind;
    c.rest = complement != 0;
    c.inv_tau = gate_kind == GLA_GATE_PRE ? 1.f / tau : 1.f;
    return launch_recur_step(c, state, state_out, out, out_dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_qk_norm_fwd(const void *q, const long long *q_strides, int H, const void *k, const long long *k_strides, int Hk, const float *q_weight,
                    const float *k_weight, float eps, const int *positions, const int *sections, int axes, float base, int pairing, int B, int T, int d,
                    int grid_h, int grid_w, int dtype, int out_dtype, int layout, void *out_q, void *out_k, gla_stream_t stream) {
    if (!out_q || (k == nullptr) != (out_k == nullptr)) return GLA_ERR_NULL;
    QkParams p;
    const int st = check_qk(p, q, q_strides, H, k, k_strides, Hk, q_weight, k_weight, eps, positions, sections, axes, base, pairing, B, T, d, grid_h, grid_w, dtype,
                            out_dtype, layout);
    if (st != GLA_OK) return st;
    if (any_misaligned((const void *)out_q, (const void *)out_k)) return GLA_ERR_ALIGN;
    const size_t row = (size_t)B * T * d * size_of(out_dtype);
    const Span xs[] = {{q, reach(p.side[0], B, T, d, dtype)}, {k, k != nullptr ? reach(p.side[1], B, T, d, dtype) : 0}};
    const Span ys[] = {{out_q, H * row}, {out_k, Hk * row}};
    // in place is each row's own place
    if (touch(ys[0], ys[1]) || touch(ys[0], xs[1]) || touch(ys[1], xs[0])) return GLA_ERR_SHAPE;
    for (int i = 0; i < 2; ++i)
        if (touch(xs[i], ys[i]) && (xs[i].p != ys[i].p || dtype != out_dtype || !dense(p.side[i], B, T, d, layout))) return GLA_ERR_SHAPE;
    p.side[0].out = out_q;
    p.side[1].out = out_k;
    return launch_qk_fwd(p, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

size_t gla_qk_norm_bwd_workspace_bytes(int B, int H, int Hk, int T, int d) {
    if (B <= 0 || H <= 0 || Hk < 0 || T <= 0 || d <= 0 || d > kRopeMaxD || (long long)B * T >= (1LL << 31)) return 0;
    return 2 * align_up((size_t)qk_slots(B, T) * d * sizeof(float));
}

int gla_qk_norm_bwd(const void *q, const long long *q_strides, int H, const void *k, const long long *k_strides, int Hk, const void *d_out_q, const void *d_out_k,
                    const float *q_weight, const float *k_weight, float eps, const int *positions, const int *sections, int axes, float base, int pairing, int B,
                    int T, int d, int grid_h, int grid_w, int dtype, int grad_dtype, int layout, void *dq, void *dk, float *dq_weight, float *dk_weight,
                    void *workspace, size_t workspace_bytes, gla_stream_t stream) {
    if (!d_out_q || !dq || (k == nullptr) != (dk == nullptr) || (k == nullptr) != (d_out_k == nullptr) || (!k && dk_weight)) return GLA_ERR_NULL;
    QkParams p;
    const int st = check_qk(p, q, q_strides, H, k, k_strides, Hk, q_weight, k_weight, eps, positions, sections, axes, base, pairing, B, T, d, grid_h, grid_w, dtype,
                            grad_dtype, layout);
    if (st != GLA_OK) return st;
    if (any_misaligned(d_out_q, d_out_k, (const void *)dq, (const void *)dk, (const void *)dq_weight, (const void *)dk_weight)) return GLA_ERR_ALIGN;
    const size_t n = (size_t)B * T * d;
    const Span outs[] = {{dq, n * H * size_of(grad_dtype)}, {dk, n * Hk * size_of(grad_dtype)}, {dq_weight, d * sizeof(float)}, {dk_weight, d * sizeof(float)}};
    const Span ins[] = {{q, reach(p.side[0], B, T, d, dtype)}, {k, k != nullptr ? reach(p.side[1], B, T, d, dtype) : 0}, {d_out_q, n * H * size_of(dtype)},
                        {d_out_k, n * Hk * size_of(dtype)}, {q_weight, d * sizeof(float)}, {k_weight, d * sizeof(float)}};
    if (any_touch(outs, ins)) return GLA_ERR_SHAPE;
    if ((dq_weight || dk_weight) && (!workspace || misaligned(workspace) || workspace_bytes < gla_qk_norm_bwd_workspace_bytes(B, H, k ? Hk : 0, T, d)))
        return GLA_ERR_WORKSPACE;
    p.slots = qk_slots(B, T);
    char *room = static_cast<char *>(workspace);
    const void *ups[] = {d_out_q, d_out_k};
    void *const downs[] = {dq, dk};
    float *const sums[] = {dq_weight, dk_weight};
    for (int i = 0; i < 2; ++i) {
        p.side[i].d_out = ups[i];
        p.side[i].out = downs[i];
        p.side[i].dweight = sums[i];
        p.side[i].part = sums[i] != nullptr ? reinterpret_cast<float *>(room + i * align_up((size_t)p.slots * d * sizeof(float))) : nullptr;
    }
    return launch_qk_bwd(p, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

size_t gla_glu_fwd_workspace_bytes(int M, int K, int F, int dtype) {
    return check_glu(nullptr, nullptr, nullptr, M, K, F, 0, dtype, dtype) == GLA_OK ? glu_room(nullptr, M, K, F, dtype, false, false).bytes : 0;
}
size_t gla_glu_bwd_workspace_bytes(int M, int K, int F, int dtype) {
    return check_glu(nullptr, nullptr, nullptr, M, K, F, 0, dtype, dtype) == GLA_OK ? glu_room(nullptr, M, K, F, dtype, true, glu_split(dtype)).bytes : 0;
}

int gla_glu_fwd(const void *x, const void *w_gate, const void *w_up, int M, int K, int F, int act, int dtype, int out_dtype, void *out, float *pre, void *workspace,
                size_t workspace_bytes, gla_stream_t stream_) {
    if (!x || !w_gate || !w_up || !out) return GLA_ERR_NULL;
    const int st = check_glu(x, w_gate, w_up, M, K, F, act, dtype, out_dtype);
    if (st != GLA_OK) return st;
    if (any_misaligned((const void *)out, (const void *)pre)) return GLA_ERR_ALIGN;
    const size_t xs = (size_t)M * K * size_of(dtype), ws = (size_t)F * K * size_of(dtype), n = (size_t)M * F;
    const Span outs[] = {{out, n * size_of(out_dtype)}, {pre, 2 * n * sizeof(float)}};
    const Span ins[] = {{x, xs}, {w_gate, ws}, {w_up, ws}};
    if (any_touch(outs, ins)) return GLA_ERR_SHAPE;
    const GluRoom room = glu_room(workspace, M, K, F, dtype, false, false);
    if (room.bytes > 0 && (!workspace || misaligned(workspace) || workspace_bytes < room.bytes)) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    GluCall c;
    const int laid = glu_operands(c, room, x, w_gate, w_up, M, K, F, act, dtype, stream);
    if (laid != GLA_OK) return laid;
    return launch_glu_fwd(c, out, out_dtype, pre, stream) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_glu_bwd(const void *x, const void *w_gate, const void *w_up, const void *d_out, const float *pre, int M, int K, int F, int act, int dtype, void *dx,
                void *dw_gate, void *dw_up, void *workspace, size_t workspace_bytes, gla_stream_t stream_) {
    if (!x || !w_gate || !w_up || !d_out || (dw_gate == nullptr) != (dw_up == nullptr) || (!dx && !dw_gate)) return GLA_ERR_NULL;
    const int st = check_glu(x, w_gate, w_up, M, K, F, act, dtype, dtype);
    if (st != GLA_OK) return st;
    if (any_misaligned(d_out, (const void *)pre, (const void *)dx, (const void *)dw_gate, (const void *)dw_up)) return GLA_ERR_ALIGN;
    const size_t xs = (size_t)M * K * size_of(dtype), ws = (size_t)F * K * size_of(dtype), n = (size_t)M * F;
    const Span outs[] = {{dx, xs}, {dw_gate, ws}, {dw_up, ws}};
    const Span ins[] = {{x, xs}, {w_gate, ws}, {w_up, ws}, {d_out, n * size_of(dtype)}, {pre, 2 * n * sizeof(float)}};
    if (any_touch(outs, ins)) return GLA_ERR_SHAPE;
    const GluRoom room = glu_room(workspace, M, K, F, dtype, true, glu_split(dtype));
    if (!workspace || misaligned(workspace) || workspace_bytes < room.bytes) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    GluCall c;
    const int laid = glu_operands(c, room, x, w_gate, w_up, M, K, F, act, dtype, stream);
    if (laid != GLA_OK) return laid;
    c.d_out = d_out;
    for (int i = 0; i < 2; ++i) {
        c.dg[i] = room.dg[i];
        c.du[i] = room.du[i];
    }
    c.part = room.part;
    if (launch_glu_slopes(c, pre, stream) != hipSuccess) return GLA_ERR_HIP;
    if (dx != nullptr && launch_glu_dx(c, dx, stream) != hipSuccess) return GLA_ERR_HIP;
    if (dw_gate != nullptr && launch_glu_dw(c, dw_gate, dw_up, stream) != hipSuccess) return GLA_ERR_HIP;
    return GLA_OK;
}

}  // extern "C"
