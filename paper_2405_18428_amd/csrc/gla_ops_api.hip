// Host side of the C ABI for linear attention with one decay a head, rotary positions and layer norm: argument checks, span plan,
// workspaces.
#include <math.h>
#include <string.h>

#include "gla_decay.h"
#include "gla_ops.h"

namespace gla {
namespace {

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
template <typename... P>
bool any_misaligned(P... p) { return (misaligned(p) || ...); }
bool off_element(const void *p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == GLA_DT_BF16 ? 1u : 3u)) != 0; }
bool bad_dtype(int d) { return d != GLA_DT_F32 && d != GLA_DT_BF16; }
// whether two tensors share memory without beginning at one place (null: none)
bool overlap(const void *p, size_t p_bytes, const void *q, size_t q_bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a != 0 && b != 0 && a != b && a < b + q_bytes && b < a + p_bytes;
}
size_t size_of(int dtype) { return dtype == GLA_DT_BF16 ? 2 : 4; }
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// Spans a sequence is walked in.  One work-group walks one span, so that few sequences leave most of the GPU idle; spans read y and z once
// more for their local states, and move their states.  Spans as short as 64 steps pay while there are up to 16 (16 sequences of 512 steps,
// 128 x 128, forward and back: 83 us in spans of 64, 108 of 128, 133 of 256; of 2048 steps 148 in 32 spans, 134 in 16), beyond that only
// such of 512 and more, and two chunks do not pay for the second pass (64 sequences of 128 steps forward: 23 us in two spans, 17 in one).
constexpr int kShortSpans = 16, kLongSpan = 512, kWhole = 128;
// Up to so many spans the walks chain the local states themselves (padded prompts of 128 sequences in 4 spans: 101 us, 112 with the
// kernel for it; at 8 spans it is even).
constexpr int kChainSpans = 4;
void plan_spans(DecayCall &c, long long groups) {
    const long long bh = (long long)c.B * c.H;
    const int units = (c.T + 63) / 64;
    long long most = c.T / kLongSpan;
    if (most < kShortSpans) most = kShortSpans;
    if (most > units) most = units;
    long long n = groups / bh;
    if (n > most) n = most;
    if (n < 1 || c.T <= kWhole) n = 1;
    const int each = (int)((units + n - 1) / n);
    c.span_len = each * 64;
    c.nspans = (units + each - 1) / each;
}

// Cuts a workspace into a call's arrays; without one (null) it only counts
struct Room {
    size_t used = 0;
    char *base;
    explicit Room(void *p) : base(static_cast<char *>(p)) {}
    template <typename E>
    E *take(size_t n) {
        const size_t at = used;
        used += align_up(n * sizeof(E));
        return base == nullptr ? nullptr : reinterpret_cast<E *>(base + at);
    }
};

struct FwdRoom {
    float *local, *decay;
    size_t bytes;
};
FwdRoom fwd_room(void *p, const DecayCall &c) {
    Room r(p);
    FwdRoom f = {};
    if (c.nspans > 1) {
        const size_t n = (size_t)c.B * c.H * c.nspans;
        f.local = r.take<float>(n * c.dk * c.dv);
        f.decay = r.take<float>(n);
    }
    f.bytes = r.used;
    return f;
}
struct BwdRoom {
    float *local, *decay, *glocal, *gdecay, *flow_q, *flow_k, *anchors, *meet;
    double *part;
    size_t bytes;
};
// the walk back has work-groups twice as large
DecayCall back_call(DecayCall c) {
    plan_spans(c, 256);
    return c;
}
BwdRoom bwd_room(void *p, const DecayCall &c) {
    Room r(p);
    BwdRoom f = {};
    const size_t bh = (size_t)c.B * c.H, blocks = bh * decay_blocks(c.T), cells = (size_t)c.dk * c.dv;
    if (c.nspans > 1) {
        f.local = r.take<float>(bh * c.nspans * cells);
        f.decay = r.take<float>(bh * c.nspans);
    }
    const int back = back_call(c).nspans;
    if (back > 1) {
        f.glocal = r.take<float>(bh * back * cells);
        f.gdecay = r.take<float>(bh * back);
    }
    f.flow_q = r.take<float>(bh * c.T);
    f.flow_k = r.take<float>(bh * c.T);
    f.anchors = r.take<float>(blocks * cells);
    f.meet = r.take<float>(blocks);
    f.part = r.take<double>(blocks);
    f.bytes = r.used;
    return f;
}

int check_call(DecayCall &c, const float *log_decay, int kind, const int *seq_lens, int B, int H, int T, int dk, int dv, int grid_h,
               int grid_w, int scan_dir, int dtype, int out_dtype, int layout) {
    if (B <= 0 || H <= 0 || T <= 0 || dk <= 0 || dv <= 0 || grid_h <= 0 || grid_w <= 0) return GLA_ERR_SHAPE;
    if ((long long)grid_h * grid_w != T || scan_dir < 0 || scan_dir > 3 || (layout != GLA_LAYOUT_BHTD && layout != GLA_LAYOUT_BTHD))
        return GLA_ERR_SHAPE;
    if (bad_dtype(dtype) || bad_dtype(out_dtype) || (kind != GLA_DECAY_HEAD && kind != GLA_DECAY_TOKEN)) return GLA_ERR_SHAPE;
    if (dk > kDecayMaxD || dv > kDecayMaxD) return GLA_ERR_UNSUPPORTED;
    if (seq_lens != nullptr && scan_dir > GLA_SCAN_ROW_REV) return GLA_ERR_UNSUPPORTED;
    // (work-groups of 512 threads, fewer than 2^32 threads in a launch; steps and spans in 32 bits)
    if (T > (1 << 30) || (long long)B * H * decay_blocks(T) >= (1LL << 23)) return GLA_ERR_UNSUPPORTED;
    if (misaligned(log_decay) || (reinterpret_cast<uintptr_t>(seq_lens) & 3u) != 0) return GLA_ERR_ALIGN;
    c.log_decay = log_decay;
    c.seq_lens = seq_lens;
    c.kind = kind == GLA_DECAY_HEAD ? kDecayHead : kDecayToken;
    c.B = B;
    c.H = H;
    c.T = T;
    c.dk = dk;
    c.dv = dv;
    c.grid_h = grid_h;
    c.grid_w = grid_w;
    c.scan_dir = scan_dir;
    c.layout = layout;
    // rows of whole dwords, at least one piece of 16 bytes long; 24-bit factors; offsets inside a chunk below 2^31 (a column's rows lie
    // all over the sequence)
    const long long wide = dk > dv ? dk : dv, least = dk < dv ? dk : dv, step = wide * 4 * (layout == GLA_LAYOUT_BTHD ? H : 1);
    const long long reach = (scan_dir >= GLA_SCAN_COL_FWD ? T : 64) * step;
    c.fast = dk % 4 == 0 && dv % 4 == 0 && least * (dtype == GLA_DT_BF16 ? 2 : 4) >= 16 && step < (1LL << 24) && T < (1 << 24) &&
             reach < (1LL << 31) - (1 << 16);
    plan_spans(c, 512);                  // two work-groups a compute unit
    return GLA_OK;
}

// How the walks get at the states that enter their spans: up to kChainSpans they chain the local ones themselves, beyond that a kernel of its
// own does so in place, and also where the last state is written over the first, which other spans may not have read by then
void enter_by(DecayEntry &in, const DecayCall &c, float *local, const float *decay, const float *last) {
    in.local = local;
    in.decay = decay;
    in.chained = c.nspans > 1 && (c.nspans > kChainSpans || (last != nullptr && last == in.first));
}

bool sized(DecayCall &c, int B, int H, int T, int dk, int dv, int dtype) {
    return check_call(c, nullptr, GLA_DECAY_HEAD, nullptr, B, H, T, dk, dv, 1, T, 0, dtype, dtype, 0) == GLA_OK;
}

}  // namespace
}  // namespace gla

using namespace gla;

extern "C" {

size_t gla_decay_fwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype) {
    DecayCall c = {};
    return sized(c, B, H, T, dk, dv, qkv_dtype) ? fwd_room(nullptr, c).bytes : 0;
}
size_t gla_decay_bwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype) {
    DecayCall c = {};
    return sized(c, B, H, T, dk, dv, qkv_dtype) ? bwd_room(nullptr, c).bytes : 0;
}

int gla_decay_fwd(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind, const int *seq_lens, int B, int H,
                  int T, int dk, int dv, int grid_h, int grid_w, int scan_dir, int qkv_dtype, int out_dtype, int layout,
                  const float *initial_state, void *out, float *final_state, void *workspace, size_t workspace_bytes, gla_stream_t stream_) {
    if (!q || !k || !v || !log_decay || !out) return GLA_ERR_NULL;
    DecayCall c = {};
    const int st = check_call(c, log_decay, decay_kind, seq_lens, B, H, T, dk, dv, grid_h, grid_w, scan_dir, qkv_dtype, out_dtype, layout);
    if (st != GLA_OK) return st;
    if (any_misaligned(q, k, v, (const void *)initial_state, (const void *)out, (const void *)final_state)) return GLA_ERR_ALIGN;
    // in place, or apart from each other: elsewhere one state would be written over another that is still to be read
    const size_t state_bytes = (size_t)B * H * dk * dv * sizeof(float);
    if (overlap(initial_state, state_bytes, final_state, state_bytes)) return GLA_ERR_SHAPE;
    const FwdRoom room = fwd_room(workspace, c);
    if (room.bytes > 0 && (!workspace || misaligned(workspace) || workspace_bytes < room.bytes)) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    c.digits = final_state != nullptr ? kDigitsStates : kDigitsRows;
    DecayWalk w = {};
    w.c = c;
    w.r.x = q;
    w.r.y = k;
    w.r.z = v;
    w.r.out = out;
    w.r.m = dk;
    w.r.n = dv;
    w.in.first = initial_state;
    w.state_out = final_state;
    w.out_dtype = out_dtype;
    if (c.nspans > 1) {
        w.local = room.local;
        w.decay = room.decay;
        if (launch_decay_states(w, nullptr, qkv_dtype, stream) != hipSuccess) return GLA_ERR_HIP;
        enter_by(w.in, c, room.local, room.decay, final_state);
        const DecayChain chain = {initial_state, room.local, room.decay, c.nspans, 0};
        if (w.in.chained && launch_decay_carry(c, chain, nullptr, stream) != hipSuccess) return GLA_ERR_HIP;
    }
    return launch_decay_walk(w, qkv_dtype, stream) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_decay_bwd(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind, const int *seq_lens,
                  const void *d_out, const float *initial_state, const float *d_final_state, int B, int H, int T, int dk, int dv, int grid_h,
                  int grid_w, int scan_dir, int qkv_dtype, int grad_dtype, int layout, void *dq, void *dk_grad, void *dv_grad,
                  float *dlog_decay, float *d_initial_state, void *workspace, size_t workspace_bytes, gla_stream_t stream_) {
    if (!q || !k || !v || !log_decay || !d_out || !dq || !dk_grad || !dv_grad) return GLA_ERR_NULL;
    DecayCall c = {};
    const int st = check_call(c, log_decay, decay_kind, seq_lens, B, H, T, dk, dv, grid_h, grid_w, scan_dir, qkv_dtype, grad_dtype, layout);
    if (st != GLA_OK) return st;
    if (any_misaligned(q, k, v, d_out, (const void *)initial_state, (const void *)d_final_state, (const void *)dq, (const void *)dk_grad,
                       (const void *)dv_grad, (const void *)dlog_decay, (const void *)d_initial_state))
        return GLA_ERR_ALIGN;
    const BwdRoom room = bwd_room(workspace, c);
    if (!workspace || misaligned(workspace) || workspace_bytes < room.bytes) return GLA_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(stream_);
    const bool gates = dlog_decay != nullptr;
    c.digits = gates && c.kind == kDecayHead ? kDigitsAll : d_initial_state != nullptr ? kDigitsStates : kDigitsRows;

    DecayWalk w = {};                    // dq: the recurrence of (dO, v, k) from the transposed states
    w.c = c;
    w.r.x = d_out;
    w.r.y = v;
    w.r.z = k;
    w.r.out = dq;
    w.r.dot = gates ? q : nullptr;
    w.r.flow = room.flow_q;
    w.r.m = dv;
    w.r.n = dk;
    w.in.first = initial_state;
    w.state_t = 1;
    w.anchors = gates ? room.anchors : nullptr;
    w.anchor_last = d_final_state != nullptr;
    w.out_dtype = grad_dtype;
    w.grad = 1;
    DecayBack b = {};
    b.c = back_call(c);
    b.q = q;
    b.k = k;
    b.v = v;
    b.d_out = d_out;
    b.dk_grad = dk_grad;
    b.dv_grad = dv_grad;
    b.in.first = d_final_state;
    b.d_initial = d_initial_state;
    b.anchors = w.anchors;
    b.anchor_last = w.anchor_last;
    b.meet = room.meet;
    b.flow_k = room.flow_k;
    b.grad_dtype = grad_dtype;
    if (c.nspans > 1) {                  // (then perhaps b.c.nspans too)
        DecayWalk s = {}, g = {};
        s.c = c;
        g.c = b.c;
        s.r.y = k;
        s.r.z = v;
        g.r.y = q;
        g.r.z = d_out;
        s.r.m = g.r.m = dk;
        s.r.n = g.r.n = dv;
        s.local = room.local;
        s.decay = room.decay;
        g.local = room.glocal;
        g.decay = room.gdecay;
        if (launch_decay_states(s, b.c.nspans > 1 ? &g : nullptr, qkv_dtype, stream) != hipSuccess) return GLA_ERR_HIP;
        enter_by(w.in, c, room.local, room.decay, nullptr);
        enter_by(b.in, b.c, room.glocal, room.gdecay, d_initial_state);
        const DecayChain chain = {initial_state, room.local, room.decay, c.nspans, 0};
        const DecayChain back = {d_final_state, room.glocal, room.gdecay, b.c.nspans, 1};
        if (w.in.chained || b.in.chained) {
            const DecayChain &one = w.in.chained ? chain : back;
            if (launch_decay_carry(c, one, w.in.chained && b.in.chained ? &back : nullptr, stream) != hipSuccess) return GLA_ERR_HIP;
        }
    }
    if (launch_decay_walk(w, qkv_dtype, stream) != hipSuccess) return GLA_ERR_HIP;
    if (launch_decay_back(b, qkv_dtype, stream) != hipSuccess) return GLA_ERR_HIP;
    if (!gates) return GLA_OK;
    DecayGate d = {};
    d.c = c;
    d.flow_q = room.flow_q;
    d.flow_k = room.flow_k;
    d.meet = room.meet;
    d.anchor_last = w.anchor_last;
    d.dlog = dlog_decay;
    d.part = room.part;
    return launch_decay_gate(d, stream) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

int gla_decay_step(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind, int B, int H, int dk, int dv,
                   int qkv_dtype, int out_dtype, const float *state, float *state_out, void *out, gla_stream_t stream) {
    if (!q || !k || !v || !log_decay || !state || !state_out || !out) return GLA_ERR_NULL;
    if (B <= 0 || H <= 0 || dk <= 0 || dv <= 0 || bad_dtype(qkv_dtype) || bad_dtype(out_dtype) ||
        (decay_kind != GLA_DECAY_HEAD && decay_kind != GLA_DECAY_TOKEN))
        return GLA_ERR_SHAPE;
    if (dk > kDecayMaxD || dv > kDecayMaxD || (long long)B * H >= (1LL << 22)) return GLA_ERR_UNSUPPORTED;
    // (rows of single tokens are often slices of something larger: any place does for them)
    if (any_misaligned((const void *)state, (const void *)state_out) || off_element(q, qkv_dtype) || off_element(k, qkv_dtype) ||
        off_element(v, qkv_dtype) || off_element(out, out_dtype) || off_element(log_decay, GLA_DT_F32))
        return GLA_ERR_ALIGN;
    // (as gla_decay_fwd's)
    const size_t bytes = (size_t)B * H * dk * dv * sizeof(float);
    if (overlap(state, bytes, state_out, bytes)) return GLA_ERR_SHAPE;
    return launch_decay_step(q, k, v, log_decay, decay_kind == GLA_DECAY_HEAD ? kDecayHead : kDecayToken, B, H, dk, dv, qkv_dtype, out_dtype,
                             state, state_out, out, static_cast<hipStream_t>(stream)) == hipSuccess
               ? GLA_OK
               : GLA_ERR_HIP;
}

int gla_rope(const void *q, const void *k, const int *positions, const int *sections, int axes, float base, int pairing, int inverse, int B,
             int H, int T, int d, int grid_h, int grid_w, int dtype, int layout, void *out_q, void *out_k, gla_stream_t stream) {
    if (!q || !out_q || !sections || (k == nullptr) != (out_k == nullptr)) return GLA_ERR_NULL;
    if (B <= 0 || H <= 0 || T <= 0 || d <= 0 || axes <= 0 || bad_dtype(dtype) || (layout != GLA_LAYOUT_BHTD && layout != GLA_LAYOUT_BTHD) ||
        (pairing != GLA_ROPE_ADJACENT && pairing != GLA_ROPE_HALVES) || !(base > 0.f) || isinf(base))
        return GLA_ERR_SHAPE;
    if (axes > kRopeMaxAxes || d > kRopeMaxD) return GLA_ERR_UNSUPPORTED;
    if (positions == nullptr) {          // from the grid: the token, its row and column, or its frame, row and column
        if (axes > 3) return GLA_ERR_SHAPE;
        if (axes > 1) {
            if (grid_h <= 0 || grid_w <= 0) return GLA_ERR_SHAPE;
            const long long cell = (long long)grid_h * grid_w;
            if (axes == 2 ? cell != T : T % cell != 0) return GLA_ERR_SHAPE;
        }
    }
    RopeParams p = {};
    int first = 0;
    for (int a = 0; a < axes; ++a) {
        const int w = sections[a];
        if (w < 2 || w % 2 != 0 || w > d - first) return GLA_ERR_SHAPE;
        p.first[a] = first;
        p.half[a] = w / 2;
        // One power a section: 64 of them took longer than the kernel of a few tokens.  Each product is off by 2^-63 more at most, in 64 bits of
        // mantissa: 128 pairs by 2^-56, which 2^31 / (2 pi) turns make 2^-25 of an angle (of the first pairs' a position; with a base below 1 the
        // last pairs turn faster and are off by as much more).
        const long double ratio = powl((long double)base, -2.0L / w);
        long double turns = 0.159154943091895335768883763372514362L;     // 1 / (2 pi)
        for (int i = 0; i < w / 2; ++i, turns *= ratio) {
            double head = (double)turns;
            uint64_t bits;
            memcpy(&bits, &head, sizeof bits);
            bits &= ~0xffffffffull;
            memcpy(&head, &bits, sizeof bits);
            p.turns[first / 2 + i] = head;
            p.rest[first / 2 + i] = (double)(turns - head);
        }
        first += w;
        p.pairs_end[a] = first / 2;
    }
    if (any_misaligned(q, k, (const void *)out_q, (const void *)out_k) || (reinterpret_cast<uintptr_t>(positions) & 3u) != 0) return GLA_ERR_ALIGN;
    // in place is each pair's own place: no tensor is turned into another's, nor two into one
    if (k != nullptr && (out_q == out_k || out_q == k || out_k == q)) return GLA_ERR_SHAPE;
    // 32-bit thread numbers
    if ((long long)B * T >= (1LL << 31) / d) return GLA_ERR_UNSUPPORTED;
    const size_t bytes = (size_t)B * T * H * d * size_of(dtype);
    if (overlap(out_q, bytes, q, bytes) || overlap(out_q, bytes, k, bytes) || overlap(out_k, bytes, q, bytes) || overlap(out_k, bytes, k, bytes) ||
        overlap(out_q, bytes, out_k, bytes))
        return GLA_ERR_SHAPE;
    p.x[0] = q;
    p.x[1] = k;
    p.y[0] = out_q;
    p.y[1] = out_k;
    p.positions = positions;
    p.axes = axes;
    p.pairs = first / 2;
    p.adjacent = pairing == GLA_ROPE_ADJACENT;
    p.inverse = inverse != 0;
    p.B = B;
    p.H = H;
    p.T = T;
    p.d = d;
    p.grid_h = grid_h;
    p.grid_w = grid_w;
    p.layout = layout;
    p.heads_each = 0;
    return launch_rope(p, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

static int check_norm(const void *x, const void *r_pre, const float *weight, const float *bias, float eps, int B, int H, int T, int D,
                      int dtype, int other_dtype, int layout) {
    if (!x) return GLA_ERR_NULL;
    if (B <= 0 || H <= 0 || T <= 0 || D <= 0 || bad_dtype(dtype) || bad_dtype(other_dtype) ||
        (layout != GLA_LAYOUT_BHTD && layout != GLA_LAYOUT_BTHD) || !(eps >= 0.f))
        return GLA_ERR_SHAPE;
    // 32-bit row and column numbers
    if (D > kNormMaxD || (long long)B * T >= (1LL << 31) || H > (1 << 17)) return GLA_ERR_UNSUPPORTED;
    if (any_misaligned(x, r_pre, (const void *)weight, (const void *)bias)) return GLA_ERR_ALIGN;
    return GLA_OK;
}

int gla_norm_fwd(const void *x, const float *weight, const float *bias, float eps, const void *r_pre, int B, int H, int T, int D, int x_dtype,
                 int out_dtype, int layout, void *out, gla_stream_t stream) {
    if (!x || !out) return GLA_ERR_NULL;
    const int st = check_norm(x, r_pre, weight, bias, eps, B, H, T, D, x_dtype, out_dtype, layout);
    if (st != GLA_OK) return st;
    if (out == x && x_dtype != out_dtype) return GLA_ERR_SHAPE;
    if (misaligned(out)) return GLA_ERR_ALIGN;
    const size_t elements = (size_t)B * T * H * D, bytes = elements * size_of(out_dtype), read = elements * size_of(x_dtype);
    if (overlap(out, bytes, x, read) || overlap(out, bytes, r_pre, read) || (out == r_pre && x_dtype != out_dtype)) return GLA_ERR_SHAPE;
    NormParams p = {};
    p.x = x;
    p.r_pre = r_pre;
    p.weight = weight;
    p.bias = bias;
    p.out = out;
    p.eps = eps;
    p.B = B;
    p.H = H;
    p.T = T;
    p.D = D;
    p.layout = layout;
    p.out_dtype = out_dtype;
    return launch_norm_fwd(p, x_dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

static size_t norm_bytes(int B, int H, int T, int D) {
    const int a = norm_partial_rows(B, H, T, D, GLA_LAYOUT_BHTD), b = norm_partial_rows(B, H, T, D, GLA_LAYOUT_BTHD);
    return align_up((size_t)2 * (a > b ? a : b) * H * D * sizeof(float));
}
size_t gla_norm_bwd_workspace_bytes(int B, int H, int T, int D) {
    if (B <= 0 || H <= 0 || T <= 0 || D <= 0 || D > kNormMaxD || (long long)B * T >= (1LL << 31) || H > (1 << 17)) return 0;
    return norm_bytes(B, H, T, D);
}

int gla_norm_bwd(const void *x, const void *d_out, const float *weight, const float *bias, float eps, const void *r_pre, int B, int H, int T,
                 int D, int x_dtype, int grad_dtype, int layout, void *dx, void *dr, float *dweight, float *dbias, void *workspace,
                 size_t workspace_bytes, gla_stream_t stream) {
    if (!x || !d_out || !dx || (r_pre == nullptr) != (dr == nullptr) || (dweight == nullptr) != (dbias == nullptr)) return GLA_ERR_NULL;
    const int st = check_norm(x, r_pre, weight, bias, eps, B, H, T, D, x_dtype, grad_dtype, layout);
    if (st != GLA_OK) return st;
    if (any_misaligned(d_out, (const void *)dx, (const void *)dr, (const void *)dweight, (const void *)dbias)) return GLA_ERR_ALIGN;
    if (!workspace || misaligned(workspace) || workspace_bytes < norm_bytes(B, H, T, D)) return GLA_ERR_WORKSPACE;
    NormParams p = {};
    p.x = x;
    p.d_out = d_out;
    p.r_pre = r_pre;
    p.weight = weight;
    p.bias = bias;
    p.dx = dx;
    p.dr = dr;
    p.part = dweight != nullptr ? static_cast<float *>(workspace) : nullptr;
    p.eps = eps;
    p.B = B;
    p.H = H;
    p.T = T;
    p.D = D;
    p.layout = layout;
    p.out_dtype = grad_dtype;
    p.slots = norm_slots(B, H, T, D, layout);
    return launch_norm_bwd(p, x_dtype, dweight, dbias, static_cast<hipStream_t>(stream)) == hipSuccess ? GLA_OK : GLA_ERR_HIP;
}

}  // extern "C"
