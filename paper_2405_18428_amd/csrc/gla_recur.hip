// Gated recurrence of channels: h_t = a_t h_{t-1} + u_t with a gate a in [0, 1] for every channel and step, given as its logarithm or as the
// pre-activation z of a = sigmoid(z)^(1/tau), and u_t = x_t or (1 - a_t) x_t.  Backward, from the end:
//   G_t = dO_t + a_{t+1} G_{t+1},   dx_t = G_t (or (1 - a_t) G_t),   dlog a_t = a_t (h_{t-1} - (0 or x_t)) G_t,   dz = dlog a sigmoid(-z) / tau.
//
// A lane has V neighbouring channels of one sequence, a wave 8 or 16 steps of them in registers: their decays a and inputs u from what it loads, the
// state they make of zero, and, once the state that enters them is known, the outputs.  The 8 waves of a work-group take 8 pieces in a row and
// hand each other decay and state through LDS.  Where channels alone fill the GPU a work-group walks its channels' whole sequence, else sequences are cut
// into units of 128 steps (chain_kernel): a work-group publishes its unit's decay and state, looks back over those of the units before it
// in its block of 16 units and takes the state behind the block before, and goes on to its outputs with its rows still in registers, so that every input is
// read once.  What a state is made of, and in which order, does not depend on which unit is ready first.
// The backward pass has chains from both ends, so a first pass leaves the decays, states from zero and adjoints from zero of rounds of 64 steps, a small
// kernel chains these, and a second pass forms the gradients.
//
// Looking back: what is published are words that hold their own validity (all ones: not there yet), written and read at device scope, so nothing
// has to be ordered.  Work-groups take their units in the order in which they start (a ticket), and a unit waits for earlier ones only, which
// have all started and publish before they wait: the earliest unit that waits can always go on.  A wait that runs out of looks all the same (`looks`) forms the
// state that enters its unit from the inputs, step by step: every wait ends.  (Calls in place have no inputs left for that: their waits end because earlier
// units go on.)
//
// Precision: a state's memory can be as long as 1 / (1 - a), and a rounded to 32 bits loses what it lacks of one: with one constant gate of
// 1 - 1e-4 over many steps the state would be off by 3e-4.  So decays leave a wave's steps as sums of log2 a, which are exact relative to
// themselves, and a state goes from one round or unit to the next by s + s expm1(sum) where the decay is near one.  log2(1 + e) of the
// pre-activation's gate gets back what 1 + e rounds off.  What a gate lacks of one comes from expm1 too.
//
// What bounds it: HBM, and beside it the vector units, which are busy for more than half of a forward call: two exponentials and a logarithm, at a quarter of
// the rate, are 12 of some 27 issue slots an element.  One MI355X, whose copies reach 5.17 TB/s; times stand at the kernels, a trace's
// unless it says call: under a trace kernels are longer (a training step's five add up to 191 us, the step takes 194 traced and 174 by itself).
#include "gla_recur.h"

namespace gla {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kSteps = kRecurSteps, kWaves = kRecurWaves;
constexpr float kLog2E = 1.44269504f;

// V neighbouring channels as they lie in memory
template <typename E, int V>
struct RawOf {
    static constexpr int kWords = (sizeof(E) * V + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(E) == 4) return __builtin_bit_cast(float, w[i]);
        else return __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void fill(uint32_t bits) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = sizeof(E) == 2 ? bits | bits << 16 : bits;
    }
};

template <typename E, int V>
__device__ __forceinline__ RawOf<E, V> load_raw(const char *p) {
    RawOf<E, V> r;
    if constexpr (sizeof(E) * V == 2) r.w[0] = *reinterpret_cast<const uint16_t *>(p);
    else __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(E) * V), sizeof(r));
    return r;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
// V values to element `at` behind a row that the whole wave shares (bytes of a lane's place in 32 bits)
template <int V>
__device__ __forceinline__ void store(void *base, int dtype, long long row, uint32_t at, const float (&v)[V]) {
    if (dtype == GLA_DT_BF16) {
        char *p = static_cast<char *>(base) + row * 2 + at * 2u;
        if constexpr (V == 1) {
            *reinterpret_cast<uint16_t *>(p) = (uint16_t)pack(v[0], 0.f);
        } else {
            uint32_t b[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) b[i] = pack(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(__builtin_assume_aligned(p, 2 * V), b, sizeof(b));
        }
    } else {
        char *p = static_cast<char *>(base) + row * 4 + at * 4u;
        __builtin_memcpy(__builtin_assume_aligned(p, 4 * V), v, sizeof(v));
    }
}

// 2^lg - 1, lg <= 0; a = 2^lg.  Near zero lg times the polynomial that meets (2^t - 1) / t at five Chebyshev points of [-1/2, 0]: off by 1.4e-8 of the
// result, with its roundings by 2.2 2^-24; below, a - 1 has lost two bits at most.
__device__ __forceinline__ float less_one(float lg, float a) {
    float p = fmaf(lg, 1.15543997e-3f, 9.54227503e-3f);
    p = fmaf(lg, p, 5.54907198e-2f);
    p = fmaf(lg, p, 0.240225675f);
    p = fmaf(lg, p, 0.693147172f);
    return lg > -0.5f ? lg * p : a - 1.f;
}
// 2^lg s
__device__ __forceinline__ float decayed(float lg, float s) {
    const float a = __builtin_amdgcn_exp2f(lg);
    return lg > -0.5f ? __builtin_fmaf(less_one(lg, a), s, s) : a * s;
}
struct Gate {
    float lg, a;                         // log2 of the gate, the gate
    float slope;                         // d log a / d of what is given
};
template <int KIND, bool SLOPE>
__device__ __forceinline__ Gate gate_of(float g, float inv_tau) {
    Gate r;
    if constexpr (KIND == GLA_GATE_LOG) {
        r.lg = g * kLog2E;
        r.slope = 1.f;
    } else {
        const float e = __builtin_amdgcn_exp2f(-__builtin_fabsf(g) * kLog2E), w = 1.f + e;      // e: 0 .. 1
        const float l = fmaf(e - (w - 1.f), kLog2E, __builtin_amdgcn_logf(w));                  // log2(1 + e)
        r.lg = fmaf(-l, inv_tau, __builtin_fminf(g, 0.f) * (kLog2E * inv_tau));
        if constexpr (SLOPE) {
            const float i = __builtin_amdgcn_rcpf(w) * inv_tau;
            r.slope = g > 0.f ? e * i : i;                                                      // sigmoid(-g) / tau
        }
    }
    r.a = __builtin_amdgcn_exp2f(r.lg);
    return r;
}

// Which channels a lane has.  `flat`: the columns (V channels of a sequence) of all sequences one after the other, so that a wave may hold those of
// several; else every sequence begins with a wave of its own (where 32-bit offsets would not reach the next sequence)
template <int V>
struct Place {
    long long row0;                      // uniform: of the wave's first sequence's token 0, or its last token in reversed row scans
    uint32_t at;                         // the lane's channels from there, in elements
    int b, channel;
    int n;                               // the sequence's length (0: no channels)
    int loads;                           // up to this step rows may be loaded: lanes without channels load those of the wave's first lane
    bool any;
    __device__ __forceinline__ Place(const RecurCall &c, bool flat, int group) {
        const int lane = threadIdx.x & 63, cols = c.D / V;
        int col;
        if (flat) {
            const long long id = (long long)group * 64 + lane;
            b = (int)(id / cols);
            col = (int)(id - (long long)b * cols);
            any = b < c.B;
        } else {
            const int each = (cols + 63) / 64;
            b = group / each;
            col = (group - b * each) * 64 + lane;
            any = col < cols;
        }
        const int b0 = __builtin_amdgcn_readfirstlane(b);
        if (!any) b = b0, col = 0;
        n = c.T;
        if (c.seq_lens != nullptr) n = min(max(c.seq_lens[b], 0), c.T);
        channel = col * V;
        row0 = (long long)b0 * c.T;
        at = (uint32_t)(b - b0) * (uint32_t)c.T * (uint32_t)c.D + (uint32_t)channel;
        if (c.scan_dir == GLA_SCAN_ROW_REV) {
            if (flat) at += (uint32_t)max(n - 1, 0) * (uint32_t)c.D;
            else row0 += __builtin_amdgcn_readfirstlane(max(n - 1, 0));
        }
        loads = n;
        if (!any) n = 0;
    }
    __device__ __forceinline__ long long cell(const RecurCall &c) const { return (long long)b * c.D + channel; }
};

// The rows of scan steps one after the other, uniform, in elements
struct Cursor {
    long long at;
    int left;                            // steps up to the end of a column (row scans: never)
    template <int V>
    __device__ __forceinline__ Cursor(const RecurCall &c, const Place<V> &p, int s) {
        if (c.scan_dir <= GLA_SCAN_ROW_REV) {
            at = p.row0 * c.D + (long long)s * c.step;
            left = 1 << 30;
        } else {
            const int k = c.scan_dir == GLA_SCAN_COL_FWD ? s : c.T - 1 - s;
            const int w = k / c.grid_h, r = k - w * c.grid_h;
            at = (p.row0 + (long long)r * c.grid_w + w) * c.D;
            left = c.scan_dir == GLA_SCAN_COL_FWD ? c.grid_h - 1 - r : r;
        }
    }
    __device__ __forceinline__ void next(const RecurCall &c) {
        const bool turn = left == 0;
        at += turn ? c.wrap : c.step;
        left = turn ? c.grid_h - 1 : left - 1;
    }
};

// V channels of L steps
template <typename E, int V, int L>
struct Rows {
    RawOf<E, V> r[L];
    __device__ __forceinline__ void load(int j, const void *base, long long row, uint32_t at) {
        r[j] = load_raw<E, V>(static_cast<const char *>(base) + row * (long long)sizeof(E) + at * (uint32_t)sizeof(E));
    }
    __device__ __forceinline__ void fill(int j, uint32_t bits) { r[j].fill(bits); }
};
// the bits of a gate of one: log 1, or the pre-activation +infinity
template <typename EG, int KIND>
constexpr uint32_t kOpenGate = KIND == GLA_GATE_LOG ? 0u : sizeof(EG) == 2 ? 0x7f80u : 0x7f800000u;

template <typename E>
__device__ __forceinline__ const char *row_of(const void *base, long long row) { return static_cast<const char *>(base) + row * (long long)sizeof(E); }

// x, gates and (backward) dO of L steps from s on.  Steps behind the sequence's end get zeros, and gates that let everything through
template <typename EX, typename EG, int V, int L, int KIND, bool BACK>
struct Given {
    Rows<EX, V, L> x, o;
    Rows<EG, V, L> g;
    bool whole;
    __device__ __forceinline__ void load(const RecurCall &c, const Place<V> &p, const void *d_out, int s) {
        whole = __all(s + L <= p.loads);
        Cursor k(c, p, s);
        if (whole && c.scan_dir <= GLA_SCAN_ROW_REV) {   // (a third of the scalar instructions)
            const char *px = row_of<EX>(c.x, k.at), *pg = row_of<EG>(c.gate, k.at), *po = BACK ? row_of<EX>(d_out, k.at) : nullptr;
            const long long sx = c.step * (long long)sizeof(EX), sg = c.step * (long long)sizeof(EG);
#pragma unroll
            for (int j = 0; j < L; ++j) {
                x.r[j] = load_raw<EX, V>(px + p.at * (uint32_t)sizeof(EX));
                g.r[j] = load_raw<EG, V>(pg + p.at * (uint32_t)sizeof(EG));
                if constexpr (BACK) o.r[j] = load_raw<EX, V>(po + p.at * (uint32_t)sizeof(EX));
                px += sx;
                pg += sg;
                if constexpr (BACK) po += sx;
            }
        } else if (whole) {
#pragma unroll
            for (int j = 0; j < L; ++j) {
                x.load(j, c.x, k.at, p.at);
                g.load(j, c.gate, k.at, p.at);
                if constexpr (BACK) o.load(j, d_out, k.at, p.at);
                k.next(c);
            }
        } else {
#pragma unroll
            for (int j = 0; j < L; ++j) {
                x.fill(j, 0);
                g.fill(j, kOpenGate<EG, KIND>);
                if constexpr (BACK) o.fill(j, 0);
                if (s + j < p.loads) {
                    x.load(j, c.x, k.at, p.at);
                    g.load(j, c.gate, k.at, p.at);
                    if constexpr (BACK) o.load(j, d_out, k.at, p.at);
                }
                k.next(c);
            }
        }
    }
};

// Decays and inputs of L steps
template <typename EX, typename EG, int V, int L, int KIND, bool REST>
struct Piece {
    float a[L][V], u[L][V];
    float lg[V];                         // log2 of all gates
    template <bool BACK>
    __device__ __forceinline__ Piece(const Given<EX, EG, V, L, KIND, BACK> &in, float inv_tau) {
#pragma unroll
        for (int i = 0; i < V; ++i) lg[i] = 0.f;
#pragma unroll
        for (int j = 0; j < L; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const Gate t = gate_of<KIND, false>(in.g.r[j][i], inv_tau);
                const float v = in.x.r[j][i];
                a[j][i] = t.a;
                u[j][i] = REST ? -less_one(t.lg, t.a) * v : v;
                lg[i] += t.lg;
            }
    }
    // the state they make of zero
    __device__ __forceinline__ float from_zero(int i) const {
        float h = 0.f;
#pragma unroll
        for (int j = 0; j < L; ++j) h = __builtin_fmaf(a[j][i], h, u[j][i]);
        return h;
    }
};

template <int V>
__device__ __forceinline__ void load_state(const float *p, long long at, float (&v)[V]) {
    __builtin_memcpy(v, __builtin_assume_aligned(p + at, 4 * V), sizeof(v));
}
template <int V>
__device__ __forceinline__ void store_state(float *p, long long at, const float (&v)[V]) {
    __builtin_memcpy(__builtin_assume_aligned(p + at, 4 * V), v, sizeof(v));
}

// Backward, first pass: a wave takes one unit of 64 V channels, 8 steps at a time with the next 8 on their way.  Reads x, gates and dO: 4 x 4096 x 2048,
// bf16, 43 us, 4.7 TB/s, the vector units busy for 83 % of it.
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(256) void units_kernel(const RecurCall c, const void *d_out, const RecurUnits u, bool flat, int groups) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const long long task = (long long)blockIdx.x * 4 + wave;
    if (task >= (long long)groups * c.nunits) return;
    // neighbouring waves: neighbouring channels, whose rows lie beside each other
    const int unit = (int)(task / groups), group = (int)(task - (long long)unit * groups);
    const Place<V> p(c, flat, group);
    const int begin = unit * c.unit, end = min(begin + c.unit, c.T);
    float lg[V] = {}, h[V] = {}, adj[V] = {};
    Given<EX, EG, V, kSteps, KIND, true> in;
    in.load(c, p, d_out, begin);         // (a unit ends at a multiple of 8 steps or at T)
    for (int s = begin; s < end; s += kSteps) {
        const Piece<EX, EG, V, kSteps, KIND, REST> q(in, c.inv_tau);
        float dd[kSteps][V];
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) dd[j][i] = in.o.r[j][i];
        if (s + kSteps < end) in.load(c, p, d_out, s + kSteps);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[i] = decayed(q.lg[i], h[i]) + q.from_zero(i);
            float b = 0.f;
#pragma unroll
            for (int j = kSteps - 1; j >= 0; --j) b = q.a[j][i] * (dd[j][i] + b);
            adj[i] += __builtin_amdgcn_exp2f(lg[i]) * b;
            lg[i] += q.lg[i];
        }
    }
    if (!p.any) return;
    const long long at = ((long long)p.b * c.nunits + unit) * c.D + p.channel;
    store_state<V>(u.decay, at, lg);
    store_state<V>(u.state, at, h);
    store_state<V>(u.adjoint, at, adj);
}

// The same with a work-group for each unit, 8 steps a wave, where there are few units and a wave's 64 steps one after the other would be the time: 4 x 1024 x 384
// fp32 6.4 us
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kWaves) void units_apart_kernel(const RecurCall c, const void *d_out, const RecurUnits u, bool flat, int groups) {
    __shared__ float lds_lg[kWaves][64][V], lds_h[kWaves][64][V], lds_o[kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int unit = blockIdx.x / (unsigned)groups, group = blockIdx.x - (unsigned)unit * (unsigned)groups;
    const Place<V> p(c, flat, group);
    Given<EX, EG, V, kSteps, KIND, true> in;
    in.load(c, p, d_out, unit * c.unit + wave * kSteps);
    const Piece<EX, EG, V, kSteps, KIND, REST> q(in, c.inv_tau);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float b = 0.f;
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j) b = q.a[j][i] * (in.o.r[j][i] + b);
        lds_lg[wave][lane][i] = q.lg[i];
        lds_h[wave][lane][i] = q.from_zero(i);
        lds_o[wave][lane][i] = b;
    }
    __syncthreads();
    if (wave > 0 || !p.any) return;
    float lg[V] = {}, h[V] = {}, adj[V] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = lds_lg[w][lane][i];
            h[i] = decayed(d, h[i]) + lds_h[w][lane][i];
            adj[i] = fmaf(__builtin_amdgcn_exp2f(lg[i]), lds_o[w][lane][i], adj[i]);
            lg[i] += d;
        }
    const long long at = ((long long)p.b * c.nunits + unit) * c.D + p.channel;
    store_state<V>(u.decay, at, lg);
    store_state<V>(u.state, at, h);
    store_state<V>(u.adjoint, at, adj);
}

// Chains the units of 64 channels: 16 waves take as many runs of units, compose each, chain the runs through LDS and walk their runs again, where
// what enters a unit takes the place of what it makes of zero.  Bound by latency: 64 units of 4 x 2048 channels, in both directions, 6.0 us.
constexpr int kCarryWaves = 16;
__global__ __launch_bounds__(64 * kCarryWaves) void carry_kernel(const RecurCall c, const RecurUnits u, const float *first, const float *last, float *d_first) {
    __shared__ float run_lg[kCarryWaves][64], run_s[kCarryWaves][64];
    constexpr int kAtOnce = 8;           // units whose loads are under way together
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = (c.D + 63) / 64;
    const int b = blockIdx.x / blocks, ch = (blockIdx.x - b * blocks) * 64 + lane;
    const bool any = ch < c.D;
    const int each = (c.nunits + kCarryWaves - 1) / kCarryWaves;
    const bool back = blockIdx.y == 1;
    float *const own = back ? u.adjoint : u.state;
    const int from = min(wave * each, c.nunits), to = min(from + each, c.nunits);
    const long long base = (long long)b * c.nunits * c.D + (any ? ch : 0);
    // the k-th unit of the chain
    auto at = [&](int k) { return base + (long long)(back ? c.nunits - 1 - k : k) * c.D; };
    auto walk = [&](float &s, auto &&each_unit) {
        for (int k = from; k < to; k += kAtOnce) {
            float d[kAtOnce], v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const long long i = at(min(k + j, to - 1));
                d[j] = u.decay[i];
                v[j] = own[i];
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (k + j < to) each_unit(k + j, d[j], v[j], s);
        }
    };
    float lg = 0.f, s = 0.f;
    walk(s, [&](int, float d, float v, float &t) {
        t = decayed(d, t) + v;
        lg += d;
    });
    run_lg[wave][lane] = lg;
    run_s[wave][lane] = s;
    __syncthreads();
    const float *enter = back ? last : first;
    s = enter != nullptr && any ? enter[(long long)b * c.D + ch] : 0.f;
    for (int w = 0; w < wave; ++w) s = decayed(run_lg[w][lane], s) + run_s[w][lane];
    walk(s, [&](int k, float d, float v, float &t) {
        if (any) own[at(k)] = t;
        t = decayed(d, t) + v;
    });
    if (back && any && d_first != nullptr && from < to && to == c.nunits) d_first[(long long)b * c.D + ch] = s;
}

// The outputs of a piece from the state that enters it
template <typename EX, typename EG, int V, int L, int KIND, bool REST>
__device__ __forceinline__ void put_outputs(const RecurCall &c, const Place<V> &p, const Piece<EX, EG, V, L, KIND, REST> &q, float (&h)[V], void *out, int dtype, int s,
                                            bool whole) {
    Cursor k(c, p, s);
    if (whole && c.scan_dir <= GLA_SCAN_ROW_REV && dtype == GLA_DT_BF16) {
        char *row = static_cast<char *>(out) + k.at * 2;
#pragma unroll
        for (int j = 0; j < L; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = __builtin_fmaf(q.a[j][i], h[i], q.u[j][i]);
            store<V>(row, GLA_DT_BF16, 0, p.at, h);
            row += c.step * 2;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < L; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = __builtin_fmaf(q.a[j][i], h[i], q.u[j][i]);
        if (whole || s + j < p.n) store<V>(out, dtype, k.at, p.at, h);
        k.next(c);
    }
}

// Forward pass with a sequence to itself: a work-group walks 64 V channels in rounds, 8 steps a wave, with the next round on its way.  Bound by HBM where
// work-groups fill the GPU (16 x 4096 x 2048, bf16: a call 160 us, 5.0 TB/s), by a round's loads, exchange and stores one after the other elsewhere (2.4 us for 64
// steps of 64 groups).
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kWaves) void walk_kernel(const RecurCall c, const float *first, void *out, int out_dtype, float *final_state, bool flat) {
    __shared__ float lds_lg[2][kWaves][64][V], lds_a[2][kWaves][64][V], lds_h[2][kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    const Place<V> p(c, flat, blockIdx.x);
    const int round = kSteps * waves;
    float carry[V] = {};
    if (first != nullptr && p.any) load_state<V>(first, p.cell(c), carry);
    Given<EX, EG, V, kSteps, KIND, false> in;
    in.load(c, p, nullptr, wave * kSteps);
    asm volatile("" : "+v"(carry[0]), "+v"(carry[V - 1]));      // (read before any wave may write a final state over it)
    int buf = 0;
    for (int s0 = 0; s0 < c.T; s0 += round, buf ^= 1) {
        const int s = s0 + wave * kSteps;
        const Piece<EX, EG, V, kSteps, KIND, REST> q(in, c.inv_tau);
        const bool whole = __all(s + kSteps <= p.n);
        if (s0 + round < c.T) in.load(c, p, nullptr, s + round);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            lds_lg[buf][wave][lane][i] = q.lg[i];
            lds_a[buf][wave][lane][i] = __builtin_amdgcn_exp2f(q.lg[i]);
            lds_h[buf][wave][lane][i] = q.from_zero(i);
        }
        __syncthreads();                 // (the other buffer's readers are past the next barrier before it is written again)
        float z[V] = {}, lg[V] = {}, mine[V] = {};
        for (int w = 0; w < waves; ++w) {
            if (w == wave) {
#pragma unroll
                for (int i = 0; i < V; ++i) mine[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(lg[i]), carry[i], z[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                z[i] = __builtin_fmaf(lds_a[buf][w][lane][i], z[i], lds_h[buf][w][lane][i]);
                lg[i] += lds_lg[buf][w][lane][i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) carry[i] = decayed(lg[i], carry[i]) + z[i];
        put_outputs(c, p, q, mine, out, out_dtype, s, whole);
    }
    if (final_state != nullptr && wave == 0 && p.any) store_state<V>(final_state, p.cell(c), carry);
}

// Words that units publish: all ones are not there yet (a NaN that would look so gets other digits)
constexpr int kChainWaves = kRecurChainWaves, kChainSteps = kRecurChain / kChainWaves;
typedef unsigned long long word_t;
__device__ __forceinline__ uint32_t bits_of(float x) { return x != x ? 0x7fc00000u : __builtin_bit_cast(uint32_t, x); }
__device__ __forceinline__ void publish(word_t *p, float lg, float h) {
    __hip_atomic_store(p, (word_t)bits_of(lg) << 32 | bits_of(h), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish(uint32_t *p, float s) { __hip_atomic_store(p, bits_of(s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename W>
__device__ __forceinline__ W published(const W *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// All words to "not there", the ticket to zero
__global__ __launch_bounds__(256) void clear_kernel(uint32_t *words, long long count, uint32_t *ticket) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    if (at < count) *reinterpret_cast<u32x4 *>(words + at) = u32x4{~0u, ~0u, ~0u, ~0u};
    if (at == 0) *ticket = 0;
}

// Forward pass in units of 128 steps, 16 a wave.  Decays and inputs of the wave's 16 steps stay in registers, 64 with two channels a lane, while the
// look-back waits, so two work-groups fit a compute unit; their loads, wait and stores overlap each other's.  65536 x 2048, bf16: a call 178 us, 4.5 TB/s
// (the kernel 189 in a trace); 4 x 4096 x 2048 with u = (1 - a) x a call 50 us (the kernel 59); 8 sequences of 1 to 2047 steps,
// 130 MB moved, a call 45 us, some 20 of them the first loads and the last stores.  In traces of 65536 x 2048 units of 64 steps (8 a wave) took 393 us, of 256 (16
// waves) 396, work-groups of 4 waves 236.  One ticket for all groups is ahead of one for each, 188 us and 215: neighbouring groups' units, whose rows lie beside each other, then run together.
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kChainWaves, 4) void chain_kernel(const RecurCall c, const RecurChain ch, const float *first, void *out, int out_dtype, float *final_state,
                                                            bool flat, int groups) {
    // of a wave's steps, and of the units that it looks back at: log2 of their decay, the state they make of zero
    __shared__ __attribute__((aligned(16))) float parts[kChainWaves][64][2 * V], fars[kChainWaves][64][2 * V];
    __shared__ float lds_s[64][V];
    __shared__ bool outs[kChainWaves];
    __shared__ uint32_t lds_ticket;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (threadIdx.x == 0) lds_ticket = __hip_atomic_fetch_add(ch.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t task = __builtin_amdgcn_readfirstlane((int)lds_ticket);
    const int unit = (int)(task / (uint32_t)groups), group = (int)(task - (uint32_t)unit * (uint32_t)groups);
    const Place<V> p(c, flat, group);
    const int begin = unit * kRecurChain, s = begin + wave * kChainSteps;
    if (unit > 0 && __all(begin >= p.n)) return;         // behind all its sequences' ends, as are the units after it
    // of unit n: its decay and state from zero; of block n of units: the state behind it
    auto local = [&](int n, int i) { return ch.local + (((long long)n * groups + group) * V + i) * 64 + lane; };
    auto after = [&](int n, int i) { return ch.after + (((long long)n * groups + group) * V + i) * 64 + lane; };
    Given<EX, EG, V, kChainSteps, KIND, false> in;
    in.load(c, p, nullptr, s);
    float enter[V] = {};
    if (wave == 0 && unit < kRecurBlock && first != nullptr && p.any) load_state<V>(first, p.cell(c), enter);
    const Piece<EX, EG, V, kChainSteps, KIND, REST> q(in, c.inv_tau);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        parts[wave][lane][i] = q.lg[i];
        parts[wave][lane][V + i] = q.from_zero(i);
    }
    __syncthreads();
    // of the waves before this one (the first wave: of the whole unit)
    float z[V] = {}, lg[V] = {};
    const int before = wave == 0 ? kChainWaves : wave;
#pragma unroll
    for (int w = 0; w < kChainWaves; ++w) {
        if (w >= before) continue;
        float part[2 * V];
        __builtin_memcpy(part, &parts[w][lane][0], sizeof(part));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            z[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(part[i]), z[i], part[V + i]);
            lg[i] += part[i];
        }
    }
    const int block = unit / kRecurBlock, in_block = unit - block * kRecurBlock;
    const bool last = unit == c.nunits - 1;
    if (wave == 0 && !last && in_block < kRecurBlock - 1) {
        // (what is published also says that this unit has read what enters it, which a final state may be written over)
        asm volatile("" ::"v"(enter[0]), "v"(enter[V - 1]));
#pragma unroll
        for (int i = 0; i < V; ++i) publish(local(unit, i), lg[i], z[i]);
    }
    // Looking back: each wave at kRecurBlock / kChainWaves units of the block, the first also for the state behind the block before
    constexpr int kEach = kRecurBlock / kChainWaves;
    const int begins = block * kRecurBlock + wave * kEach, count = min(max(unit - begins, 0), kEach);
    float far_lg[V] = {}, far_z[V] = {};
    bool ran_out = false;
    if (count > 0) {
        word_t part[kEach][V] = {};
        bool there = false;
        for (RecurLooks looks = {ch.looks, 0}; !there && looks.another();) {
            there = true;
#pragma unroll
            for (int k = 0; k < kEach; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) part[k][i] = published(local(begins + min(k, count - 1), i));
#pragma unroll
            for (int k = 0; k < kEach; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) there = there && part[k][i] != ~0ull;
            there = __all(there);
        }
        ran_out = !there;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (k < count) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = __builtin_bit_cast(float, (uint32_t)(part[k][i] >> 32));
                    far_z[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(d), far_z[i], __builtin_bit_cast(float, (uint32_t)part[k][i]));
                    far_lg[i] += d;
                }
            }
    }
    if (wave == 0 && block > 0) {
        bool there = false;
        for (RecurLooks looks = {ch.looks, 0}; !there && !ran_out && looks.another();) {
            there = true;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t w = published(after(block - 1, i));
                there = there && w != ~0u;
                enter[i] = __builtin_bit_cast(float, w);
            }
            there = __all(there);
        }
        ran_out = !there;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        fars[wave][lane][i] = far_lg[i];
        fars[wave][lane][V + i] = far_z[i];
        if (wave == 0) lds_s[lane][i] = enter[i];
    }
    if (lane == 0) outs[wave] = ran_out;
    __syncthreads();
    // each wave's units through the decay behind them, and the state through all of it
#pragma unroll
    for (int i = 0; i < V; ++i) far_lg[i] = far_z[i] = 0.f;
    ran_out = false;
#pragma unroll
    for (int w = kChainWaves - 1; w >= 0; --w) {
        ran_out = ran_out || outs[w];
        float part[2 * V];
        __builtin_memcpy(part, &fars[w][lane][0], sizeof(part));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            far_z[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(far_lg[i]), part[V + i], far_z[i]);
            far_lg[i] += part[i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) enter[i] = decayed(far_lg[i], lds_s[lane][i]) + far_z[i];
    if (__builtin_amdgcn_readfirstlane(ran_out)) {       // from the inputs, step by step
#pragma unroll
        for (int i = 0; i < V; ++i) enter[i] = 0.f;
        if (first != nullptr && p.any) load_state<V>(first, p.cell(c), enter);
        for (int t = 0; t < begin; ++t) {
            Given<EX, EG, V, 1, KIND, false> again;
            again.load(c, p, nullptr, t);
            const Piece<EX, EG, V, 1, KIND, REST> r(again, c.inv_tau);
#pragma unroll
            for (int i = 0; i < V; ++i) enter[i] = decayed(r.lg[i], enter[i]) + r.u[0][i];
        }
    }
    if (wave == 0) {
        const bool ends = p.n <= begin + kRecurChain && (p.n > begin || unit == 0);      // a sequence's last unit
        float leave[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            leave[i] = decayed(lg[i], enter[i]) + z[i];
            if (!last && in_block == kRecurBlock - 1) publish(after(block, i), leave[i]);
        }
        if (ends && final_state != nullptr && p.any) store_state<V>(final_state, p.cell(c), leave);
    }
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) enter[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(lg[i]), enter[i], z[i]);
    }
    put_outputs(c, p, q, enter, out, out_dtype, s, __all(s + kChainSteps <= p.n));
}

// Gradients of one round of 64 V channels: states from the front, adjoints from behind, 8 steps a wave.  Bound by HBM and the vector units (72 % busy):
// 4 x 4096 x 2048, bf16, 335 MB, 78 us, 4.3 TB/s.  118 registers let two work-groups share a compute unit; the compiler's own order takes 163
// (110 us), and held to 128 without the fences below it spills (160 us).
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kWaves, 4) void back_kernel(const RecurCall c, const void *d_out, const RecurUnits u, const float *first, const float *last,
                                                           void *dx, void *dgate, int grad_dtype, float *d_first, bool flat, int groups) {
    __shared__ float lds_lg[kWaves][64][V], lds_h[kWaves][64][V], lds_o[kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    const int unit = blockIdx.x / (unsigned)groups, group = blockIdx.x - (unsigned)unit * (unsigned)groups;
    const Place<V> p(c, flat, group);
    const int s = unit * kRecurRound + wave * kSteps;
    Given<EX, EG, V, kSteps, KIND, true> in;
    in.load(c, p, d_out, s);
    float h[V] = {}, adj[V] = {};
    if (p.any) {
        const long long at = ((long long)p.b * c.nunits + unit) * c.D + p.channel;
        if (c.nunits > 1) {
            load_state<V>(u.state, at, h);
            load_state<V>(u.adjoint, at, adj);
        } else {
            if (first != nullptr) load_state<V>(first, p.cell(c), h);
            if (last != nullptr) load_state<V>(last, p.cell(c), adj);
        }
    }
    // of each step: the gate, what it lacks of one, the gate times its slope, then times what the adjoint meets there
    float a[kSteps][V], rest[REST ? kSteps : 1][V], b[kSteps][V], lg[V] = {}, z[V] = {};
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Gate gt = gate_of<KIND, true>(in.g.r[j][i], c.inv_tau);
            const float x = in.x.r[j][i];
            a[j][i] = gt.a;
            b[j][i] = KIND == GLA_GATE_PRE ? gt.a * gt.slope : gt.a;
            asm volatile("" : "+v"(b[j][i]));            // (formed here: left for later its parts take twice the registers)
            if constexpr (REST) rest[j][i] = -less_one(gt.lg, gt.a);
            lg[i] += gt.lg;
            z[i] = REST ? fmaf(a[j][i], z[i], rest[j][i] * x) : fmaf(a[j][i], z[i], x);
        }
        // (all steps at once take more registers than there are)
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        lds_lg[wave][lane][i] = lg[i];
        lds_h[wave][lane][i] = z[i];
        float r = 0.f;
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j) r = a[j][i] * (in.o.r[j][i] + r);
        lds_o[wave][lane][i] = r;
        lg[i] = z[i] = 0.f;
    }
    __syncthreads();
    // the other waves' states and adjoints through the decay between, what enters the round through all of it
    for (int w = wave - 1; w >= 0; --w)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            z[i] = fmaf(__builtin_amdgcn_exp2f(lg[i]), lds_h[w][lane][i], z[i]);
            lg[i] += lds_lg[w][lane][i];
        }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        h[i] = fmaf(__builtin_amdgcn_exp2f(lg[i]), h[i], z[i]);
        z[i] = lg[i] = 0.f;
    }
    for (int w = wave + 1; w < waves; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            z[i] = fmaf(__builtin_amdgcn_exp2f(lg[i]), lds_o[w][lane][i], z[i]);
            lg[i] += lds_lg[w][lane][i];
        }
#pragma unroll
    for (int i = 0; i < V; ++i) adj[i] = fmaf(__builtin_amdgcn_exp2f(lg[i]), adj[i], z[i]);
    Cursor k(c, p, s);
    long long rows[kSteps];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        rows[j] = k.at;
        k.next(c);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float x = in.x.r[j][i];
            b[j][i] *= REST ? h[i] - x : h[i];           // (the state before the step)
            h[i] = REST ? fmaf(a[j][i], h[i], rest[j][i] * x) : fmaf(a[j][i], h[i], x);
        }
    }
    const bool whole = __all(s + kSteps <= p.n);
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
        float gx[V], gg[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float G = in.o.r[j][i] + adj[i];
            gx[i] = REST ? rest[j][i] * G : G;
            gg[i] = b[j][i] * G;
            adj[i] = a[j][i] * G;
        }
        if (whole || s + j < p.n) {
            store<V>(dx, grad_dtype, rows[j], p.at, gx);
            store<V>(dgate, grad_dtype, rows[j], p.at, gg);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!whole && p.any && c.seq_lens != nullptr) {      // rows behind a sequence's end are cleared: step t stands for token t there, in both directions
        const float zero[V] = {};
#pragma unroll 1
        for (int t = max(s, p.n); t < min(s + kSteps, c.T); ++t) {
            const long long row = ((long long)p.b * c.T + t) * c.D;
            store<V>(dx, grad_dtype, row, (uint32_t)p.channel, zero);
            store<V>(dgate, grad_dtype, row, (uint32_t)p.channel, zero);
        }
    }
    if (unit == 0 && c.nunits == 1 && wave == 0 && d_first != nullptr && p.any) store_state<V>(d_first, p.cell(c), adj);
}

// One step of every sequence: a thread has V channels.  2.5 us for 2048 channels, a launch's own time.
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64) void step_kernel(const RecurCall c, const float *state, float *state_out, void *out, int out_dtype) {
    const long long at = ((long long)blockIdx.x * 64 + threadIdx.x) * V;
    if (at >= (long long)c.B * c.D) return;
    const RawOf<EX, V> x = load_raw<EX, V>(static_cast<const char *>(c.x) + at * (long long)sizeof(EX));
    const RawOf<EG, V> g = load_raw<EG, V>(static_cast<const char *>(c.gate) + at * (long long)sizeof(EG));
    float h[V];
    load_state<V>(state, at, h);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const Gate t = gate_of<KIND, false>(g[i], c.inv_tau);
        const float v = x[i], rest = -less_one(t.lg, t.a);
        const float near = t.a > 0.7f ? __builtin_fmaf(-rest, h[i], h[i]) : t.a * h[i];
        h[i] = near + (REST ? rest * v : v);
    }
    store_state<V>(state_out, at, h);
    store<V>(out, out_dtype, at, 0, h);
}

// Element types, gate, input and vector width of a call -> a kernel's instance: two channels a lane where the rows allow it
template <typename F>
hipError_t instance(const RecurCall &c, bool two, F &&run) {
    auto wide = [&](auto x, auto g, auto kind, auto rest) {
        return two ? run(x, g, kind, rest, std::integral_constant<int, 2>{}) : run(x, g, kind, rest, std::integral_constant<int, 1>{});
    };
    auto with = [&](auto x, auto g, auto kind) { return c.rest ? wide(x, g, kind, std::true_type{}) : wide(x, g, kind, std::false_type{}); };
    using Log = std::integral_constant<int, GLA_GATE_LOG>;
    using Pre = std::integral_constant<int, GLA_GATE_PRE>;
    if (c.kind == GLA_GATE_LOG) return c.dtype == GLA_DT_BF16 ? with(uint16_t{}, float{}, Log{}) : with(float{}, float{}, Log{});
    return c.dtype == GLA_DT_BF16 ? with(uint16_t{}, uint16_t{}, Pre{}) : with(float{}, float{}, Pre{});
}

// Whether a wave's columns may be those of several sequences, and the groups of 64 columns
struct Groups {
    bool flat;
    int count;                           // (of calls within the limits)
};
constexpr int width(const RecurCall &c) { return c.D % 2 == 0 ? 2 : 1; }
bool is_flat(const RecurCall &c, int V) {
    const long long cols = c.D / V, spanned = 64 / cols + 2;                       // sequences that a wave can touch
    // (elements up to the last of them in 32 bits as bytes)
    return cols % 64 != 0 && spanned * c.T < (1LL << 30) / c.D;
}
long long count_of(const RecurCall &c, int V) {
    const long long cols = c.D / V;
    return is_flat(c, V) ? (c.B * cols + 63) / 64 : c.B * ((cols + 63) / 64);
}
Groups groups_of(const RecurCall &c, int V) { return {is_flat(c, V), (int)count_of(c, V)}; }

}  // namespace

// Below so many units each gets a work-group, not a wave (backward calls: 192 units 18 us instead of 26, 1152 47 instead of 52, 2048 66 instead of 65)
constexpr long long kFewUnits = 2048;
hipError_t launch_recur_units(const RecurCall &c, const void *d_out, const RecurUnits &u, hipStream_t stream) {
    return instance(c, width(c) == 2, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        const long long units = (long long)n.count * c.nunits;
        if (units < kFewUnits)
            hipLaunchKernelGGL((units_apart_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)units), dim3(64 * kWaves), 0, stream, c, d_out, u,
                               n.flat, n.count);
        else
            hipLaunchKernelGGL((units_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, stream, c, d_out, u,
                               n.flat, n.count);
        return hipGetLastError();
    });
}

hipError_t launch_recur_carry(const RecurCall &c, const RecurUnits &u, const float *first, const float *last, float *d_first, hipStream_t stream) {
    hipLaunchKernelGGL(carry_kernel, dim3((unsigned)((c.D + 63) / 64) * (unsigned)c.B, 2), dim3(64 * kCarryWaves), 0, stream, c, u, first, last, d_first);
    return hipGetLastError();
}

static unsigned waves_for(int steps) {
    const int w = (steps + kSteps - 1) / kSteps;
    return 64u * (unsigned)(w < kWaves ? w : kWaves);
}

hipError_t launch_recur_walk(const RecurCall &c, const float *first, void *out, int out_dtype, float *final_state, hipStream_t stream) {
    return instance(c, width(c) == 2, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        hipLaunchKernelGGL((walk_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)n.count), dim3(waves_for(c.T)), 0, stream, c, first, out,
                           out_dtype, final_state, n.flat);
        return hipGetLastError();
    });
}

long long recur_groups(const RecurCall &c) { return count_of(c, width(c)); }
long long recur_chain_columns(const RecurCall &c) { return recur_groups(c) * width(c) * 64; }

hipError_t launch_recur_chain(const RecurCall &c, const RecurChain &ch, const float *first, void *out, int out_dtype, float *final_state, hipStream_t stream) {
    const long long words = recur_chain_columns(c) * recur_chain_words(c);
    hipLaunchKernelGGL(clear_kernel, dim3((unsigned)((words + 1023) / 1024)), dim3(256), 0, stream, reinterpret_cast<uint32_t *>(ch.local), words, ch.ticket);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return instance(c, width(c) == 2, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        hipLaunchKernelGGL((chain_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((long long)n.count * c.nunits)), dim3(64 * kChainWaves), 0, stream,
                           c, ch, first, out, out_dtype, final_state, n.flat, n.count);
        return hipGetLastError();
    });
}

hipError_t launch_recur_back(const RecurCall &c, const void *d_out, const RecurUnits &u, const float *first, const float *last, void *dx,
                             void *dgate, int grad_dtype, float *d_first, hipStream_t stream) {
    return instance(c, width(c) == 2, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        hipLaunchKernelGGL((back_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((long long)n.count * c.nunits)),
                           dim3(waves_for(c.T)), 0, stream, c, d_out, u, first, last, dx, dgate, grad_dtype, d_first, n.flat, n.count);
        return hipGetLastError();
    });
}

hipError_t launch_recur_step(const RecurCall &c, const float *state, float *state_out, void *out, int out_dtype, hipStream_t stream) {
    // (rows of single tokens are often slices of something larger)
    const uintptr_t all = reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(c.x) | reinterpret_cast<uintptr_t>(c.gate);
    return instance(c, width(c) == 2 && all % 8 == 0, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const long long lanes = (long long)c.B * c.D / V;
        hipLaunchKernelGGL((step_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((lanes + 63) / 64)), dim3(64), 0, stream, c,
                           state, state_out, out, out_dtype);
        return hipGetLastError();
    });
}

}  // namespace gla
