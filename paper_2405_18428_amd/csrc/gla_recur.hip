// Gated recurrence of channels: h_t = a_t h_{t-1} + u_t with a gate a in [0, 1] for every channel and step, given as its logarithm or as the
// pre-activation z of a = sigmoid(z)^(1/tau), and u_t = x_t or (1 - a_t) x_t.  Backward, from the end:
//   G_t = dO_t + a_{t+1} G_{t+1},   dx_t = G_t (or (1 - a_t) G_t),   dlog a_t = a_t (h_{t-1} - (0 or x_t)) G_t,   dz = dlog a sigmoid(-z) / tau.
//
// A lane has V neighbouring channels of one sequence, a wave 8 steps of them in registers: their decays a and inputs u from what it loads, the
// state they make of zero, and, once the state that enters them is known, the outputs.  The 8 waves of a work-group take 8 pieces in a row
// (a round of 64 steps) and hand each other decay and state through LDS.  Where channels alone leave the GPU idle, the sequence is cut into
// units: a pass over x and the gates leaves each unit's decay and state, a small kernel chains these, and the outputs come from a second pass.
// The backward pass has both chains at once: its units are rounds, whose states from zero and adjoints from zero come from one reading.
//
// Precision: a state's memory can be as long as 1 / (1 - a), and a rounded to 32 bits loses what it lacks of one: with one constant gate of
// 1 - 1e-4 over many steps the state would be off by 3e-4.  So decays leave a wave's 8 steps as sums of log2 a, which are exact relative to
// themselves, and a state goes from one round to the next by s + s expm1(sum) where the decay is near one.  log(1 + e) of the pre-activation's
// gate is 2 atanh(e / (2 + e)), a series that is as exact for small e as for e = 1.  What a gate lacks of one comes from expm1 too.
#include "gla_recur.h"

namespace gla {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kSteps = kRecurSteps, kWaves = kRecurWaves;
constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147181f;

template <typename E, int V> struct RawOf { E e[V]; };

template <typename E, int V>
__device__ __forceinline__ RawOf<E, V> load_raw(const char *p) {
    RawOf<E, V> r;
    __builtin_memcpy(&r, __builtin_assume_aligned(p, sizeof(E) * V), sizeof(r));
    return r;
}
__device__ __forceinline__ float to_float(float e) { return e; }
__device__ __forceinline__ float to_float(uint16_t e) { return __builtin_bit_cast(float, (uint32_t)e << 16); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
// V values to element `at` of a tensor of this type
template <int V>
__device__ __forceinline__ void store(void *base, int dtype, long long row, uint32_t at, const float (&v)[V]) {
    if (dtype == GLA_DT_BF16) {
        uint16_t *p = static_cast<uint16_t *>(base) + row + at;
        if constexpr (V == 1) {
            *p = (uint16_t)pack(v[0], 0.f);
        } else {
            uint32_t b[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) b[i] = pack(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(__builtin_assume_aligned(p, 2 * V), b, sizeof(b));
        }
    } else {
        float *p = static_cast<float *>(base) + row + at;
        __builtin_memcpy(__builtin_assume_aligned(p, 4 * V), v, sizeof(v));
    }
}

// exp(y) - 1, y <= 0 (natural units); a = exp(y)
__device__ __forceinline__ float less_one(float y, float a) {
    float p = 1.f + y * (1.f / 7.f);
    p = 1.f + y * (1.f / 6.f) * p;
    p = 1.f + y * (1.f / 5.f) * p;
    p = 1.f + y * (1.f / 4.f) * p;
    p = 1.f + y * (1.f / 3.f) * p;
    p = 1.f + y * (1.f / 2.f) * p;
    return y > -0.35f ? y * p : a - 1.f;     // (the next term of the series is 2e-8 of the result)
}
// 2^lg s
__device__ __forceinline__ float decayed(float lg, float s) {
    const float a = __builtin_amdgcn_exp2f(lg), y = lg * kLn2;
    return y > -0.35f ? __builtin_fmaf(less_one(y, a), s, s) : a * s;
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
        const float e = __builtin_amdgcn_exp2f(-__builtin_fabsf(g) * kLog2E);          // 0 .. 1
        const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;                // 0 .. 1/3
        float p = q * (1.f / 13.f) + 1.f / 11.f;
        p = p * q + 1.f / 9.f;
        p = p * q + 1.f / 7.f;
        p = p * q + 1.f / 5.f;
        p = p * q + 1.f / 3.f;
        p = p * q + 1.f;                                                              // the next term is 1.4e-8
        r.lg = (__builtin_fminf(g, 0.f) - 2.f * s * p) * (kLog2E * inv_tau);
        if constexpr (SLOPE) {
            const float i = __builtin_amdgcn_rcpf(1.f + e) * inv_tau;
            r.slope = g > 0.f ? e * i : i;                                            // sigmoid(-g) / tau
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
    // the row of a scan step, uniform, in elements
    __device__ __forceinline__ long long row(const RecurCall &c, int s) const {
        long long t;
        if (c.scan_dir <= GLA_SCAN_ROW_REV) {
            t = c.scan_dir == GLA_SCAN_ROW_FWD ? s : -s;
        } else {
            const int k = c.scan_dir == GLA_SCAN_COL_FWD ? s : c.T - 1 - s;
            const int w = k / c.grid_h;
            t = (long long)(k - w * c.grid_h) * c.grid_w + w;
        }
        return (row0 + t) * c.D;
    }
};

// V channels of the steps s0 .. s0 + 7.  Steps behind the sequence's end (`loads`) get `other`: zeros, and gates that let everything through
template <typename E, int V>
struct Rows {
    RawOf<E, V> r[kSteps];
    __device__ __forceinline__ void load(const void *base, const RecurCall &c, const Place<V> &p, int s0, bool whole, E other) {
        const char *x = static_cast<const char *>(base);
        const uint32_t at = p.at * (uint32_t)sizeof(E);
        if (whole) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j) r[j] = load_raw<E, V>(x + p.row(c, s0 + j) * (long long)sizeof(E) + at);
        } else {
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
#pragma unroll
                for (int i = 0; i < V; ++i) r[j].e[i] = other;
                if (s0 + j < p.loads) r[j] = load_raw<E, V>(x + p.row(c, s0 + j) * (long long)sizeof(E) + at);
            }
        }
    }
};
// a gate of one: log 1, or the pre-activation +infinity
template <typename EG, int KIND>
__device__ __forceinline__ EG open_gate() {
    if constexpr (KIND == GLA_GATE_LOG) return (EG)0;
    else if constexpr (sizeof(EG) == 2) return (EG)0x7f80;
    else return __builtin_inff();
}

// Decays and inputs of 8 steps
template <typename EX, typename EG, int V, int KIND, bool REST>
struct Piece {
    float a[kSteps][V], u[kSteps][V];
    float lg[V];                         // log2 of all 8 gates
    __device__ __forceinline__ Piece(const Rows<EX, V> &x, const Rows<EG, V> &g, float inv_tau) {
#pragma unroll
        for (int i = 0; i < V; ++i) lg[i] = 0.f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const Gate t = gate_of<KIND, false>(to_float(g.r[j].e[i]), inv_tau);
                const float v = to_float(x.r[j].e[i]);
                a[j][i] = t.a;
                u[j][i] = REST ? -less_one(t.lg * kLn2, t.a) * v : v;
                lg[i] += t.lg;
            }
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

// First pass: a wave takes one unit of 64 V channels, 8 steps at a time with the next 8 on their way.
template <typename EX, typename EG, int V, int KIND, bool REST, bool BACK>
__global__ __launch_bounds__(256) void units_kernel(const RecurCall c, const void *d_out, const RecurUnits u, bool flat, int groups) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const long long task = (long long)blockIdx.x * 4 + wave;
    if (task >= (long long)groups * c.nunits) return;
    // neighbouring waves: neighbouring channels, whose rows lie beside each other
    const int unit = (int)(task / groups), group = (int)(task - (long long)unit * groups);
    const Place<V> p(c, flat, group);
    const int begin = unit * c.unit, end = min(begin + c.unit, c.T);
    float lg[V] = {}, h[V] = {}, adj[V] = {};
    Rows<EX, V> x, o;
    Rows<EG, V> g;
    auto fetch = [&](int s) {
        const bool whole = __all(s + kSteps <= p.loads);
        x.load(c.x, c, p, s, whole, (EX)0);
        g.load(c.gate, c, p, s, whole, open_gate<EG, KIND>());
        if constexpr (BACK) o.load(d_out, c, p, s, whole, (EX)0);
    };
    fetch(begin);                        // (a unit ends at a multiple of 8 steps or at T)
    for (int s = begin; s < end; s += kSteps) {
        const Piece<EX, EG, V, KIND, REST> q(x, g, c.inv_tau);
        float dd[BACK ? kSteps : 1][V];
        if constexpr (BACK) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) dd[j][i] = to_float(o.r[j].e[i]);
        }
        if (s + kSteps < end) fetch(s + kSteps);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) t = __builtin_fmaf(q.a[j][i], t, q.u[j][i]);
            h[i] = decayed(q.lg[i], h[i]) + t;
            if constexpr (BACK) {
                float b = 0.f;
#pragma unroll
                for (int j = kSteps - 1; j >= 0; --j) b = q.a[j][i] * (dd[j][i] + b);
                adj[i] += __builtin_amdgcn_exp2f(lg[i]) * b;
            }
            lg[i] += q.lg[i];
        }
    }
    if (!p.any) return;
    const long long at = ((long long)p.b * c.nunits + unit) * c.D + p.channel;
    store_state<V>(u.decay, at, lg);
    store_state<V>(u.state, at, h);
    if constexpr (BACK) store_state<V>(u.adjoint, at, adj);
}

// Chains the units of 64 channels: 16 waves take as many runs of units, compose each, chain the runs through LDS and walk their runs again, where
// what enters a unit takes the place of what it makes of zero.
constexpr int kCarryWaves = 16;
template <bool BACK>
__global__ __launch_bounds__(64 * kCarryWaves) void carry_kernel(const RecurCall c, const RecurUnits u, const float *first, const float *last, float *d_first) {
    __shared__ float run_lg[kCarryWaves][64], run_s[kCarryWaves][64];
    constexpr int kAtOnce = 8;           // units whose loads are under way together
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int blocks = (c.D + 63) / 64;
    const int b = blockIdx.x / blocks, ch = (blockIdx.x - b * blocks) * 64 + lane;
    const bool any = ch < c.D;
    const int each = (c.nunits + kCarryWaves - 1) / kCarryWaves;
    const bool back = BACK && blockIdx.y == 1;
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

// Second pass: a work-group walks one span (unit) of 64 V channels in rounds, 8 steps a wave.  Bound by HBM.
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kWaves) void walk_kernel(const RecurCall c, const RecurUnits u, const float *first, void *out, int out_dtype,
                                                           float *final_state, bool flat, int groups) {
    __shared__ float lds_lg[2][kWaves][64][V], lds_a[2][kWaves][64][V], lds_h[2][kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    const int unit = blockIdx.x / (unsigned)groups, group = blockIdx.x - (unsigned)unit * (unsigned)groups;
    const Place<V> p(c, flat, group);
    const int begin = unit * c.unit, end = min(begin + c.unit, c.T);
    const int round = kSteps * waves;
    float carry[V] = {};
    if (c.nunits > 1) {
        if (p.any) load_state<V>(u.state, ((long long)p.b * c.nunits + unit) * c.D + p.channel, carry);
    } else if (first != nullptr) {
        if (p.any) load_state<V>(first, p.cell(c), carry);
    }
    Rows<EX, V> x;
    Rows<EG, V> g;
    auto fetch = [&](int s) {
        const bool whole = __all(s + kSteps <= p.loads);
        x.load(c.x, c, p, s, whole, (EX)0);
        g.load(c.gate, c, p, s, whole, open_gate<EG, KIND>());
    };
    fetch(begin + wave * kSteps);
    int buf = 0;
    for (int s0 = begin; s0 < end; s0 += round, buf ^= 1) {
        const int s = s0 + wave * kSteps;
        const Piece<EX, EG, V, KIND, REST> q(x, g, c.inv_tau);
        if (s0 + round < end) fetch(s + round);
        float h[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            h[i] = 0.f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) h[i] = __builtin_fmaf(q.a[j][i], h[i], q.u[j][i]);
            lds_lg[buf][wave][lane][i] = q.lg[i];
            lds_a[buf][wave][lane][i] = __builtin_amdgcn_exp2f(q.lg[i]);
            lds_h[buf][wave][lane][i] = h[i];
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
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) mine[i] = __builtin_fmaf(q.a[j][i], mine[i], q.u[j][i]);
            if (s + j < p.n) store<V>(out, out_dtype, p.row(c, s + j), p.at, mine);
        }
    }
    if (final_state != nullptr && unit == c.nunits - 1 && wave == 0 && p.any) store_state<V>(final_state, p.cell(c), carry);
}

// Gradients of one round of 64 V channels: states from the front, adjoints from behind, 8 steps a wave.  Bound by HBM.
template <typename EX, typename EG, int V, int KIND, bool REST>
__global__ __launch_bounds__(64 * kWaves) void back_kernel(const RecurCall c, const void *d_out, const RecurUnits u, const float *first, const float *last,
                                                           void *dx, void *dgate, int grad_dtype, float *d_first, bool flat, int groups) {
    __shared__ float lds_lg[kWaves][64][V], lds_h[kWaves][64][V], lds_o[kWaves][64][V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    const int unit = blockIdx.x / (unsigned)groups, group = blockIdx.x - (unsigned)unit * (unsigned)groups;
    const Place<V> p(c, flat, group);
    const int s = unit * kRecurRound + wave * kSteps;
    Rows<EX, V> x, o;
    Rows<EG, V> g;
    const bool whole = __all(s + kSteps <= p.loads);
    x.load(c.x, c, p, s, whole, (EX)0);
    g.load(c.gate, c, p, s, whole, open_gate<EG, KIND>());
    o.load(d_out, c, p, s, whole, (EX)0);
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
    Piece<EX, EG, V, KIND, REST> q(x, g, c.inv_tau);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float t = 0.f, b = 0.f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) t = __builtin_fmaf(q.a[j][i], t, q.u[j][i]);
#pragma unroll
        for (int j = kSteps - 1; j >= 0; --j) b = q.a[j][i] * (to_float(o.r[j].e[i]) + b);
        lds_lg[wave][lane][i] = q.lg[i];
        lds_h[wave][lane][i] = t;
        lds_o[wave][lane][i] = b;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = decayed(lds_lg[w][lane][i], h[i]) + lds_h[w][lane][i];
    for (int w = waves - 1; w > wave; --w)
#pragma unroll
        for (int i = 0; i < V; ++i) adj[i] = decayed(lds_lg[w][lane][i], adj[i]) + lds_o[w][lane][i];
    // the state before each step takes the place of its input
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float before = h[i];
            h[i] = __builtin_fmaf(q.a[j][i], h[i], q.u[j][i]);
            q.u[j][i] = before;
        }
#pragma unroll
    for (int j = kSteps - 1; j >= 0; --j) {
        float gx[V], gg[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const Gate t = gate_of<KIND, true>(to_float(g.r[j].e[i]), c.inv_tau);
            const float G = to_float(o.r[j].e[i]) + adj[i], v = to_float(x.r[j].e[i]);
            gx[i] = REST ? -less_one(t.lg * kLn2, t.a) * G : G;
            // a closed gate lets nothing through, whatever stands before it; nor does the gate of a step behind the end, which is open and has no slope
            gg[i] = q.a[j][i] * (REST ? q.u[j][i] - v : q.u[j][i]) * G * t.slope;
            adj[i] = q.a[j][i] * G;
        }
        const int t = s + j;
        if (t < c.T && p.any) {          // rows behind a sequence's end are cleared
            if (t >= p.n)
#pragma unroll
                for (int i = 0; i < V; ++i) gx[i] = gg[i] = 0.f;
            if (whole || t < p.n || c.seq_lens == nullptr) {
                store<V>(dx, grad_dtype, p.row(c, t), p.at, gx);
                store<V>(dgate, grad_dtype, p.row(c, t), p.at, gg);
            } else {                     // (step t of a reversed scan would lie before the sequence: its token is t itself)
                const long long row = ((long long)p.b * c.T + t) * c.D;
                store<V>(dx, grad_dtype, row, (uint32_t)p.channel, gx);
                store<V>(dgate, grad_dtype, row, (uint32_t)p.channel, gg);
            }
        }
    }
    if (unit == 0 && c.nunits == 1 && wave == 0 && d_first != nullptr && p.any) store_state<V>(d_first, p.cell(c), adj);
}

// One step of every sequence: a thread has V channels
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
        const Gate t = gate_of<KIND, false>(to_float(g.e[i]), c.inv_tau);
        const float v = to_float(x.e[i]), rest = -less_one(t.lg * kLn2, t.a);
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
    int count;
};
Groups groups_of(const RecurCall &c, int V) {
    const long long cols = c.D / V, spanned = 64 / cols + 2;                       // sequences that a wave can touch
    // (elements up to the last of them in 32 bits as bytes)
    const bool flat = cols % 64 != 0 && spanned * c.T < (1LL << 30) / c.D;
    return {flat, (int)(flat ? (c.B * cols + 63) / 64 : c.B * ((cols + 63) / 64))};
}

}  // namespace

hipError_t launch_recur_units(const RecurCall &c, const void *d_out, const RecurUnits &u, hipStream_t stream) {
    return instance(c, c.D % 2 == 0, [&](auto x, auto g, auto kind, auto rest, auto v) {
        using EX = decltype(x);
        using EG = decltype(g);
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        const dim3 grid((unsigned)(((long long)n.count * c.nunits + 3) / 4));
        if (d_out != nullptr)
            hipLaunchKernelGGL((units_kernel<EX, EG, V, kind.value, rest.value, true>), grid, dim3(256), 0, stream, c, d_out, u, n.flat, n.count);
        else
            hipLaunchKernelGGL((units_kernel<EX, EG, V, kind.value, rest.value, false>), grid, dim3(256), 0, stream, c, d_out, u, n.flat, n.count);
        return hipGetLastError();
    });
}

hipError_t launch_recur_carry(const RecurCall &c, const RecurUnits &u, const float *first, const float *last, float *d_first, hipStream_t stream) {
    const unsigned blocks = (unsigned)((c.D + 63) / 64) * (unsigned)c.B;
    if (u.adjoint != nullptr)
        hipLaunchKernelGGL(carry_kernel<true>, dim3(blocks, 2), dim3(64 * kCarryWaves), 0, stream, c, u, first, last, d_first);
    else
        hipLaunchKernelGGL(carry_kernel<false>, dim3(blocks), dim3(64 * kCarryWaves), 0, stream, c, u, first, last, d_first);
    return hipGetLastError();
}

static unsigned waves_for(int steps) {
    const int w = (steps + kSteps - 1) / kSteps;
    return 64u * (unsigned)(w < kWaves ? w : kWaves);
}

hipError_t launch_recur_walk(const RecurCall &c, const RecurUnits &u, const float *first, void *out, int out_dtype, float *final_state,
                             hipStream_t stream) {
    return instance(c, c.D % 2 == 0, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const Groups n = groups_of(c, V);
        hipLaunchKernelGGL((walk_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((long long)n.count * c.nunits)),
                           dim3(waves_for(c.unit)), 0, stream, c, u, first, out, out_dtype, final_state, n.flat, n.count);
        return hipGetLastError();
    });
}

hipError_t launch_recur_back(const RecurCall &c, const void *d_out, const RecurUnits &u, const float *first, const float *last, void *dx,
                             void *dgate, int grad_dtype, float *d_first, hipStream_t stream) {
    return instance(c, c.D % 2 == 0, [&](auto x, auto g, auto kind, auto rest, auto v) {
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
    return instance(c, c.D % 2 == 0 && all % 8 == 0, [&](auto x, auto g, auto kind, auto rest, auto v) {
        constexpr int V = decltype(v)::value;
        const long long lanes = (long long)c.B * c.D / V;
        hipLaunchKernelGGL((step_kernel<decltype(x), decltype(g), V, kind.value, rest.value>), dim3((unsigned)((lanes + 63) / 64)), dim3(64), 0, stream, c,
                           state, state_out, out, out_dtype);
        return hipGetLastError();
    });
}

}  // namespace gla
