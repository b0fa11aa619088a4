// Linear attention with one decay a head: the walks that go forward (outputs; for the backward pass dq), the local states of spans and
// the chain that joins them, and the form for single tokens.  The mathematics and the chunk are in gla_decay.h and gla_decay_util.h.
#include "gla_decay_util.h"

namespace gla {
namespace {

constexpr int kThreads = 256;

template <typename E, int M, int N>
struct WalkLds {
    static constexpr int kRowsM = Tile<E, M, kBoth>::kBytes, kRowsN = Tile<E, N, kAcross>::kBytes, kX = 0, kY = Tile<E, M, kAlong>::kBytes, kZ = kY + kRowsM,
                         kP = kZ + kRowsN, kG = kP + Pairs<E>::kBytes, kFlow = kG + 2 * (int)sizeof(Gates<Elem<E>::kChunk>),
                         kDiag = kFlow + 2 * 4 * Elem<E>::kChunk * 4, kBytes = kDiag + Elem<E>::kChunk * 4;
};

// GRAD: the walk for dq, with the dot products and the states that the gates' gradient takes
template <typename E, int M, int N, bool FAST, bool GRAD>
__global__ __launch_bounds__(kThreads, 2) void decay_walk_kernel(const DecayWalk p) {
    constexpr int C = Elem<E>::kChunk;
    typedef WalkLds<E, M, N> L;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Tile<E, M, kAlong> tx{lds + L::kX};
    const Tile<E, M, kBoth> ty{lds + L::kY};
    const Tile<E, N, kAcross> tz{lds + L::kZ};
    const Pairs<E> P{lds + L::kP};
    Gates<C> *gates = reinterpret_cast<Gates<C> *>(lds + L::kG);
    float *flow_part = reinterpret_cast<float *>(lds + L::kFlow), *diag = reinterpret_cast<float *>(lds + L::kDiag);

    const int tid = threadIdx.x, lane = tid & 63;
    const int bh = blockIdx.x / p.c.nspans, sp = blockIdx.x - bh * p.c.nspans;
    const Order ord = order_of(p.c, bh);
    const int len = ord.len;
    const int s0 = sp * p.c.span_len, s1 = min(s0 + p.c.span_len, p.c.T), end = min(s1, len);
    const int m = p.r.m, n = p.r.n;
    const size_t cells = (size_t)m * n;
    const Rows rx = rows_of<E>(p.c, p.r.x, bh, m), ry = rows_of<E>(p.c, p.r.y, bh, m), rz = rows_of<E>(p.c, p.r.z, bh, n);
    const Rows ro = rows_of<E>(p.c, p.r.out, bh, n, p.out_dtype == GLA_DT_BF16 ? 2 : 4);

    Walker<E, M, N, FAST, false> wk;
    wk.init(tid);
    Pieces<E, M, kThreads, FAST> px, py;
    Pieces<E, N, kThreads, FAST> pz;
    float gate = 0.f;
    auto issue = [&](int s) __attribute__((always_inline)) {
        const int tid = recompute_per_chunk(threadIdx.x), lane = tid & 63;
        const Steps st = ord.steps(s, min(C, end - s), false);
        if (wk.w == 3) gate = lane < st.count ? gate_of(p.c, ord, bh, s + lane) : 0.f;
        px.issue(rx, tid, st);
        py.issue(ry, tid, st);
        pz.issue(rz, tid, st);
    };
    if (s0 < end) issue(s0);
    wk.enter(p.in, bh, sp, p.c.nspans, false, m, n, p.state_t);
    auto bring = [&](int turn) __attribute__((always_inline)) {
        px.commit(rx, tid, tx);
        py.commit(ry, tid, ty);
        pz.commit(rz, tid, tz);
        if (wk.w == 3) form_gates(gates[turn], gate, lane);
    };
    const bool dots = GRAD && p.r.dot != nullptr;
    // the dot products of a chunk are added over the waves once the barrier behind it is passed
    auto put_flow = [&](int s, int count, int turn) __attribute__((always_inline)) {
        const float *f = flow_part + 4 * C * turn;
        if (tid < count) p.r.flow[(size_t)bh * p.c.T + s + tid] = (f[tid] + f[C + tid]) + (f[2 * C + tid] + f[3 * C + tid]);
    };
    if (s0 < end) bring(0);
    int turn = 0;
    for (int s = s0; s < end; s += C, turn ^= 1) {
        const int count = min(C, end - s), e = s + count;
        const Gates<C> &gt = gates[turn];
        u32x4 zf[C / Elem<E>::kDeep][N / 64];
        typename Walker<E, M, N, FAST, false>::Dots d;
        __syncthreads();
        if (dots) wk.fetch_dots(d, rows_of<E>(p.c, p.r.dot, bh, n), ord.steps(s, count, false));
        if (e < end) issue(e);
        if (dots && s > s0) put_flow(s - C, C, turn ^ 1);
        __builtin_amdgcn_s_setprio(1);                   // before the other work-group's loads and stores (3 % less time)
        wk.pairs(tx, ty, P, gt, dots, diag);
        wk.from_state(tx, gt);
        wk.update(ty, tz, gt, zf);
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();
        wk.finish(P, zf);
        if (dots) {                                      // the diagonal has no part in the dot products (gla_decay.h)
            wk.dot_rows(d, flow_part + 4 * C * turn);
            wk.add_diagonal(diag, zf);
        }
        const Steps st = ord.steps(s, count, false);
        wk.store_rows(ro, p.out_dtype, st);
        if (e < end) bring(turn ^ 1);
        if (GRAD && p.anchors != nullptr && (e < len ? e % kFlowBlock == 0 : p.anchor_last != 0))
            wk.store_state(p.anchors + ((size_t)bh * decay_blocks(p.c.T) + (e - 1) / kFlowBlock) * cells, m, n, p.state_t);
    }
    if (dots && s0 < end) {
        __syncthreads();
        const int s = s0 + (end - s0 - 1) / C * C;
        put_flow(s, end - s, turn ^ 1);
    }
    if (p.state_out != nullptr && sp == p.c.nspans - 1) wk.store_state(p.state_out + (size_t)bh * cells, m, n, p.state_t);
    if (GRAD) clear_behind<kThreads>(ro, p.out_dtype == GLA_DT_BF16 ? 2 : 4, len, s0, s1, tid);
}

struct StatePair {
    DecayWalk w[2];
};

// Local states: y, z of the role only.  blockIdx.y = 1: the reversed recurrence
template <typename E, int M, int N, bool FAST>
__global__ __launch_bounds__(kThreads, 2) void decay_state_kernel(const StatePair both) {
    constexpr int C = Elem<E>::kChunk;
    typedef WalkLds<E, M, N> L;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Tile<E, M, kBoth> ty{lds};
    const Tile<E, N, kAcross> tz{lds + L::kRowsM};
    Gates<C> *gates = reinterpret_cast<Gates<C> *>(lds + L::kRowsM + L::kRowsN);

    const bool back = blockIdx.y != 0;
    const DecayWalk &p = both.w[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63;
    const int walked = p.c.nspans - 1;                   // nobody needs the last one's
    if ((int)blockIdx.x >= p.c.B * p.c.H * walked) return;
    const int bh = blockIdx.x / walked, sp = blockIdx.x - bh * walked + (back ? 1 : 0);
    const Order ord = order_of(p.c, bh);
    const int s0 = sp * p.c.span_len, end = min(min(s0 + p.c.span_len, p.c.T), ord.len);
    const int m = p.r.m, n = p.r.n;
    const Rows ry = rows_of<E>(p.c, p.r.y, bh, m), rz = rows_of<E>(p.c, p.r.z, bh, n);

    Walker<E, M, N, FAST, false> wk;
    wk.init(tid);
    wk.load_state(nullptr, m, n, false);
    Pieces<E, M, kThreads, FAST> py;
    Pieces<E, N, kThreads, FAST> pz;
    float gate = 0.f, sum = 0.f;
    const int chunks = s0 < end ? (end - s0 + C - 1) / C : 0;
    auto issue = [&](int i) __attribute__((always_inline)) {
        const int tid = recompute_per_chunk(threadIdx.x), lane = tid & 63;
        const int s = s0 + (back ? chunks - 1 - i : i) * C, e = min(s + C, end);
        const Steps st = ord.steps(s, e - s, back);
        if (wk.w == 3) gate = lane < e - s ? gate_of(p.c, ord, bh, back ? e - lane : s + lane) : 0.f;
        py.issue(ry, tid, st);
        pz.issue(rz, tid, st);
    };
    if (chunks > 0) {
        issue(0);
        if (wk.w == 3) form_gates(gates[0], gate, lane);
    }
    for (int i = 0; i < chunks; ++i) {
        const Gates<C> &gt = gates[i & 1];
        py.commit(ry, tid, ty);
        pz.commit(rz, tid, tz);
        __syncthreads();
        if (i + 1 < chunks) issue(i + 1);
        sum += gt.sum;
        u32x4 zf[C / Elem<E>::kDeep][N / 64];
        wk.update(ty, tz, gt, zf);
        if (wk.w == 3 && i + 1 < chunks) form_gates(gates[(i + 1) & 1], gate, lane);
        __syncthreads();
    }
    const size_t at = (size_t)bh * p.c.nspans + sp;
    wk.store_state(p.local + at * m * n, m, n, p.state_t);
    if (tid == 0) p.decay[at] = sum;
}

// local [B*H, nspans, cells]: entry sp becomes the state that enters span sp.  A thread has one element of all of a sequence's spans; it asks
// for eight of them before it uses the first, as each one's place is written in turn (65536 steps of 16 heads 128 x 128 in 32 spans: 19 us, 3.5 TB/s).
// blockIdx.y: the forward and the reversed chain.
__global__ __launch_bounds__(kThreads) void decay_carry_kernel(const DecayChain c0, const DecayChain c1, int cells) {
    constexpr int kAhead = 8;
    const DecayChain c = blockIdx.y == 0 ? c0 : c1;
    const int parts = (cells + kThreads - 1) / kThreads;
    const int bh = blockIdx.x / parts, i = (blockIdx.x - bh * parts) * kThreads + threadIdx.x;
    if (c.nspans < 2 || i >= cells) return;
    float *u = c.local + (size_t)bh * c.nspans * cells + i;
    const float *decay = c.decay + (size_t)bh * c.nspans;
    float s = c.first != nullptr ? c.first[(size_t)bh * cells + i] : 0.f;
    for (int k0 = 0; k0 < c.nspans; k0 += kAhead) {
        float own[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int sp = c.reversed ? c.nspans - 1 - k0 - k : k0 + k;
            own[k] = k0 + k < c.nspans - 1 ? u[(size_t)sp * cells] : 0.f;       // (the last one walked has no local state)
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k0 + k >= c.nspans) break;
            const int sp = c.reversed ? c.nspans - 1 - k0 - k : k0 + k;
            u[(size_t)sp * cells] = s;
            if (k0 + k < c.nspans - 1) s = fmaf(exp2_fast(decay[sp]), s, own[k]);
        }
    }
}

template <typename K>
hipError_t configured(K kernel, int bytes, std::atomic<bool> (&done)[kMaxDevices]) {
    return allow_dynamic_lds(reinterpret_cast<const void *>(kernel), bytes, done);
}

template <typename E, int M, int N, bool FAST, bool GRAD>
hipError_t walk(const DecayWalk &w, hipStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    constexpr int bytes = WalkLds<E, M, N>::kBytes;
    const hipError_t e = configured(decay_walk_kernel<E, M, N, FAST, GRAD>, bytes, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((decay_walk_kernel<E, M, N, FAST, GRAD>), dim3((unsigned)(w.c.B * w.c.H * w.c.nspans)), dim3(kThreads), bytes, stream, w);
    return hipGetLastError();
}

template <typename E, int M, int N, bool FAST>
hipError_t states(const StatePair &w, int directions, hipStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    constexpr int bytes = WalkLds<E, M, N>::kRowsM + WalkLds<E, M, N>::kRowsN + 2 * (int)sizeof(Gates<Elem<E>::kChunk>);
    const hipError_t e = configured(decay_state_kernel<E, M, N, FAST>, bytes, done);
    if (e != hipSuccess) return e;
    const DecayCall &c = w.w[0].c;
    const int spans = directions == 2 && w.w[1].c.nspans > c.nspans ? w.w[1].c.nspans : c.nspans;
    hipLaunchKernelGGL((decay_state_kernel<E, M, N, FAST>), dim3((unsigned)(c.B * c.H * (spans - 1)), (unsigned)directions), dim3(kThreads),
                       bytes, stream, w);
    return hipGetLastError();
}

// One token.  A work-group takes 32 columns of one (batch, head)'s state, eight lanes of four columns by 32 rows, all of whose rows it asks for
// before it uses the first.  Columns need nothing of each other, so that few states are dealt to many work-groups (16 states 128 x 128:
// 3.8 us, 5.0 with whole rows).  Bound by the states' way in and out (192 sequences of 16 heads: 80 us, 5.1 TB/s, a copy reaches 5.2), for few by the launch.
constexpr int kStepCols = 32, kStepLanes = kStepCols / 4, kStepRows = kThreads / kStepLanes, kStepTimes = kDecayMaxD / kStepRows;
template <typename E>
__device__ inline float element(const void *p, size_t i) {
    if constexpr (sizeof(E) == 2) return bf16_bits_to_float(static_cast<const uint16_t *>(p)[i]);
    else return static_cast<const float *>(p)[i];
}

template <typename E>
__global__ __launch_bounds__(kThreads) void decay_step_kernel(const void *q, const void *k, const void *v, const float *log_decay, int kind,
                                                              int H, int dk, int dv, int out_dtype, const float *state, float *state_out,
                                                              void *out) {
    __shared__ float s_q[kDecayMaxD], s_k[kDecayMaxD], s_o[kThreads / 64][kStepCols];
    const int tid = threadIdx.x, parts = (dv + kStepCols - 1) / kStepCols;
    const int bh = blockIdx.x / parts, h = bh % H, c0 = (blockIdx.x - bh * parts) * kStepCols;
    const int col = c0 + tid % kStepLanes * 4, row0 = tid / kStepLanes;
    const size_t cells = (size_t)dk * dv;
    const float *s = state + bh * cells;
    float *t = state_out + bh * cells;
    f32x4 c[kStepTimes];
#pragma unroll
    for (int i = 0; i < kStepTimes; ++i) {
        const int r = row0 + i * kStepRows;
        c[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (r >= dk) continue;
        if (col + 4 <= dv) {
            __builtin_memcpy(&c[i], s + (size_t)r * dv + col, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + j < dv) c[i][j] = s[(size_t)r * dv + col + j];
        }
    }
    if (tid < kDecayMaxD) s_q[tid] = tid < dk ? element<E>(q, (size_t)bh * dk + tid) : 0.f;
    else if (tid < 2 * kDecayMaxD) s_k[tid - kDecayMaxD] = tid - kDecayMaxD < dk ? element<E>(k, (size_t)bh * dk + tid - kDecayMaxD) : 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < dv) x[j] = element<E>(v, (size_t)bh * dv + col + j);
    const float a = exp2_fast(gate_log2(log_decay[kind == kDecayHead ? h : bh]));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kStepTimes; ++i) {
        const int r = row0 + i * kStepRows;
        c[i] = c[i] * a + x * s_k[r];
        o += c[i] * s_q[r];
        if (r >= dk) continue;
        if (col + 4 <= dv) {
            __builtin_memcpy(t + (size_t)r * dv + col, &c[i], 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + j < dv) t[(size_t)r * dv + col + j] = c[i][j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float y = o[j];
#pragma unroll
        for (int d = kStepLanes; d < 64; d *= 2) y += __shfl_xor(y, d);
        if ((tid & 63) < kStepLanes) s_o[tid >> 6][(tid & 63) * 4 + j] = y;
    }
    __syncthreads();
    if (tid < kStepCols && c0 + tid < dv) {
        const float y = (s_o[0][tid] + s_o[1][tid]) + (s_o[2][tid] + s_o[3][tid]);
        const size_t at = (size_t)bh * dv + c0 + tid;
        if (out_dtype == GLA_DT_BF16) static_cast<uint16_t *>(out)[at] = float_to_bf16_bits(y);
        else static_cast<float *>(out)[at] = y;
    }
}

}  // namespace

template <typename E, bool GRAD>
static hipError_t walk_of_size(const DecayWalk &w, hipStream_t stream) {
    return decay_sizes(w.r.m, w.r.n, w.c.fast, [&](auto m, auto n, auto fast) {
        return walk<E, decltype(m)::value, decltype(n)::value, decltype(fast)::value, GRAD>(w, stream);
    });
}

hipError_t launch_decay_walk(const DecayWalk &w, int dtype, hipStream_t stream) {
    if (dtype == GLA_DT_BF16) {
        // (the walk for dq gives no state)
        if (w.grad) return w.c.digits == kDigitsAll ? walk_of_size<Bf16<3, 3>, true>(w, stream) : walk_of_size<Bf16<2, 2>, true>(w, stream);
        return w.c.digits == kDigitsStates ? walk_of_size<Bf16<3, 2>, false>(w, stream) : walk_of_size<Bf16<2, 2>, false>(w, stream);
    }
    return w.grad ? walk_of_size<float, true>(w, stream) : walk_of_size<float, false>(w, stream);
}

hipError_t launch_decay_states(const DecayWalk &w, const DecayWalk *back, int dtype, hipStream_t stream) {
    StatePair both;
    both.w[0] = w;
    both.w[1] = back != nullptr ? *back : w;
    const int d = back != nullptr ? 2 : 1;
    return decay_sizes(w.r.m, w.r.n, w.c.fast, [&](auto m, auto n, auto fast) {
        constexpr int M = decltype(m)::value, N = decltype(n)::value;
        constexpr bool F = decltype(fast)::value;
        if (dtype != GLA_DT_BF16) return states<float, M, N, F>(both, d, stream);
        return w.c.digits == kDigitsRows ? states<Bf16<2, 2>, M, N, F>(both, d, stream) : states<Bf16<3, 3>, M, N, F>(both, d, stream);
    });
}

hipError_t launch_decay_carry(const DecayCall &c, const DecayChain &chain, const DecayChain *other, hipStream_t stream) {
    const int cells = c.dk * c.dv;
    const long long groups = (long long)c.B * c.H * ((cells + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(decay_carry_kernel, dim3((unsigned)groups, other != nullptr ? 2u : 1u), dim3(kThreads), 0, stream, chain,
                       other != nullptr ? *other : chain, cells);
    return hipGetLastError();
}

hipError_t launch_decay_step(const void *q, const void *k, const void *v, const float *log_decay, int kind, int B, int H, int dk, int dv,
                             int dtype, int out_dtype, const float *state, float *state_out, void *out, hipStream_t stream) {
    const dim3 grid((unsigned)(B * H * ((dv + kStepCols - 1) / kStepCols)));
    hipLaunchKernelGGL((dtype == GLA_DT_BF16 ? decay_step_kernel<uint16_t> : decay_step_kernel<float>), grid, dim3(kThreads), 0, stream, q, k, v,
                       log_decay, kind, H, dk, dv, out_dtype, state, state_out, out);
    return hipGetLastError();
}

}  // namespace gla
