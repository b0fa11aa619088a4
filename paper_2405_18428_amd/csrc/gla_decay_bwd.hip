// Backward pass of linear attention with one decay a head: the walk that goes backwards, for dv and dk at once, and the gates' gradient
// (gla_decay.h has the mathematics; the walk for dq is the forward kernel of gla_decay.hip on other rows).
#include "gla_decay_util.h"

namespace gla {
namespace {

// Eight waves: four walk the adjoint state G [dk, dv] for dv (rows k, q, dO), four its transpose for dk (rows v, dO, q), from the same
// four tiles.  Two copies of G cost matrix instructions, which there is room for, and save both a second reading of the rows and the
// sum over waves that a product along a wave's own columns would need.
constexpr int kThreads = 512;

template <typename E, typename E1, int K, int V>
struct BackLds {
    static constexpr int kRowsV = Tile<E, V, kBoth>::kBytes, kQ = 0, kK = Tile<E, K, kBoth>::kBytes, kV = kK + Tile<E, K, kAlong>::kBytes,
                         kD = kV + Tile<E, V, kAlong>::kBytes, kPa = kD + kRowsV, kPb = kPa + Pairs<E>::kBytes, kG = kPb + Pairs<E1>::kBytes,
                         kFlow = kG + 2 * (int)sizeof(Gates<Elem<E>::kChunk>), kDiag = kFlow + 2 * 4 * Elem<E>::kChunk * 4,
                         kMeet = kDiag + Elem<E>::kChunk * 4, kBytes = kMeet + 16;
};

// ROLE 0: dv and the initial state's gradient, ROLE 1: dk and the flows.  L: where what both share lies in LDS
template <typename E, typename L, int K, int V, bool FAST, int ROLE>
__device__ __forceinline__ void walk_back(const DecayBack &p, char *lds) {
    constexpr int C = Elem<E>::kChunk, M = ROLE == 0 ? K : V, N = ROLE == 0 ? V : K;
    const Tile<E, K, kBoth> tq{lds + L::kQ};
    const Tile<E, K, kAlong> tk{lds + L::kK};
    const Tile<E, V, kAlong> tv{lds + L::kV};
    const Tile<E, V, kBoth> td{lds + L::kD};
    const Pairs<E> P{lds + (ROLE == 0 ? L::kPa : L::kPb)};
    Gates<C> *gates = reinterpret_cast<Gates<C> *>(lds + L::kG);
    float *flow_part = reinterpret_cast<float *>(lds + L::kFlow), *diag = reinterpret_cast<float *>(lds + L::kDiag),
          *meet_part = reinterpret_cast<float *>(lds + L::kMeet);

    const int tid = threadIdx.x;
    const int bh = blockIdx.x / p.c.nspans, sp = blockIdx.x - bh * p.c.nspans;
    const Order ord = order_of(p.c, bh);
    const int len = ord.len, dk = p.c.dk, dv = p.c.dv;
    const int s0 = sp * p.c.span_len, s1 = min(s0 + p.c.span_len, p.c.T), end = min(s1, len);
    const size_t cells = (size_t)dk * dv;
    const int m = ROLE == 0 ? dk : dv, n = ROLE == 0 ? dv : dk;
    const Rows rq = rows_of<E>(p.c, p.q, bh, dk), rk = rows_of<E>(p.c, p.k, bh, dk), rv = rows_of<E>(p.c, p.v, bh, dv),
               rd = rows_of<E>(p.c, p.d_out, bh, dv);
    const Rows ro = rows_of<E>(p.c, ROLE == 0 ? p.dv_grad : p.dk_grad, bh, n, p.grad_dtype == GLA_DT_BF16 ? 2 : 4);

    Walker<E, M, N, FAST, true> wk;
    wk.init(tid);
    Pieces<E, K, kThreads, FAST> pq, pk;
    Pieces<E, V, kThreads, FAST> pv, pd;
    float gate = 0.f;
    auto issue = [&](int s, int e) __attribute__((always_inline)) {      // steps [s, e), row 0 = step e - 1
        const int tid = recompute_per_chunk(threadIdx.x), lane = tid & 63;
        const Steps st = ord.steps(s, e - s, true);
        if (ROLE == 0 && wk.w == 3) gate = lane < st.count ? gate_of(p.c, ord, bh, e - lane) : 0.f;   // the gate that led out of the step
        pq.issue(rq, tid, st);
        pk.issue(rk, tid, st);
        pv.issue(rv, tid, st);
        pd.issue(rd, tid, st);
    };
    const int chunks = s0 < end ? (end - s0 + C - 1) / C : 0;
    auto bring = [&](int turn) __attribute__((always_inline)) {
        pq.commit(rq, tid, tq);
        pk.commit(rk, tid, tk);
        pv.commit(rv, tid, tv);
        pd.commit(rd, tid, td);
        if (ROLE == 0 && wk.w == 3) form_gates(gates[turn], gate, wk.lane);
    };
    const bool flows = ROLE == 1 && p.anchors != nullptr;
    // the dot products of a chunk are added over the waves once the barrier behind it is passed
    auto put_flow = [&](int s, int e, int turn) __attribute__((always_inline)) {
        const int i = tid - 256;
        const float *f = flow_part + 4 * C * turn;
        if (i < e - s) p.flow_k[(size_t)bh * p.c.T + e - 1 - i] = (f[i] + f[C + i]) + (f[2 * C + i] + f[3 * C + i]);
    };
    if (chunks > 0) issue(s0 + (chunks - 1) * C, end);
    wk.enter(p.in, bh, sp, p.c.nspans, true, m, n, ROLE == 1);
    if (chunks > 0) bring((chunks - 1) & 1);
    for (int ci = chunks - 1; ci >= 0; --ci) {
        const int s = s0 + ci * C, e = min(s + C, end), count = e - s;
        const Gates<C> &gt = gates[ci & 1];
        u32x4 zf[C / Elem<E>::kDeep][N / 64];
        typename Walker<E, M, N, FAST, true>::Dots d;
        __syncthreads();
        if (ci > 0) issue(s - C, s);
        if (flows && ci < chunks - 1) put_flow(s + C, min(s + 2 * C, end), ci + 1 & 1);
        // the state at the end of a block, met by its adjoint
        const size_t block = (size_t)bh * decay_blocks(p.c.T) + (e - 1) / kFlowBlock;
        const bool meets = flows && (e < len ? e % kFlowBlock == 0 : p.anchor_last != 0);
        if (meets) {
            float sum = wk.meet_state(p.anchors + block * cells, m, n, true);
#pragma unroll
            for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
            if (wk.lane == 0) meet_part[wk.w] = sum;
        }
        if constexpr (ROLE == 0) {
            wk.pairs(tk, tq, P, gt);
            wk.from_state(tk, gt);
            wk.update(tq, td, gt, zf);
        } else {
            wk.pairs(tv, td, P, gt, flows, diag);
            wk.from_state(tv, gt);
            wk.update(td, tq, gt, zf);
            if (flows) wk.fetch_dots(d, tk);
        }
        __syncthreads();
        if (meets && tid == 256) p.meet[block] = (meet_part[0] + meet_part[1]) + (meet_part[2] + meet_part[3]);
        wk.finish(P, zf);
        if (flows) {                                     // the diagonal has no part in the dot products (gla_decay.h)
            wk.dot_rows(d, flow_part + 4 * C * (ci & 1));
            wk.add_diagonal(diag, zf);
        }
        wk.store_rows(ro, p.grad_dtype, ord.steps(s, count, true));
        if (ci > 0) bring((ci - 1) & 1);
    }
    if (chunks > 0) {
        __syncthreads();
        if (flows) put_flow(s0, min(s0 + C, end), 0);
    }
    if (ROLE == 0 && p.d_initial != nullptr && sp == 0)
        wk.store_state(p.d_initial + (size_t)bh * cells, m, n, false, exp2_fast(gate_log2(gate_of(p.c, ord, bh, 0))));
    clear_behind<256>(ro, p.grad_dtype == GLA_DT_BF16 ? 2 : 4, len, s0, s1, tid & 255);
}

template <typename E0, typename E1, int K, int V, bool FAST>
__global__ __launch_bounds__(kThreads, 2) void decay_back_kernel(const DecayBack p) {
    typedef BackLds<E0, E1, K, V> L;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    // both branches meet at the same barriers: the same chunks, two each, and one behind them
    if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8) == 0) walk_back<E0, L, K, V, FAST, 0>(p, lds);
    else walk_back<E1, L, K, V, FAST, 1>(p, lds);
}

// A block of kFlowBlock steps a work-group: what flows into each, in 64 bits
__global__ __launch_bounds__(kFlowBlock) void decay_gate_kernel(const DecayGate p) {
    __shared__ double sum[kFlowBlock];
    const int t = threadIdx.x, blocks = decay_blocks(p.c.T);
    const int bh = blockIdx.x / blocks, k = blockIdx.x - bh * blocks;
    const Order ord = order_of(p.c, bh);
    const int s = k * kFlowBlock + t, len = ord.len;
    const size_t at = (size_t)bh * p.c.T + s;
    double x = s < len ? (double)p.flow_q[at] - (double)p.flow_k[at] : 0.0;
    const int e = min((k + 1) * kFlowBlock, len);
    // across the block's end: the adjoint state behind it decays once more on its way to the state before it
    double across = 0.0;
    if (k * kFlowBlock < len) {
        if (e < len) across = (double)p.meet[blockIdx.x] * (double)exp2_fast(gate_log2(gate_of(p.c, ord, bh, e)));
        else if (p.anchor_last) across = (double)p.meet[blockIdx.x];
    }
    sum[t] = x;
    __syncthreads();
    for (int d = 1; d < kFlowBlock; d *= 2) {                            // sums from each step to the block's end
        const double y = t + d < kFlowBlock ? sum[t + d] : 0.0;
        __syncthreads();
        sum[t] += y;
        __syncthreads();
    }
    // (what a gate that lets nothing through adds up to is rounding)
    const bool open = s < len && exp2_fast(gate_log2(gate_of(p.c, ord, bh, s))) != 0.f;
    const double flow = open ? sum[t] + across : 0.0;
    if (p.c.kind == kDecayToken) {
        if (s < p.c.T) {
            const int h = bh % p.c.H;
            const long long n = s < len ? ord.token(s) : s;
            p.dlog[p.c.layout == GLA_LAYOUT_BHTD ? (long long)bh * p.c.T + n : ((long long)(bh / p.c.H) * p.c.T + n) * p.c.H + h] = (float)flow;
        }
        return;
    }
    __syncthreads();
    sum[t] = flow;
    __syncthreads();
    for (int d = kFlowBlock / 2; d > 0; d /= 2) {
        if (t < d) sum[t] += sum[t + d];
        __syncthreads();
    }
    if (t == 0) p.part[blockIdx.x] = sum[0];
}

// One decay a head: the sum over its batches and blocks, in one order
__global__ __launch_bounds__(256) void decay_gate_sum_kernel(const double *part, float *dlog, int B, int H, int blocks) {
    __shared__ double sum[256];
    const int h = blockIdx.x, t = threadIdx.x;
    double x = 0.0;
    const long long all = (long long)B * blocks;
    for (long long i = t; i < all; i += 256) x += part[((i / blocks) * H + h) * blocks + i % blocks];
    sum[t] = x;
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (t < d) sum[t] += sum[t + d];
        __syncthreads();
    }
    if (t == 0) dlog[h] = (float)sum[0];
}

template <typename E0, typename E1, int K, int V, bool FAST>
hipError_t back(const DecayBack &w, hipStream_t stream) {
    static std::atomic<bool> done[kMaxDevices];
    constexpr int bytes = BackLds<E0, E1, K, V>::kBytes;
    const hipError_t e = allow_dynamic_lds(reinterpret_cast<const void *>(&decay_back_kernel<E0, E1, K, V, FAST>), bytes, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((decay_back_kernel<E0, E1, K, V, FAST>), dim3((unsigned)(w.c.B * w.c.H * w.c.nspans)), dim3(kThreads), bytes, stream, w);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_decay_back(const DecayBack &w, int dtype, hipStream_t stream) {
    return decay_sizes(w.c.dk, w.c.dv, w.c.fast, [&](auto k, auto v, auto fast) {
        constexpr int K = decltype(k)::value, V = decltype(v)::value;
        constexpr bool F = decltype(fast)::value;
        if (dtype != GLA_DT_BF16) return back<float, float, K, V, F>(w, stream);
        if (w.c.digits == kDigitsRows) return back<Bf16<2, 2>, Bf16<2, 2>, K, V, F>(w, stream);
        return w.c.digits == kDigitsStates ? back<Bf16<3, 2>, Bf16<2, 2>, K, V, F>(w, stream) : back<Bf16<3, 3>, Bf16<3, 3>, K, V, F>(w, stream);
    });
}

hipError_t launch_decay_gate(const DecayGate &w, hipStream_t stream) {
    const int blocks = decay_blocks(w.c.T);
    hipLaunchKernelGGL(decay_gate_kernel, dim3((unsigned)((long long)w.c.B * w.c.H * blocks)), dim3(kFlowBlock), 0, stream, w);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || w.c.kind == kDecayToken) return e;
    hipLaunchKernelGGL(decay_gate_sum_kernel, dim3((unsigned)w.c.H), dim3(256), 0, stream, w.part, w.dlog, w.c.B, w.c.H, blocks);
    return hipGetLastError();
}

}  // namespace gla
