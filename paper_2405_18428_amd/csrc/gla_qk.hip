// Norm of queries and keys with the rotation behind it, in one pass over each row:
//   n = x r,  r = (mean(x^2) + eps)^-1/2,  y = R (n w),
// R turning the pairs of channels by the token's angles as in gla_rope.hip; and backward, with dy' = R^-1 dy and dn = dy' w:
//   dx = r (dn - n mean(dn n)),   dw = sum over rows of dy' n.
//
// A wave takes one token, forms the sines and cosines of its angles, a pair a lane, and goes through its heads, queries and then keys: 4 to 32 lanes hold a
// row, 8 channels each, so that a wave has 2 to 16 heads at a time, which lie together where a token's heads do, with the next ones on their way.  A pair
// of neighbouring channels lies in one lane; the other channel of a pair of halves is fetched through LDS, as the sines and cosines are; all of it is
// one wave's, so there are no barriers.  Forward the norm's factor is applied last, so that the exchange does not wait for the row's sum.  Sums
// for dw stay in registers, are added over a work-group and go to memory as one partial sum a work-group, which a second kernel adds in one order.
//
// Bound by HBM: 4 x 4095 tokens of 16 + 16 heads of 128 channels, bf16, forward 268 MB in 52 us, 5.2 TB/s, backward 403 MB in 82, 4.9 TB/s.  Work-groups of 16
// tokens, a group of lanes each, which read 256 bytes a token at a time: 110 and 139 us.  Three or four turns of heads on their way instead of two: 65 and
// 91, 63 and 90 (63 and 82 then).  Rows asked for before the angles are formed: 51 and 85.  64 single tokens of 16 + 4 heads 4.7 us a call in a
// graph (6.0 in a trace), a launch and one row's loads, sum and stores.
#include "gla_qk.h"
#include "gla_rope_util.h"
#include "gla_rows.h"

namespace gla {
namespace {

constexpr int kThreads = 256;

// Over the lanes of a row, in all of them: neighbours, pairs, fours and eights of 16 lanes exchange inside the vector unit
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
    v += dpp<0xb1>(v);
    v += dpp<0x4e>(v);
    if constexpr (LANES >= 8) v += dpp<0x141>(v);        // (lane i and 7 - i)
    if constexpr (LANES >= 16) v += dpp<0x140>(v);       // (lane i and 15 - i)
    if constexpr (LANES >= 32) v += __shfl_xor(v, 16);
    return v;
}

// What a channel's turning needs, in one word (eight a lane, for all tokens): its pair, axis, whether it is the pair's second channel, whether it is
// turned at all, and the pair's other channel
struct Channel {
    uint32_t word;
    __device__ __forceinline__ Channel() = default;
    __device__ __forceinline__ Channel(const RopeParams &r, int c) {
        if (c >= 2 * r.pairs) {
            word = (uint32_t)c << 16;
            return;
        }
        int x = 0;
        while (c >= 2 * r.pairs_end[x]) ++x;
        const int off = c - r.first[x], h = r.half[x];
        const bool second = r.adjacent ? (off & 1) != 0 : off >= h;
        const int pair = r.pairs_end[x] - h + (r.adjacent ? off / 2 : second ? off - h : off);
        const int other = r.adjacent ? c ^ 1 : second ? c - h : c + h;
        word = (uint32_t)pair | (uint32_t)x << 8 | (uint32_t)second << 12 | 1u << 13 | (uint32_t)other << 16;
    }
    __device__ __forceinline__ int pair() const { return word & 255; }
    __device__ __forceinline__ int axis() const { return (word >> 8) & 15; }
    __device__ __forceinline__ bool second() const { return (word >> 12) & 1; }
    __device__ __forceinline__ bool turned() const { return (word >> 13) & 1; }
    __device__ __forceinline__ int other() const { return word >> 16; }
};

// MODE: any call, or rows that fill their lanes, all turned by neighbours, or by halves that lanes have whole (forward 82 -> 63 us, backward 104 -> 82)
enum { kAny, kNeighbours, kHalves };
template <typename E, int LANES, bool BACK, int MODE>
__global__ __launch_bounds__(kThreads) void qk_kernel(const QkParams p, int each, int parts) {
    constexpr int kRows = 64 / LANES, kWaves = kThreads / 64, kWidth = LANES * kEach, kPairs = kWidth / 2;
    __shared__ __attribute__((aligned(16))) float rows[kWaves * kRows][kWidth];
    __shared__ float2 angles[kWaves][kPairs];            // cosine, sine
    const RopeParams &r = p.rope;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int gi = threadIdx.x / LANES, sub = lane / LANES, c0 = lane % LANES * kEach, d = MODE == kAny ? r.d : kWidth;
    const uint32_t items = (uint32_t)r.B * (uint32_t)r.T * (uint32_t)parts;      // < 2^31 (host check)
    const bool turns = MODE != kAny || r.pairs > 0, halves = MODE == kHalves || (MODE == kAny && r.pairs > 0 && !r.adjacent);
    const float inv = 1.f / (float)d;
    const int out_size = p.out_dtype == GLA_DT_BF16 ? 2 : 4;

    float dw[2][kEach];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < kEach; ++j) dw[t][j] = 0.f;
    Channel ch[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) ch[j] = Channel(r, c0 + j);

    // the pairs' other channels
    auto others = [&](const float (&v)[kEach], float (&o)[kEach]) __attribute__((always_inline)) {
        if (!halves) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) o[j] = v[j ^ 1];
            return;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_memcpy(__builtin_assume_aligned(&rows[gi][c0], 16), v, sizeof(v));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if constexpr (MODE == kHalves) {
            __builtin_memcpy(o, __builtin_assume_aligned(&rows[gi][ch[0].other()], 16), sizeof(o));
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) o[j] = rows[gi][ch[j].other()];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };

    for (uint32_t item = blockIdx.x * (uint32_t)kWaves + wave; item < items; item += gridDim.x * (uint32_t)kWaves) {
        const uint32_t token = item / (uint32_t)parts;
        const int part = (int)(item - token * (uint32_t)parts);
        const int b = (int)(token / (uint32_t)r.T), n = (int)(token - (uint32_t)b * (uint32_t)r.T);
        float cs[kEach], sn[kEach];      // y[c] = v[c] cs + v[other] sn
        if (turns) {
            for (int pair = lane; pair < r.pairs; pair += 64) {
                int axis = 0;
                while (pair >= r.pairs_end[axis]) ++axis;
                float2 a;
                turn(r, pair, (double)position(r, token, n, axis), &a.x, &a.y);
                angles[wave][pair] = a;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const float2 a = angles[wave][ch[j].pair()];
                cs[j] = MODE != kAny || ch[j].turned() ? a.x : 1.f;
                sn[j] = MODE != kAny || ch[j].turned() ? (ch[j].second() ? a.y : -a.y) : 0.f;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j) cs[j] = 1.f, sn[j] = 0.f;
        }
        // the part's turns: those of the queries, then those of the keys
        const int turns_q = (p.side[0].heads + kRows - 1) / kRows, t0 = part * each, t1 = t0 + each;
        auto one_side = [&](auto side) __attribute__((always_inline)) {
            constexpr int t = decltype(side)::value;
            const QkSide &s = p.side[t];
            const int first = (t ? max(t0 - turns_q, 0) : t0) * kRows, end = min((t ? t1 - turns_q : t1) * kRows, s.heads);
            if (first >= end) return;
            // uniform places of the first row, and each lane's row from there
            const char *x = static_cast<const char *>(s.x) + (b * s.sb + first * s.sh + n * s.st) * (long long)sizeof(E);
            const long long next_x = s.sh * (long long)sizeof(E), mine_x = sub * next_x;
            const long long row = (r.layout == GLA_LAYOUT_BHTD ? ((long long)b * s.heads + first) * r.T + n : (long long)token * s.heads + first) * d;
            const long long next = r.layout == GLA_LAYOUT_BHTD ? (long long)r.T * d : d, mine = sub * next;
            const char *o = BACK ? static_cast<const char *>(s.d_out) + row * (long long)sizeof(E) : nullptr;
            char *out = static_cast<char *>(s.out) + row * out_size;
            float w[kEach], ws[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) w[j] = 1.f;
            if (s.weight != nullptr) load_piece<float>(reinterpret_cast<const char *>(s.weight), c0, d, w);
            if constexpr (!BACK) {       // the weight, through the turning
                others(w, ws);
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    w[j] *= cs[j];
                    ws[j] *= sn[j];
                }
            }
            constexpr int kAhead = 2;
            Raw<E> nx[kAhead], no[BACK ? kAhead : 1];
            auto ask = [&](int i, int h) __attribute__((always_inline)) {
                nx[i] = {};
                if constexpr (BACK) no[i] = {};
                if (h + sub < end) {
                    nx[i] = load_raw<E>(x + mine_x, c0, d);
                    if constexpr (BACK) no[i] = load_raw<E>(o + mine * (long long)sizeof(E), c0, d);
                }
                x += kRows * next_x;
                if constexpr (BACK) o += kRows * next * (long long)sizeof(E);
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (first + i * kRows < end) ask(i, first + i * kRows);
            for (int h0 = first; h0 < end; h0 += kAhead * kRows) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int h = h0 + i * kRows;
                    if (h >= end) continue;
                    float v[kEach], g[kEach], q[kEach];
                    to_floats<E>(nx[i], v);
                    if constexpr (BACK) to_floats<E>(no[i], g);
                    if (h + kAhead * kRows < end) ask(i, h + kAhead * kRows);
                    float ss = 0.f;
#pragma unroll
                    for (int j = 0; j < kEach; ++j) ss = fmaf(v[j], v[j], ss);
                    if constexpr (!BACK) {
                        if (turns) others(v, q);
                        const float rstd = __builtin_amdgcn_rsqf(fmaf(row_sum<LANES>(ss), inv, p.eps));
#pragma unroll
                        for (int j = 0; j < kEach; ++j) {
                            float y = v[j] * w[j];
                            if (turns) y = fmaf(q[j], ws[j], y);
                            v[j] = y * rstd;
                        }
                    } else {
                        if (turns) {
                            others(g, q);
#pragma unroll
                            for (int j = 0; j < kEach; ++j) g[j] = fmaf(q[j], -sn[j], g[j] * cs[j]);
                        }
                        // (lanes without a row add to the weight's sums too: nothing, also where no eps keeps their root from zero)
                        const float root = __builtin_amdgcn_rsqf(fmaf(row_sum<LANES>(ss), inv, p.eps)), rstd = h + sub < end ? root : 0.f;
                        float m = 0.f;
#pragma unroll
                        for (int j = 0; j < kEach; ++j) {
                            v[j] *= rstd;
                            dw[t][j] = fmaf(g[j], v[j], dw[t][j]);
                            g[j] *= w[j];
                            m = fmaf(g[j], v[j], m);
                        }
                        m = row_sum<LANES>(m) * -inv;
#pragma unroll
                        for (int j = 0; j < kEach; ++j) v[j] = rstd * fmaf(v[j], m, g[j]);
                    }
                    if (h + sub < end) store_piece(out + mine * out_size, c0, d, p.out_dtype, v);
                    out += kRows * next * out_size;
                }
            }
        };
        one_side(std::integral_constant<int, 0>{});
        one_side(std::integral_constant<int, 1>{});
    }
    if constexpr (BACK) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (p.side[t].part == nullptr) continue;
            __syncthreads();
            __builtin_memcpy(__builtin_assume_aligned(&rows[gi][c0], 16), dw[t], sizeof(dw[t]));
            __syncthreads();
            for (int c = threadIdx.x; c < d; c += kThreads) {
                float sum = 0.f;
#pragma unroll 8
                for (int k = 0; k < kWaves * kRows; ++k) sum += rows[k][c];
                p.side[t].part[(size_t)blockIdx.x * d + c] = sum;
            }
        }
    }
}

// Adds the work-groups' partial sums: 16 columns and 64 rows at a time.  1024 sums of 128 channels, twice: 5 us
__global__ __launch_bounds__(1024) void qk_sum_kernel(const QkParams p) {
    __shared__ float s[64][17];
    const int c = threadIdx.x & 15, k = threadIdx.x >> 4, col = blockIdx.x * 16 + c, d = p.rope.d;
    const QkSide &t = p.side[blockIdx.y];
    if (t.part == nullptr) return;
    float x = 0.f;
    if (col < d) {
#pragma unroll 8
        for (int i = k; i < p.slots; i += 64) x += t.part[(size_t)i * d + col];
    }
    s[k][c] = x;
    __syncthreads();
    for (int n = 32; n > 0; n /= 2) {
        if (k < n) s[k][c] += s[k + n][c];
        __syncthreads();
    }
    if (k == 0 && col < d) t.dweight[col] = s[0][c];
}

// Work-groups of the backward pass: four a compute unit, each with one partial sum (16380 tokens of 16 + 4 heads 46 us, with 512 or 2048 of them 49)
constexpr int kSlots = 1024;

template <typename E, int LANES, bool BACK>
hipError_t qk(const QkParams &p, hipStream_t stream) {
    constexpr int kRows = 64 / LANES, kWaves = kThreads / 64;
    const int turns = (p.side[0].heads + kRows - 1) / kRows + (p.side[1].heads + kRows - 1) / kRows;
    const long long tokens = (long long)p.rope.B * p.rope.T;
    // turns that share a token's sines and cosines: all, unless that leaves the GPU idle (64 tokens of 16 + 4 heads 4.7 us, with all turns together 6.2; 2048
    // tokens 8.0, in parts 13.2)
    int each = turns;
    while (each > 1 && tokens * ((turns + each - 1) / each) < 2048) each = (each + 1) / 2;
    const int parts = (turns + each - 1) / each;         // (at most 2048 items where there is more than one)
    const long long groups = (tokens * parts + kWaves - 1) / kWaves;
    const RopeParams &r = p.rope;
    bool whole = 2 * r.pairs == LANES * kEach;           // (sections, or their halves, in whole pieces)
    for (int x = 0; x < r.axes; ++x) whole = whole && r.first[x] % kEach == 0 && r.half[x] % (r.adjacent ? 1 : kEach) == 0;
    auto run = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        // forward as many work-groups as the GPU holds (4 x 4095 tokens of 16 + 16 heads of 128 channels 52 us, with one for each four tokens 63; 20000 of
        // 12 + 12 heads of 64 38 and 51)
        static const int held = [] {
            int n = 0;
            return hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, (const void *)qk_kernel<E, LANES, BACK, MODE>, kThreads, 0) == hipSuccess && n > 0 ? 256 * n : 1024;
        }();
        const unsigned grid = BACK ? (unsigned)p.slots : (unsigned)(groups < held ? groups : held);
        hipLaunchKernelGGL((qk_kernel<E, LANES, BACK, MODE>), dim3(grid), dim3(kThreads), 0, stream, p, each, parts);
        return hipGetLastError();
    };
    if (whole) return r.adjacent ? run(std::integral_constant<int, kNeighbours>{}) : run(std::integral_constant<int, kHalves>{});
    return run(std::integral_constant<int, kAny>{});
}
template <bool BACK>
hipError_t qk_of(const QkParams &p, int dtype, hipStream_t stream) {
    auto wide = [&](auto e) {
        using E = decltype(e);
        if (p.rope.d <= 32) return qk<E, 4, BACK>(p, stream);
        if (p.rope.d <= 64) return qk<E, 8, BACK>(p, stream);
        if (p.rope.d <= 128) return qk<E, 16, BACK>(p, stream);
        return qk<E, 32, BACK>(p, stream);
    };
    return dtype == GLA_DT_BF16 ? wide(uint16_t{}) : wide(float{});
}

}  // namespace

int qk_slots(int B, int T) {
    const long long tokens = (long long)B * T;
    return tokens < kSlots ? (int)tokens : kSlots;
}

hipError_t launch_qk_fwd(const QkParams &p, int dtype, hipStream_t stream) { return qk_of<false>(p, dtype, stream); }

hipError_t launch_qk_bwd(const QkParams &p, int dtype, hipStream_t stream) {
    const hipError_t e = qk_of<true>(p, dtype, stream);
    if (e != hipSuccess || (p.side[0].part == nullptr && p.side[1].part == nullptr)) return e;
    hipLaunchKernelGGL(qk_sum_kernel, dim3((unsigned)((p.rope.d + 15) / 16), 2), dim3(1024), 0, stream, p);
    return hipGetLastError();
}

}  // namespace gla
