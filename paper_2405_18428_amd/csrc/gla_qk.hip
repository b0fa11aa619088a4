// Norm of queries and keys with the rotation behind it, in one pass over each row:
//   n = x r,  r = (mean(x^2) + eps)^-1/2,  y = R (n w),
// R turning the pairs of channels by the token's angles as in gla_rope.hip; and backward, with dy' = R^-1 dy and dn = dy' w:
//   dx = r (dn - n mean(dn n)),   dw = sum over rows of dy' n.
//
// 4 to 32 lanes hold a row, 8 channels each; they take one token, form the sines and cosines of its angles once and go through some
// of its heads, queries and keys alike, with the next row on its way.  A pair of neighbouring channels lies in one lane; the other channel of a
// pair of halves is fetched through LDS, where a row's lanes, which are in one wave, leave their values.  Sums for dw stay in registers, are
// added over a work-group and go to memory as one partial sum a work-group, which a second kernel adds in one order.  Bound by HBM.
#include "gla_qk.h"
#include "gla_rope_util.h"
#include "gla_rows.h"

namespace gla {
namespace {

constexpr int kThreads = 256;

template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
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

template <typename E, int LANES, bool BACK>
__global__ __launch_bounds__(kThreads) void qk_kernel(const QkParams p, int each, int parts) {
    constexpr int kGroups = kThreads / LANES, kWidth = LANES * kEach;
    __shared__ __attribute__((aligned(16))) float rows[kGroups][kWidth];
    const RopeParams &r = p.rope;
    const int gi = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int c0 = lane * kEach, d = r.d;
    const int heads = p.side[0].heads + p.side[1].heads;
    const uint32_t items = (uint32_t)r.B * (uint32_t)r.T * (uint32_t)parts;      // < 2^31 (host check)
    const bool halves = r.pairs > 0 && !r.adjacent;
    const float inv = 1.f / (float)d;
    const int out_size = p.out_dtype == GLA_DT_BF16 ? 2 : 4;

    float w[2][kEach], dw[2][kEach];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) w[t][j] = 1.f, dw[t][j] = 0.f;
        if (p.side[t].weight != nullptr) load_piece<float>(reinterpret_cast<const char *>(p.side[t].weight), c0, d, w[t]);
    }
    Channel ch[kEach];
    float cs[kEach], sn[kEach];         // y[c] = v[c] cs + v[other] sn
#pragma unroll
    for (int j = 0; j < kEach; ++j) ch[j] = Channel(r, c0 + j);
    // halves: the others are eight in a row that begin at a multiple of 4
    bool together = ch[0].other() % 4 == 0;
#pragma unroll
    for (int j = 1; j < kEach; ++j) together = together && ch[j].other() == ch[0].other() + j;

    auto rotate = [&](float (&v)[kEach], float sign) __attribute__((always_inline)) {
        if (r.pairs == 0) return;
        float o[kEach];
        if (!halves) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) o[j] = v[j ^ 1];
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_memcpy(__builtin_assume_aligned(&rows[gi][c0], 16), v, sizeof(v));
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (together) {
                __builtin_memcpy(o, __builtin_assume_aligned(&rows[gi][ch[0].other()], 16), sizeof(o));
            } else {
#pragma unroll
                for (int j = 0; j < kEach; ++j) o[j] = rows[gi][ch[j].other()];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = fmaf(o[j], sign * sn[j], v[j] * cs[j]);
    };

    for (uint32_t item = blockIdx.x * (uint32_t)kGroups + gi; item < items; item += gridDim.x * (uint32_t)kGroups) {
        const uint32_t token = item / (uint32_t)parts;
        const int part = (int)(item - token * (uint32_t)parts);
        const int b = (int)(token / (uint32_t)r.T), n = (int)(token - (uint32_t)b * (uint32_t)r.T);
        const int h0 = part * each, h1 = min(h0 + each, heads);
        if (r.pairs > 0) {
            // neighbouring channels of a pair share an angle
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                float c = 1.f, s = 0.f;
                if (r.adjacent && (j & 1)) {
                    c = cs[j - 1];
                    s = -sn[j - 1];
                } else if (ch[j].turned()) {
                    turn(r, ch[j].pair(), (double)position(r, token, n, ch[j].axis()), &c, &s);
                    if (!ch[j].second()) s = -s;
                }
                cs[j] = c;
                sn[j] = s;
            }
        }
        Raw<E> nx, no;
        auto ask = [&](int h) __attribute__((always_inline)) {
            const int t = h >= p.side[0].heads;
            const QkSide &s = p.side[t];
            const int head = h - (t ? p.side[0].heads : 0);
            nx = load_raw<E>(static_cast<const char *>(s.x) + (b * s.sb + head * s.sh + n * s.st) * (long long)sizeof(E), c0, d);
            if constexpr (BACK) {
                const long long row = r.layout == GLA_LAYOUT_BHTD ? ((long long)b * s.heads + head) * r.T + n : (long long)token * s.heads + head;
                no = load_raw<E>(static_cast<const char *>(s.d_out) + row * d * (long long)sizeof(E), c0, d);
            }
        };
        ask(h0);
        for (int h = h0; h < h1; ++h) {
            const int t = h >= p.side[0].heads;
            const QkSide &s = p.side[t];
            const int head = h - (t ? p.side[0].heads : 0);
            const long long row = r.layout == GLA_LAYOUT_BHTD ? ((long long)b * s.heads + head) * r.T + n : (long long)token * s.heads + head;
            float x[kEach], o[kEach];
            to_floats<E>(nx, x);
            if constexpr (BACK) to_floats<E>(no, o);
            if (h + 1 < h1) ask(h + 1);
            float ss = 0.f;
#pragma unroll
            for (int j = 0; j < kEach; ++j) ss = fmaf(x[j], x[j], ss);
            const float rstd = 1.f / __builtin_sqrtf(fmaf(row_sum<LANES>(ss), inv, p.eps));
            char *out = static_cast<char *>(s.out) + row * d * out_size;
            if constexpr (!BACK) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) x[j] *= rstd * (t ? w[1][j] : w[0][j]);
                rotate(x, 1.f);
                store_piece(out, c0, d, p.out_dtype, x);
            } else {
                rotate(o, -1.f);
                float m = 0.f;
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const float nn = x[j] * rstd, g = o[j] * nn;
                    dw[0][j] += t ? 0.f : g;
                    dw[1][j] += t ? g : 0.f;
                    const float dn = o[j] * (t ? w[1][j] : w[0][j]);
                    m = fmaf(dn, nn, m);
                    x[j] = nn;
                    o[j] = dn;
                }
                m = row_sum<LANES>(m) * inv;
#pragma unroll
                for (int j = 0; j < kEach; ++j) x[j] = rstd * (o[j] - x[j] * m);
                store_piece(out, c0, d, p.out_dtype, x);
            }
        }
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
                for (int k = 0; k < kGroups; ++k) sum += rows[k][c];
                p.side[t].part[(size_t)blockIdx.x * d + c] = sum;
            }
        }
    }
}

// Adds the work-groups' partial sums: 16 columns and 64 rows at a time
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

constexpr int kSlots = 1024;            // work-groups of the backward pass: four a compute unit, each with one partial sum

template <typename E, int LANES, bool BACK>
hipError_t qk(const QkParams &p, hipStream_t stream) {
    constexpr int kGroups = kThreads / LANES;
    const int heads = p.side[0].heads + p.side[1].heads;
    const long long tokens = (long long)p.rope.B * p.rope.T;
    // heads that share a token's sines and cosines: all, unless that leaves the GPU idle
    int each = heads;
    while (each > 1 && tokens * ((heads + each - 1) / each) < 2048LL * kGroups) each = (each + 1) / 2;
    // (items in 31 bits)
    while (each < heads && tokens * ((heads + each - 1) / each) >= (1LL << 31)) each *= 2;
    const int parts = (heads + each - 1) / each;
    const long long groups = (tokens * parts + kGroups - 1) / kGroups;
    const unsigned grid = BACK ? (unsigned)p.slots : (unsigned)(groups < (1 << 23) ? groups : 1 << 23);
    hipLaunchKernelGGL((qk_kernel<E, LANES, BACK>), dim3(grid), dim3(kThreads), 0, stream, p, each, parts);
    return hipGetLastError();
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
    // (a work-group has 8 to 64 rows at a time, and at least one token's heads)
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
