// Layer norm over the channels of each row, y = (x - mean) / sqrt(var + eps) * weight + bias, with the output gate of the mixer behind it
// if r is given, y * r sigmoid(r) (Eq. (attn_gla) rows 4-5 of the DiG paper), and both backward:
//   n = (x - mean) rstd,  dy = dO r sigmoid(r) (or dO),  dn = dy weight,
//   dx = rstd (dn - mean(dn) - n mean(dn n)),   dr = dO y sigmoid(r) (1 + r (1 - sigmoid(r))),
//   dweight = sum over rows of dy n,   dbias = sum over rows of dy.
// A row is held in registers by a group of lanes (4 to 1024 by its width), so it is read once; mean and variance are taken in two
// steps from these registers, and the backward pass takes them again instead of reading them.  Each group stays with one head, whose weights
// it holds, and walks the head's rows, the next of which is on its way while it works on one; the sums for dweight and dbias stay in its
// registers, are added over the groups of a work-group where these share a head, and go to memory as one partial sum a slot, which a
// second kernel adds in one order.  Bound by HBM.
#include "gla_ops.h"
#include "gla_rows.h"

namespace gla {
namespace {

// Sum over the LANES lanes of a group, in every lane.  Groups wider than a wave are the whole work-group and go through LDS: each of a row's
// sums has its own place there, so that one barrier a sum does (a place is written again behind the barriers of the others).
template <int LANES, int SUMS>
__device__ __forceinline__ void group_sum(float (&v)[SUMS], float *lds) {
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int d = 1; d < (LANES < 64 ? LANES : 64); d *= 2) v[s] += __shfl_xor(v[s], d);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int s = 0; s < SUMS; ++s) lds[s * kWaves + w] = v[s];
        __syncthreads();
#pragma unroll
        for (int s = 0; s < SUMS; ++s) {
            v[s] = 0.f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) v[s] += lds[s * kWaves + i];
        }
    }
}

// Which rows a group takes: head h, rows number first, first + step, ... of the head's B * T
struct Walk {
    int h, slot;
    uint32_t first, step;
};
// All groups of a work-group walk rows of one head
__host__ __device__ inline bool one_head(const NormParams &p) { return p.layout == GLA_LAYOUT_BHTD || p.H == 1; }
__host__ __device__ inline int partial_rows(const NormParams &p, int groups) { return one_head(p) ? p.slots / groups : p.slots; }
// Neighbouring groups take rows that are neighbours in memory: of one head where a head's rows lie together, of neighbouring heads where a
// token's heads do
__device__ __forceinline__ Walk walk_of(const NormParams &p, int groups, int gi) {
    Walk w;
    if (one_head(p)) {
        const int per_head = p.slots / groups;                   // work-groups of a head
        w.h = blockIdx.x / per_head;
        w.slot = (blockIdx.x - w.h * per_head) * groups + gi;
    } else {
        const uint32_t l = blockIdx.x * (uint32_t)groups + gi;
        w.slot = (int)(l / (uint32_t)p.H);
        w.h = (int)(l - (uint32_t)w.slot * p.H);
    }
    w.first = (uint32_t)w.slot;
    w.step = (uint32_t)p.slots;
    return w;
}
__device__ __forceinline__ long long row_of(const NormParams &p, int h, uint32_t i) {
    if (p.layout != GLA_LAYOUT_BHTD) return (long long)i * p.H + h;
    const uint32_t b = i / (uint32_t)p.T;
    return ((long long)b * p.H + h) * p.T + (i - b * (uint32_t)p.T);
}

template <int LANES>
struct Shape {
    static constexpr int kThreads = LANES > 256 ? LANES : 256, kGroups = kThreads / LANES;
};

// 1 / (1 + exp(-r)); the reciprocal is off by one unit in the last place
__device__ __forceinline__ float sigmoid(float r) { return __builtin_amdgcn_rcpf(1.f + __expf(-r)); }

template <typename E, int LANES, int NP, bool GATED, bool BACK>
__global__ __launch_bounds__(Shape<LANES>::kThreads) void norm_kernel(const NormParams p) {
    constexpr int kGroups = Shape<LANES>::kGroups, kWaves = LANES > 64 ? LANES / 64 : 1, kWidth = LANES * NP * kEach;
    __shared__ float lds[BACK && kGroups > 1 ? kGroups * kWidth : 4 * kWaves];
    const int gi = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const Walk wk = walk_of(p, kGroups, gi);
    const uint32_t rows = (uint32_t)p.B * (uint32_t)p.T;         // < 2^31 (host check)
    const int D = p.D;
    const float inv = 1.f / (float)D;
    const int out_size = p.out_dtype == GLA_DT_BF16 ? 2 : 4;
    const bool mine = wk.slot < p.slots && wk.h < p.H;

    float w[NP][kEach], b[NP][kEach], dw[BACK ? NP : 1][kEach], db[BACK ? NP : 1][kEach];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c = (i * LANES + lane) * kEach;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            w[i][j] = 1.f;
            b[i][j] = 0.f;
            if constexpr (BACK) dw[i][j] = db[i][j] = 0.f;
        }
        if (mine && p.weight != nullptr) load_piece<float>(reinterpret_cast<const char *>(p.weight + (size_t)wk.h * D), c, D, w[i]);
        if (mine && p.bias != nullptr) load_piece<float>(reinterpret_cast<const char *>(p.bias + (size_t)wk.h * D), c, D, b[i]);
    }
    Raw<E> nx[NP], nr[GATED ? NP : 1], no[BACK ? NP : 1];
    auto ask = [&](uint32_t i0) __attribute__((always_inline)) {
        const long long at = row_of(p, wk.h, i0) * D * (int)sizeof(E);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c = (i * LANES + lane) * kEach;
            nx[i] = load_raw<E>(static_cast<const char *>(p.x) + at, c, D);
            if constexpr (GATED) nr[i] = load_raw<E>(static_cast<const char *>(p.r_pre) + at, c, D);
            if constexpr (BACK) no[i] = load_raw<E>(static_cast<const char *>(p.d_out) + at, c, D);
        }
    };
    if (mine && wk.first < rows) ask(wk.first);
    // (groups of one wave or less end on their own; the wider ones are the work-group)
    for (uint32_t i0 = wk.first; mine && i0 < rows; i0 += wk.step) {
        const long long row = row_of(p, wk.h, i0);
        float x[NP][kEach], r[GATED ? NP : 1][kEach], o[BACK ? NP : 1][kEach];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            to_floats<E>(nx[i], x[i]);
            if constexpr (GATED) to_floats<E>(nr[i], r[i]);
            if constexpr (BACK) to_floats<E>(no[i], o[i]);
        }
        if (i0 + wk.step < rows) ask(i0 + wk.step);
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < kEach; ++j) s[0] += x[i][j];
        group_sum<LANES, 1>(s, lds);
        const float mean = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                x[i][j] = (i * LANES + lane) * kEach + j < D ? x[i][j] - mean : 0.f;
                s[0] = fmaf(x[i][j], x[i][j], s[0]);
            }
        group_sum<LANES, 1>(s, lds + kWaves);
        const float rstd = 1.f / __builtin_sqrtf(fmaf(s[0], inv, p.eps));
        if constexpr (!BACK) {
            char *po = static_cast<char *>(p.out) + row * D * out_size;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float y[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    y[j] = fmaf(x[i][j] * rstd, w[i][j], b[i][j]);
                    if constexpr (GATED) y[j] *= r[i][j] * sigmoid(r[i][j]);
                }
                store_piece(po, (i * LANES + lane) * kEach, D, p.out_dtype, y);
            }
        } else {
            char *pdx = static_cast<char *>(p.dx) + row * D * out_size;
            char *pdr = static_cast<char *>(p.dr) + row * D * out_size;
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float dr[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) {
                    const float n = x[i][j] * rstd;
                    float dy = o[i][j];
                    if constexpr (GATED) {
                        const float sg = sigmoid(r[i][j]), gate = r[i][j] * sg;
                        dr[j] = o[i][j] * fmaf(n, w[i][j], b[i][j]) * fmaf(gate, 1.f - sg, sg);
                        dy *= gate;
                    }
                    dw[i][j] = fmaf(dy, n, dw[i][j]);
                    db[i][j] += dy;
                    const float dn = dy * w[i][j];
                    m[0] += dn;
                    m[1] = fmaf(dn, n, m[1]);
                    x[i][j] = n;
                    o[i][j] = dn;
                }
                if constexpr (GATED) store_piece(pdr, (i * LANES + lane) * kEach, D, p.out_dtype, dr);
            }
            group_sum<LANES, 2>(m, lds + 2 * kWaves);
            const float m0 = m[0] * inv, m1 = m[1] * inv;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                float dx[kEach];
#pragma unroll
                for (int j = 0; j < kEach; ++j) dx[j] = rstd * (o[i][j] - m0 - x[i][j] * m1);
                store_piece(pdx, (i * LANES + lane) * kEach, D, p.out_dtype, dx);
            }
        }
    }
    if constexpr (BACK) {
        if (p.part == nullptr) return;
        const bool shared = kGroups > 1 && one_head(p);          // the work-group's slots become one
        const size_t second = (size_t)partial_rows(p, kGroups) * p.H * D;
        if (shared) {
            float *part = p.part + ((size_t)(wk.slot / kGroups) * p.H + wk.h) * D;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NP; ++i)
#pragma unroll
                    for (int j = 0; j < kEach; ++j) lds[gi * kWidth + (i * LANES + lane) * kEach + j] = which ? db[i][j] : dw[i][j];
                __syncthreads();
                for (int c = threadIdx.x; c < D; c += Shape<LANES>::kThreads) {
                    float sum = 0.f;
#pragma unroll
                    for (int k = 0; k < kGroups; ++k) sum += lds[k * kWidth + c];
                    part[which * second + c] = sum;
                }
            }
        } else if (mine) {
            float *part = p.part + ((size_t)wk.slot * p.H + wk.h) * D;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c = (i * LANES + lane) * kEach;
                store_piece(reinterpret_cast<char *>(part), c, D, GLA_DT_F32, dw[i]);
                store_piece(reinterpret_cast<char *>(part + second), c, D, GLA_DT_F32, db[i]);
            }
        }
    }
}

// Adds the partial sums: 16 columns and 64 rows at a time a work-group, which goes on to further columns where there are more than work-groups
// (of 2^32 threads, a launch's limit, 2^26 columns would need them all)
constexpr int kMostSums = 1 << 20;
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float *part, float *dweight, float *dbias, int rows, int cols) {
    __shared__ float s[64][17];
    const int c = threadIdx.x & 15, k = threadIdx.x >> 4;
    const float *src = part + (blockIdx.y ? (size_t)rows * cols : 0);
    for (int col0 = blockIdx.x * 16; col0 < cols; col0 += gridDim.x * 16) {
        const int col = col0 + c;
        float x = 0.f;
        if (col < cols) {
#pragma unroll 8
            for (int i = k; i < rows; i += 64) x += src[(size_t)i * cols + col];
        }
        s[k][c] = x;
        __syncthreads();
        for (int d = 32; d > 0; d /= 2) {
            if (k < d) s[k][c] += s[k + d][c];
            __syncthreads();
        }
        if (k == 0 && col < cols) (blockIdx.y ? dbias : dweight)[col] = s[0][c];
    }
}

// lanes of a row's group: as few as hold it (16 for rows of 64 took 37 us forward where 8 take 21, 4 x 16 x 4096 of them).  Rows of 65 to 96,
// nine pieces for 72, leave lanes of 16 idle: forward four lanes of three take them in 19 us instead of 22 (2 x 16 x 4096), backward
// they take as long in head order and 67 us instead of 55 in token order, both directions together, where each group's sums go to memory.
int lanes_of(int D, bool back) {
    if (!back && D > 64 && D <= 96) return 4;
    return D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : D <= 1536 ? 64 : D <= 2048 ? 256 : D <= 4096 ? 512 : 1024;
}
int groups_of(int D, bool back) { return lanes_of(D, back) >= 256 ? 1 : 256 / lanes_of(D, back); }

// Rows of each head are dealt to `slots` groups: `groups` in all if there are so many rows, `least` rows each; a multiple of the groups of a
// work-group where a work-group stays with one head
int slots_for(const NormParams &p, int least, long long groups, bool back) {
    const long long rows = (long long)p.B * p.T, most = (rows + least - 1) / least, of_group = groups_of(p.D, back);
    long long slots = groups / p.H;
    if (slots > most) slots = most;
    if (slots < 1) slots = 1;
    if (one_head(p)) slots = (slots + of_group - 1) / of_group * of_group;
    return (int)slots;
}

template <typename E, int LANES, int NP, bool BACK>
hipError_t norm(const NormParams &p, hipStream_t stream) {
    constexpr int kThreads = Shape<LANES>::kThreads, kGroups = Shape<LANES>::kGroups;
    const long long groups = (long long)p.slots * p.H;
    const dim3 grid((unsigned)((groups + kGroups - 1) / kGroups));
    if (p.r_pre != nullptr) hipLaunchKernelGGL((norm_kernel<E, LANES, NP, true, BACK>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((norm_kernel<E, LANES, NP, false, BACK>), grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

template <typename E, bool BACK>
hipError_t norm_of_width(const NormParams &p, hipStream_t stream) {
    if (p.D <= 32) return norm<E, 4, 1, BACK>(p, stream);
    if (p.D <= 64) return norm<E, 8, 1, BACK>(p, stream);
    if constexpr (!BACK) {
        if (p.D <= 96) return norm<E, 4, 3, BACK>(p, stream);
    }
    if (p.D <= 128) return norm<E, 16, 1, BACK>(p, stream);
    if (p.D <= 512) return norm<E, 64, 1, BACK>(p, stream);
    if (p.D <= 1024) return norm<E, 64, 2, BACK>(p, stream);
    if (p.D <= 1536) return norm<E, 64, 3, BACK>(p, stream);
    if (p.D <= 2048) return norm<E, 256, 1, BACK>(p, stream);
    if (p.D <= 4096) return norm<E, 512, 1, BACK>(p, stream);
    return norm<E, 1024, 1, BACK>(p, stream);
}

}  // namespace

int norm_slots(int B, int H, int T, int D, int layout) {
    NormParams p = {};
    p.B = B;
    p.H = H;
    p.T = T;
    p.D = D;
    p.layout = layout;
    // 4096 waves (2048 where a lane holds two pieces of a row and more): with twice as many 16384 rows of 1152 took 63 us both ways, 57 with
    // these, 2000 of 8192 69 and 58; with half as many 16384 rows of 384 took 33, 29 with these
    return slots_for(p, 1, (long long)(D > 512 && D <= 1536 ? 2048 : 4096) * 64 / lanes_of(D, true), true);
}

int norm_partial_rows(int B, int H, int T, int D, int layout) {
    NormParams p = {};
    p.H = H;
    p.layout = layout;
    p.slots = norm_slots(B, H, T, D, layout);
    return partial_rows(p, groups_of(D, true));
}

hipError_t launch_norm_fwd(const NormParams &p0, int dtype, hipStream_t stream) {
    NormParams p = p0;
    // two rows a group at least, if that leaves a thousand groups: it holds the weights (4096 rows of 1152: 9.9 us with one, 8.7 with two)
    p.slots = slots_for(p, (long long)p.B * p.T * p.H < 2048 ? 1 : 2, 2048LL * groups_of(p.D, false), false);
    return dtype == GLA_DT_BF16 ? norm_of_width<uint16_t, false>(p, stream) : norm_of_width<float, false>(p, stream);
}

hipError_t launch_norm_bwd(const NormParams &p0, int dtype, float *dweight, float *dbias, hipStream_t stream) {
    NormParams p = p0;
    const hipError_t e = dtype == GLA_DT_BF16 ? norm_of_width<uint16_t, true>(p, stream) : norm_of_width<float, true>(p, stream);
    if (e != hipSuccess || dweight == nullptr) return e;
    const int cols = p.H * p.D, tiles = (cols + 15) / 16;
    hipLaunchKernelGGL(norm_sum_kernel, dim3((unsigned)(tiles < kMostSums ? tiles : kMostSums), 2), dim3(1024), 0, stream, p.part, dweight, dbias,
                       partial_rows(p, groups_of(p.D, true)), cols);
    return hipGetLastError();
}

}  // namespace gla
