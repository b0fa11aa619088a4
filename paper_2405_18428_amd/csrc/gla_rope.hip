// Rotary positions with several axes: the channels of a head fall into sections, one for each axis of a token's position (row and column
// of a patch, with the frame in front for video, or whatever the caller counts); pair i of a section of w channels turns by
// position * base^(-2 i / w).
//
// A thread turns four neighbouring pairs of a token, for several heads and for queries and keys, by the same sines and cosines: these
// cost far more than the rotation.  Angles are formed in turns, from a frequency in two 64-bit numbers, and reduced there: in 32 bits a position
// of some ten thousand would be off by 1e-3 of a turn, with one number of 64 one of 2^31 by 1e-7 and more, and a sine's own reduction is not
// needed any more.  Bound by HBM.
#include "gla_ops.h"

namespace gla {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256;

__device__ inline uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
template <typename E>
__device__ inline f32x4 load4(const char *p) {
    if constexpr (sizeof(E) == 2) {
        u32x2 b;
        __builtin_memcpy(&b, p, 8);
        return f32x4{__builtin_bit_cast(float, b[0] << 16), __builtin_bit_cast(float, b[0] & 0xffff0000u),
                     __builtin_bit_cast(float, b[1] << 16), __builtin_bit_cast(float, b[1] & 0xffff0000u)};
    } else {
        f32x4 v;
        __builtin_memcpy(&v, p, 16);
        return v;
    }
}
template <typename E>
__device__ inline void store4(char *p, f32x4 v) {
    if constexpr (sizeof(E) == 2) {
        const u32x2 b = {pack(v[0], v[1]), pack(v[2], v[3])};
        __builtin_memcpy(p, &b, 8);
    } else {
        __builtin_memcpy(p, &v, 16);
    }
}
template <typename E>
__device__ inline float load1(const char *p) {
    if constexpr (sizeof(E) == 2) return bf16_bits_to_float(*reinterpret_cast<const uint16_t *>(p));
    else return *reinterpret_cast<const float *>(p);
}
template <typename E>
__device__ inline void store1(char *p, float v) {
    if constexpr (sizeof(E) == 2) *reinterpret_cast<uint16_t *>(p) = (uint16_t)pack(v, 0.f);
    else *reinterpret_cast<float *>(p) = v;
}

__device__ inline int position(const RopeParams &p, long long token, int n, int axis) {
    if (p.positions != nullptr) return p.positions[token * p.axes + axis];
    if (p.axes == 1) return n;
    const int cell = p.grid_h * p.grid_w, f = n / cell, r = n - f * cell;
    const int which = p.axes == 2 ? axis + 1 : axis;
    return which == 0 ? f : which == 1 ? r / p.grid_w : r % p.grid_w;
}

// VP pairs a thread: 4 where every section has a multiple of 4 pairs, else 1.  Items behind the pairs are the channels behind the last
// section, copied VP at a time.
template <typename E, int VP>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeParams p) {
    const int tail = p.d - 2 * p.pairs;
    const uint32_t items = (uint32_t)(p.pairs / VP + (tail + VP - 1) / VP);
    const uint32_t id = blockIdx.x * (uint32_t)kThreads + threadIdx.x;      // < 2^31 (host check)
    const uint32_t token_ = id / items;                  // over the batches
    if (token_ >= (uint32_t)p.B * (uint32_t)p.T) return;
    const int item = (int)(id - token_ * items);
    const int b = (int)(token_ / (uint32_t)p.T), n = (int)(token_ - (uint32_t)b * (uint32_t)p.T);
    const long long token = token_;
    const int h0 = blockIdx.y * p.heads_each, h1 = min(h0 + p.heads_each, p.H);
    const long long head = (p.layout == GLA_LAYOUT_BHTD ? (long long)p.T : 1LL) * p.d * (int)sizeof(E);
    const long long row = (p.layout == GLA_LAYOUT_BHTD ? (long long)b * p.H * p.T + n : token * p.H) * p.d * (int)sizeof(E);
    const bool turned = item < p.pairs / VP;

    if (!turned) {
        const int c0 = 2 * p.pairs + (item - p.pairs / VP) * VP, c1 = min(c0 + VP, p.d);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (p.x[t] == nullptr || p.x[t] == p.y[t]) continue;
            for (int h = h0; h < h1; ++h)
                for (int c = c0; c < c1; ++c) {
                    const long long at = row + h * head + c * (int)sizeof(E);
                    store1<E>(static_cast<char *>(p.y[t]) + at, load1<E>(static_cast<const char *>(p.x[t]) + at));
                }
        }
        return;
    }
    const int pair = item * VP;
    int axis = 0;
    while (axis + 1 < p.axes && pair >= p.pairs_end[axis]) ++axis;
    const int i = pair - (p.pairs_end[axis] - p.half[axis]);
    const double pos = (double)position(p, token, n, axis);
    float cs[VP], sn[VP];
#pragma unroll
    for (int j = 0; j < VP; ++j) {
        const double whole = pos * p.turns[pair + j];                    // exact
        const double turns = __builtin_fma(pos, p.rest[pair + j], whole - __builtin_rint(whole));
        const float f = (float)(turns - __builtin_rint(turns));          // -1/2 .. 1/2
        sincospif(2.f * f, &sn[j], &cs[j]);
        if (p.inverse) sn[j] = -sn[j];
    }
    const int c0 = p.first[axis] + (p.adjacent ? 2 * i : i), c1 = p.adjacent ? c0 + VP : c0 + p.half[axis];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (p.x[t] == nullptr) continue;
        const char *x = static_cast<const char *>(p.x[t]) + row;
        char *y = static_cast<char *>(p.y[t]) + row;
        const long long a0 = c0 * (int)sizeof(E), a1 = c1 * (int)sizeof(E);
        if constexpr (VP == 4) {
            // two heads at once, whose loads come before the first store (a video's 46665 tokens of 16 heads of 128: 165 us, one at a time 176, four 171)
            constexpr int kAtOnce = 2;
            for (int h = h0; h < h1; h += kAtOnce) {
                f32x4 u[kAtOnce], v[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (h + k >= h1) continue;
                    u[k] = load4<E>(x + (h + k) * head + a0);
                    v[k] = load4<E>(x + (h + k) * head + a1);
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    if (h + k >= h1) continue;
                    f32x4 s, w;
                    if (p.adjacent) {
                        s = f32x4{u[k][0] * cs[0] - u[k][1] * sn[0], u[k][1] * cs[0] + u[k][0] * sn[0], u[k][2] * cs[1] - u[k][3] * sn[1],
                                  u[k][3] * cs[1] + u[k][2] * sn[1]};
                        w = f32x4{v[k][0] * cs[2] - v[k][1] * sn[2], v[k][1] * cs[2] + v[k][0] * sn[2], v[k][2] * cs[3] - v[k][3] * sn[3],
                                  v[k][3] * cs[3] + v[k][2] * sn[3]};
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            s[j] = u[k][j] * cs[j] - v[k][j] * sn[j];
                            w[j] = v[k][j] * cs[j] + u[k][j] * sn[j];
                        }
                    }
                    store4<E>(y + (h + k) * head + a0, s);
                    store4<E>(y + (h + k) * head + a1, w);
                }
            }
        } else {
            for (int h = h0; h < h1; ++h) {
                const float u = load1<E>(x + h * head + a0), v = load1<E>(x + h * head + a1);
                store1<E>(y + h * head + a0, u * cs[0] - v * sn[0]);
                store1<E>(y + h * head + a1, v * cs[0] + u * sn[0]);
            }
        }
    }
}

template <typename E, int VP>
hipError_t rope(RopeParams p, hipStream_t stream) {
    const long long items = p.pairs / VP + (p.d - 2 * p.pairs + VP - 1) / VP;
    const long long groups = ((long long)p.B * p.T * items + kThreads - 1) / kThreads;
    // heads a thread: as many as leave the GPU a few work-groups a compute unit
    p.heads_each = p.H;
    while (p.heads_each > 1 && groups * ((p.H + p.heads_each - 1) / p.heads_each) < 2048) p.heads_each = (p.heads_each + 1) / 2;
    // (the second dimension of a grid ends at 65535)
    if ((p.H + p.heads_each - 1) / p.heads_each > 65535) p.heads_each = (p.H + 65534) / 65535;
    hipLaunchKernelGGL((rope_kernel<E, VP>), dim3((unsigned)groups, (unsigned)((p.H + p.heads_each - 1) / p.heads_each)), dim3(kThreads), 0,
                       stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeParams &p, int dtype, hipStream_t stream) {
    bool four = true;
    for (int a = 0; a < p.axes; ++a) four = four && p.half[a] % 4 == 0;
    if (dtype == GLA_DT_BF16) return four ? rope<uint16_t, 4>(p, stream) : rope<uint16_t, 1>(p, stream);
    return four ? rope<float, 4>(p, stream) : rope<float, 1>(p, stream);
}

}  // namespace gla
