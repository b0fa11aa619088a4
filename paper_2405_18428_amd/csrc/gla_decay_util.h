// Device side of the walks of gla_decay.h: tiles of rows in LDS, the operands that the matrix instructions take from them, and one
// chunk of the recurrence.
//
// Four waves walk one state [m, n] (padded to M, N): wave w holds all rows of columns w * N/4 .. + N/4 - 1 in registers, as
// accumulators of 16 x 16 products with lane = column, and works on these columns of the outputs.  A chunk is
//   (1) P^T = y x^T of the lower triangle, 16 columns a wave, times exp(b_i - b_j), to LDS; and out^T = S^T x^T, all in-wave
//   (2) out^T = exp(b_i) out^T + z^T P^T, and S = exp(b_last) S + y^T (exp(b_last - b_j) z).
// Everything is formed transposed, so that the accumulators of one product are an operand of the next as they stand: an operand
// is eight (bf16) or four (fp32) values of the contracted index in a lane, and which index stands where does not matter as long as
// both operands agree.  The state's rows are ordered (state_row) so that x's operands are 16 contiguous bytes of a row.
// bf16 calls split what is not bf16 by itself (the state, P, the decayed z) into two bf16 numbers, head and remainder: what is
// lost is 2^-18 of each, so states and gate gradients, which are given in 32 bits, hold about 2e-6 where one bf16 would leave 2e-3.
// fp32 calls run on the fp32 matrix instructions.
#pragma once
#include "gla_decay.h"
#include "gla_mfma_util.h"

namespace gla {
namespace {

constexpr int kPadBytes = 16;        // behind each row of a tile: rows 4 banks apart, 16 of them cover all 64

template <typename E> struct Elem;
template <> struct Elem<uint16_t> {
    static constexpr int kChunk = 64;            // steps
    static constexpr int kDeep = 32;             // contracted values of an operand over the wave
    static constexpr int kParts = 2;             // head and remainder
};
template <> struct Elem<float> {
    static constexpr int kChunk = 32;
    static constexpr int kDeep = 16;
    static constexpr int kParts = 1;
};

// 16 bytes of an operand; products of operands
template <typename E>
__device__ inline f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (sizeof(E) == 2) {
        return mfma(a, b, c);
    } else {
        const f32x4 af = __builtin_bit_cast(f32x4, a), bf = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(af[r], bf[r], c, 0, 0, 0);
        return c;
    }
}

// State row of element r of lane group g in the 16-row tile t (see the head comment): for bf16 two tiles share 32 rows, and
// group g's eight are contiguous.
template <typename E>
__device__ inline int state_row(int t, int g, int r) {
    if constexpr (sizeof(E) == 2) return (t >> 1) * 32 + g * 8 + (t & 1) * 4 + r;
    else return t * 16 + g * 4 + r;
}

// A tile of C rows of W elements in LDS
template <typename E, int W>
struct Tile {
    static constexpr int C = Elem<E>::kChunk;
    static constexpr int kRow = W * (int)sizeof(E) + kPadBytes;      // bytes
    static constexpr int kBytes = C * kRow;
    char *p;
    // 16 bytes of row `row`: the operand of contraction step ks whose other index is the row
    __device__ __forceinline__ u32x4 along(int row, int ks, int g) const {
        return *reinterpret_cast<const u32x4 *>(p + row * kRow + (ks * 4 + g) * 16);
    }
    // the operand that contracts over rows: step jk of kDeep rows, other index = the lane's column `lm` of 16.  With PERM the
    // columns of state tile t (state_row), else columns 16 t and on.
    template <bool PERM>
    __device__ __forceinline__ u32x4 across(int jk, int t, int lm, int g) const {
        if constexpr (sizeof(E) == 2) {
            const int col = PERM ? state_row<E>(t, lm & 3, 0) : t * 16 + 4 * (lm & 3);
            const char *a = p + (jk * 32 + g * 4 + (lm >> 2)) * kRow + col * 2;
            const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(a));
            const u32x2 hi = lds_read_tr(reinterpret_cast<const uint16_t *>(a + 16 * kRow));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const char *a = p + (jk * 16 + g * 4) * kRow + (t * 16 + lm) * 4;
            u32x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const uint32_t *>(a + r * kRow);
            return v;
        }
    }
};

// Rows of a [.., d] tensor of one (batch, head): 64-bit offsets, so any length does
struct Rows {
    const char *base;
    long long step;                     // bytes between tokens
    int d;
};
template <typename E>
__device__ inline Rows rows_of(const DecayCall &c, const void *t, int bh, int d, int size = (int)sizeof(E)) {
    const int b = bh / c.H, h = bh - b * c.H;
    Rows r;
    r.d = d;
    if (c.layout == GLA_LAYOUT_BHTD) {
        r.step = (long long)d * size;
        r.base = static_cast<const char *>(t) + (long long)bh * c.T * r.step;
    } else {
        r.step = (long long)c.H * d * size;
        r.base = static_cast<const char *>(t) + (long long)b * c.T * r.step + (long long)h * d * size;
    }
    return r;
}

__device__ inline u32x4 load16(const char *p) {          // any alignment
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// The pieces (16 bytes) of a tile that one of THREADS threads brings: issue() asks for them, commit() puts them into the tile once
// the one before has been used.  Rows from `count` on and columns from d on are zeros and are not read.
template <typename E, int W, int THREADS>
struct Pieces {
    static constexpr int kPerRow = W * (int)sizeof(E) / 16, kEach = 16 / (int)sizeof(E);
    static constexpr int kCount = Tile<E, W>::C * kPerRow / THREADS;
    static_assert(Tile<E, W>::C * kPerRow % THREADS == 0, "whole pieces a thread");
    u32x4 v[kCount];
    template <typename TokenOf>
    __device__ __forceinline__ void issue(const Rows &r, int tid, int count, TokenOf token) {
        const int col = tid % kPerRow * kEach;           // (THREADS is a multiple of kPerRow)
        // the last piece of a row of odd length is read as the row's last 16 bytes and shifted in commit()
        const int at = col + kEach <= r.d ? col : r.d - kEach;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int row = (i * THREADS + tid) / kPerRow;
            u32x4 x = {0u, 0u, 0u, 0u};
            if (row < count && col < r.d) {
                const char *p = r.base + token(row) * r.step;
                if (at >= 0) {
                    x = load16(p + at * (int)sizeof(E));
                } else {                                 // rows shorter than a piece
#pragma unroll
                    for (int j = 0; j < kEach; ++j) {
                        if (j >= r.d) continue;
                        if constexpr (sizeof(E) == 2)
                            x[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[j] << (16 * (j & 1));
                        else
                            x[j] = reinterpret_cast<const uint32_t *>(p)[j];
                    }
                }
            }
            v[i] = x;
        }
    }
    __device__ __forceinline__ void commit(const Rows &r, int tid, const Tile<E, W> &t) const {
        const int piece = tid % kPerRow, over = (piece + 1) * kEach - r.d;
        const bool shifted = over > 0 && over < kEach && r.d >= kEach;
        const int bits = over * (int)sizeof(E) * 8;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            u32x4 x = v[i];
            if (shifted) x = __builtin_bit_cast(u32x4, __builtin_bit_cast(unsigned __int128, x) >> bits);
            const int row = (i * THREADS + tid) / kPerRow;
            *reinterpret_cast<u32x4 *>(t.p + row * Tile<E, W>::kRow + piece * 16) = x;
        }
    }
};

// What a chunk needs of the gates.  A sum of gates b (base 2) is held as a whole number and a rest, so that differences of near steps
// keep their digits whatever lies before them.
template <int C>
struct Gates {
    float whole[C], rest[C];
    float in[C];                        // exp(b_i)
    float out[C];                       // exp(b_last - b_i)
    float last;                         // exp(b_last)
    float sum;                          // b_last, base 2
};

// One wave forms them: lane i brings gate i (natural log; 0 where there is no step)
template <int C>
__device__ inline void form_gates(Gates<C> &s, float gate, int lane) {
    // below 2^-65536 nothing changes, and a gate of exactly zero (-inf) has to stay a number
    const float g2 = fmaxf(gate * kLog2e, -65536.f);
    float whole = __builtin_rintf(g2), rest = g2 - whole;
    whole = wave_inclusive_scan(whole);
    rest = wave_inclusive_scan(rest);
    const float wl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, whole), 63));
    const float rl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, rest), 63));
    if (lane < C) {
        s.whole[lane] = whole;
        s.rest[lane] = rest;
        s.in[lane] = exp2_fast(whole + rest);
        s.out[lane] = exp2_fast((wl - whole) + (rl - rest));
    }
    if (lane == 0) {
        s.last = exp2_fast(wl + rl);
        s.sum = wl + rl;
    }
}

// P^T of a chunk in LDS, as the operands that (2) reads: entry (i tile, jk, part) of 64 lanes x 16 bytes
template <typename E>
struct Pairs {
    static constexpr int C = Elem<E>::kChunk, kI = C / 16, kJ = C / Elem<E>::kDeep, kParts = Elem<E>::kParts;
    static constexpr int kBytes = kI * kJ * kParts * 1024;
    char *p;
    __device__ __forceinline__ char *at(int it, int jk, int part, int lane) const { return p + (((it * kJ + jk) * kParts + part) * 64 + lane) * 16; }
};

// One wave's part of a walk
template <typename E, int M, int N>
struct Walker {
    static constexpr int C = Elem<E>::kChunk, kDeep = Elem<E>::kDeep, kI = C / 16, kJ = C / kDeep;
    static constexpr int kRows = M / 16, kCols = N / 64, kSteps = M / kDeep, kParts = Elem<E>::kParts;
    f32x4 S[kRows][kCols];
    f32x4 O[kCols][kI];
    int lane, lm, g, w;

    __device__ __forceinline__ void init(int tid) {
        lane = tid & 63;
        lm = lane & 15;
        g = lane >> 4;
        w = __builtin_amdgcn_readfirstlane((tid >> 6) & 3);
    }
    __device__ __forceinline__ int col_tile(int n) const { return w * kCols + n; }
    // the same lane, unknown to the optimiser: the addresses and edges of rows and states are formed where they are needed instead of
    // being held over the chunk loop (they would take more registers than the state)
    struct Lane {
        int lm, g;
    };
    __device__ __forceinline__ Lane fresh() const {
        const int l = recompute_per_chunk(lane);
        return Lane{l & 15, l >> 4};
    }

    // element (row, col) of the state at p[row * n + col], or with t at p[col * m + row]
    __device__ __forceinline__ void load_state(const float *p, int m, int n, bool t) {
        const auto [lm, g] = fresh();
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int row = state_row<E>(a, g, 0), col = col_tile(c) * 16 + lm;
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                if (p != nullptr && col < n && row < m) {
                    if (t && row + 4 <= m) {
                        __builtin_memcpy(&x, p + (size_t)col * m + row, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m) x[r] = t ? p[(size_t)col * m + row + r] : p[(size_t)(row + r) * n + col];
                    }
                }
                S[a][c] = x;
            }
    }
    __device__ __forceinline__ void store_state(float *p, int m, int n, bool t, float factor = 1.f) const {
        const auto [lm, g] = fresh();
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int row = state_row<E>(a, g, 0), col = col_tile(c) * 16 + lm;
                const f32x4 x = S[a][c] * factor;
                if (col < n && row < m) {
                    if (t && row + 4 <= m) {
                        __builtin_memcpy(p + (size_t)col * m + row, &x, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m) (t ? p[(size_t)col * m + row + r] : p[(size_t)(row + r) * n + col]) = x[r];
                    }
                }
            }
    }
    // this lane's part of <state at p, S>
    __device__ __forceinline__ float meet_state(const float *p, int m, int n, bool t) const {
        const auto [lm, g] = fresh();
        float sum = 0.f;
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int row = state_row<E>(a, g, 0), col = col_tile(c) * 16 + lm;
                if (col < n && row < m) {
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
                    if (t && row + 4 <= m) {
                        __builtin_memcpy(&x, p + (size_t)col * m + row, 16);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (row + r < m) x[r] = t ? p[(size_t)col * m + row + r] : p[(size_t)(row + r) * n + col];
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum = fmaf(x[r], S[a][c][r], sum);
                }
            }
        return sum;
    }

    // (1) P^T of the lower triangle.  The triangle's tiles are dealt to the waves in turn.
    __device__ __forceinline__ void pairs(const Tile<E, M> &x, const Tile<E, M> &y, const Pairs<E> &P, const Gates<C> &gt) const {
#pragma unroll
        for (int it = 0; it < kI; ++it)
#pragma unroll
            for (int jt = 0; jt < kI; ++jt) {
                if (jt > it || ((it * (it + 1) / 2 + jt) & 3) != w) continue;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) acc = product<E>(y.along(jt * 16 + lm, ks, g), x.along(it * 16 + lm, ks, g), acc);
                const int i = it * 16 + lm, j0 = jt * 16 + g * 4;
                const float wi = gt.whole[i], ri = gt.rest[i];
                const f32x4 wj = *reinterpret_cast<const f32x4 *>(&gt.whole[j0]), rj = *reinterpret_cast<const f32x4 *>(&gt.rest[j0]);
                f32x4 p;
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = j0 + r <= i ? acc[r] * exp2_fast((wi - wj[r]) + (ri - rj[r])) : 0.f;
                if constexpr (sizeof(E) == 2) {
                    u32x2 hi, lo;
                    SPLIT_PAIR(p[0], p[1], hi[0], lo[0]);
                    SPLIT_PAIR(p[2], p[3], hi[1], lo[1]);
                    *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, 0, lane) + 8 * (jt & 1)) = hi;
                    *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, 1, lane) + 8 * (jt & 1)) = lo;
                    // the upper half of a diagonal operand
                    if (jt == it && (jt & 1) == 0) {
                        *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, 0, lane) + 8) = u32x2{0u, 0u};
                        *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, 1, lane) + 8) = u32x2{0u, 0u};
                    }
                } else {
                    *reinterpret_cast<f32x4 *>(P.at(it, jt, 0, lane)) = p;
                }
            }
    }
    // (1) out^T = exp(b_i) S^T x^T
    __device__ __forceinline__ void from_state(const Tile<E, M> &x, const Gates<C> &gt) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int it = 0; it < kI; ++it) O[c][it] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
            u32x4 a[kCols][kParts];
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                if constexpr (sizeof(E) == 2) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            SPLIT_PAIR(S[2 * ks + h][c][2 * r], S[2 * ks + h][c][2 * r + 1], a[c][0][2 * h + r], a[c][1][2 * h + r]);
                } else {
                    a[c][0] = __builtin_bit_cast(u32x4, S[ks][c]);
                }
            }
#pragma unroll
            for (int it = 0; it < kI; ++it) {
                const u32x4 b = x.along(it * 16 + lm, ks, g);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int q = 0; q < kParts; ++q) O[c][it] = product<E>(a[c][q], b, O[c][it]);
            }
        }
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const float e = gt.in[it * 16 + lm];
#pragma unroll
            for (int c = 0; c < kCols; ++c) O[c][it] *= e;
        }
    }
    // (2) OUT: out^T += z^T P^T.  The state: S = exp(b_last) S + y^T (exp(b_last - b_j) z)
    template <bool OUT>
    __device__ __forceinline__ void advance(const Tile<E, M> &y, const Tile<E, N> &z, const Pairs<E> &P, const Gates<C> &gt) {
        const float last = gt.last;
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) S[a][c] *= last;
#pragma unroll
        for (int jk = 0; jk < kJ; ++jk) {
            u32x4 zf[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) zf[c] = z.template across<false>(jk, col_tile(c), lm, g);
            if constexpr (OUT) {
#pragma unroll
                for (int it = 0; it < kI; ++it) {
                    if (jk * kDeep > it * 16 + 15) continue;
#pragma unroll
                    for (int q = 0; q < kParts; ++q) {
                        const u32x4 b = *reinterpret_cast<const u32x4 *>(P.at(it, jk, q, lane));
#pragma unroll
                        for (int c = 0; c < kCols; ++c) O[c][it] = product<E>(zf[c], b, O[c][it]);
                    }
                }
            }
            u32x4 zd[kCols][kParts];
            if constexpr (sizeof(E) == 2) {
                const f32x4 d0 = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 32 + g * 4]);
                const f32x4 d1 = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 32 + 16 + g * 4]);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 &d = r < 2 ? d0 : d1;
                        SPLIT_PAIR(bf16_lo_as_float(zf[c][r]) * d[2 * (r & 1)], bf16_hi_as_float(zf[c][r]) * d[2 * (r & 1) + 1], zd[c][0][r],
                                   zd[c][1][r]);
                    }
            } else {
                const f32x4 d = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 16 + g * 4]);
#pragma unroll
                for (int c = 0; c < kCols; ++c) zd[c][0] = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, zf[c]) * d);
            }
#pragma unroll
            for (int a = 0; a < kRows; ++a) {
                const u32x4 yf = y.template across<true>(jk, a, lm, g);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int q = 0; q < kParts; ++q) S[a][c] = product<E>(yf, zd[c][q], S[a][c]);
            }
        }
    }
    // out row . dot row, this wave's columns, to part[w * C + row]; the dot rows from memory, or with LDS_ROWS from the tile
    template <bool LDS_ROWS, typename TokenOf>
    __device__ __forceinline__ void dot_rows(const Rows &r, const Tile<E, N> &t, float *part, int count, TokenOf token) const {
        const auto [lm, g] = fresh();
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const int i = it * 16 + lm;
            float sum = 0.f;
            if (LDS_ROWS || i < count) {
                const char *row = LDS_ROWS ? t.p + i * Tile<E, N>::kRow : r.base + token(i) * r.step;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const int col = col_tile(c) * 16 + g * 4;
                    f32x4 x = {0.f, 0.f, 0.f, 0.f};
                    if (LDS_ROWS || col + 4 <= r.d) {
                        if constexpr (sizeof(E) == 2) {
                            u32x2 b;
                            __builtin_memcpy(&b, row + col * 2, 8);
                            x = f32x4{bf16_lo_as_float(b[0]), bf16_hi_as_float(b[0]), bf16_lo_as_float(b[1]), bf16_hi_as_float(b[1])};
                        } else {
                            __builtin_memcpy(&x, row + col * 4, 16);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + j < r.d) {
                                if constexpr (sizeof(E) == 2) x[j] = bf16_bits_to_float(reinterpret_cast<const uint16_t *>(row)[col + j]);
                                else x[j] = reinterpret_cast<const float *>(row)[col + j];
                            }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum = fmaf(x[j], O[c][it][j], sum);
                }
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0) part[w * C + i] = sum;
        }
    }
    // rows of the chunk out of the accumulators; token(i) of row i
    template <typename TokenOf>
    __device__ __forceinline__ void store_rows(const Rows &r, int out_dtype, int count, TokenOf token) const {
        const auto [lm, g] = fresh();
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const int i = it * 16 + lm;
            if (i >= count) continue;
            char *row = const_cast<char *>(r.base) + token(i) * r.step;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int col = col_tile(c) * 16 + g * 4;
                const f32x4 x = O[c][it];
                if (out_dtype == GLA_DT_BF16) {
                    const u32x2 v = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
                    if (col + 4 <= r.d) {
                        __builtin_memcpy(row + col * 2, &v, 8);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + j < r.d) reinterpret_cast<uint16_t *>(row)[col + j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
                    }
                } else if (col + 4 <= r.d) {
                    __builtin_memcpy(row + col * 4, &x, 16);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col + j < r.d) reinterpret_cast<float *>(row)[col + j] = x[j];
                }
            }
        }
    }
};

// Rows of one sequence: what a walk visits in which order.  Chunk number ci covers steps [ci * C, min((ci + 1) * C, len)) whichever
// way it is walked; backwards row 0 is the last of them.
struct Order {
    int scan_dir, len, grid_h, grid_w;
    int T;
    __device__ __forceinline__ int token(int s) const { return scan_token(scan_dir, s, len, grid_h, grid_w); }
};
__device__ inline Order order_of(const DecayCall &c, int bh) {
    Order o;
    o.scan_dir = c.scan_dir;
    o.grid_h = c.grid_h;
    o.grid_w = c.grid_w;
    o.T = c.T;
    o.len = c.T;
    if (c.seq_lens != nullptr) {
        const int n = c.seq_lens[bh / c.H];
        o.len = n < 0 ? 0 : n < c.T ? n : c.T;       // (a length outside 0 .. T counts as the nearer end)
    }
    return o;
}

// log_decay of step s (0 outside the sequence)
__device__ inline float gate_of(const DecayCall &c, const Order &o, int bh, int s) {
    if (s < 0 || s >= o.len) return 0.f;
    const int h = bh % c.H;
    if (c.kind == kDecayHead) return c.log_decay[h];
    const long long n = o.token(s);
    const long long at = c.layout == GLA_LAYOUT_BHTD ? (long long)bh * c.T + n : ((long long)(bh / c.H) * c.T + n) * c.H + h;
    return c.log_decay[at];
}

// Clears the rows of steps behind the sequence's end that the span [s0, s1) covers
template <int THREADS>
__device__ inline void clear_behind(const Rows &r, int size, int len, int s0, int s1, int tid) {
    const int from = len > s0 ? len : s0;
    const int words = r.d;
    for (int n = from; n < s1; ++n) {
        char *row = const_cast<char *>(r.base) + n * r.step;
        for (int j = tid; j < words; j += THREADS) {
            if (size == 2) reinterpret_cast<uint16_t *>(row)[j] = 0;
            else reinterpret_cast<float *>(row)[j] = 0.f;
        }
    }
}

}  // namespace
}  // namespace gla
