// Device side of the walks of gla_decay.h: tiles of rows in LDS, the operands that the matrix instructions take from them, and one
// chunk of the recurrence.
//
// Four waves walk one state [m, n] (padded to M, N): wave w holds all rows of columns w * N/4 .. + N/4 - 1 in registers, as
// accumulators of 16 x 16 products with lane = column, and works on these columns of the outputs.  A chunk is
//   (1) P^T = y x^T of the lower triangle times exp(b_i - b_j), its tiles dealt to the waves, to LDS; out^T = exp(b_i) S^T x^T and then
//       S = exp(b_last) S + y^T (exp(b_last - b_j) z), all in-wave; a barrier, behind which the rows are not read any more
//   (2) out^T += z^T P^T with z's operands from registers, out to memory, the next chunk's rows into LDS; a barrier.
// Everything is formed transposed, so that the accumulators of one product are an operand of the next as they stand: an operand
// is eight (bf16) or four (fp32) values of the contracted index in a lane, and which index stands where does not matter as long as
// both operands agree.  The state's rows are ordered (state_row) so that x's operands are 16 contiguous bytes of a row.
// bf16 calls split what is not bf16 by itself (the state, P, the decayed z) into bf16 numbers, head and remainders (Elem).  Two leave 2^-18 of
// each: outputs in 32 bits and a token's gate gradient hold 2e-6 to 7e-6 where one bf16 would leave 2e-3, which rows of 16 bits (2^-9) do not show.
// Three leave what fp32 leaves, 1e-7 to 4e-7.  They are taken (DecayDigits)
//   for the decayed z where a state is given back, which stands in 32 bits for all that comes after it (2.4e-6 with two; forward, 65536 steps
//   of 16 heads 128 x 128: 420 us, 392 with two; prompts of 128 sequences 100 us, 92);
//   for all where a head's one decay is learnt: its gradient is a sum over all steps in which each block's flows count by their place, so that errors
//   add up to 256 / (memory in steps) times as much, 2e-5 to 6e-5 for a single head of 30 steps' memory with two (a training step of 64
//   sequences of 4096 steps, 128 x 128: 660 us, 490 with two).
// For all that a bf16 call gives in 32 bits they would cost as much again for tokens' gates and 10 to 60 % forward; calls on the same rows in fp32 have
// these digits.
// fp32 calls run on the fp32 matrix instructions.
#pragma once
#include "gla_decay.h"
#include "gla_mfma_util.h"

namespace gla {
namespace {

template <typename E> struct Elem;
// bf16 rows.  A factor that is no input by itself is as many bf16 numbers, head and remainders: STATE the decayed z that the state takes up, OUT the
// state and P that the outputs are formed from (DecayDigits).
template <int STATE, int OUT>
struct Bf16 {
    uint16_t bits;
};
template <int STATE, int OUT>
struct Elem<Bf16<STATE, OUT>> {
    static constexpr int kChunk = 64;            // steps
    static constexpr int kDeep = 32;             // contracted values of an operand over the wave
    static constexpr int kStateParts = STATE, kOutParts = OUT;
};
template <> struct Elem<float> {
    static constexpr int kChunk = 32;
    static constexpr int kDeep = 16;
    static constexpr int kStateParts = 1, kOutParts = 1;
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

// How a tile's rows are read: along them (the row is an operand's other index), across them (the contracted one), or both
enum Reads { kAlong, kAcross, kBoth };

// A tile of C rows of W elements in LDS.  Rows lie so far apart that the banks are met evenly: 16 rows' same piece when read along, 8 rows' 32
// bytes (bf16) or 4 rows' 64 (fp32) when read across.  (With rows 16 bytes apart throughout, near half of the time that LDS was busy
// went to conflicts.  An exchange of pieces by the row's number is free of them, but then no read's address is a constant from
// another's: 6 % more instructions.)
// A bf16 tile for both holds each 32 columns in the order in which state_row() counts a state's rows: the 8 bytes number 4 h + c are columns
// 8 c + 4 h and on.  The four c are exchanged by the row's number over four (xor), which reads across see as a constant of the lane,
// and without which reads along met each bank four times (2.9e7 cycles of conflicts in the walk of 65536 steps of 16 heads, 1.0e7 with it).
template <typename E, int W, Reads R>
struct Tile {
    static constexpr int C = Elem<E>::kChunk;
    static constexpr int kRow = W * (int)sizeof(E) + (sizeof(E) == 2 && R != kAlong ? 32 : 16);      // bytes
    static constexpr int kBytes = C * kRow;
    static constexpr bool kMoved = R == kBoth && sizeof(E) == 2;
    char *p;
    // 16 bytes of row 16 tile + lm: the operand of contraction step ks whose other index is the row
    __device__ __forceinline__ u32x4 along(int tile, int lm, int ks, int g) const {
        const char *a = p + tile * 16 * kRow + lm * kRow;
        if constexpr (kMoved) {
            const u32x2 lo = *reinterpret_cast<const u32x2 *>(a + (g ^ (lm >> 2)) * 8 + ks * 64);
            const u32x2 hi = *reinterpret_cast<const u32x2 *>(a + (g ^ (lm >> 2)) * 8 + ks * 64 + 32);
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            return *reinterpret_cast<const u32x4 *>(a + g * 16 + ks * 64);
        }
    }
    // the operand that contracts over rows: step jk of kDeep rows, other index = the lane's of the 16 columns of tile t (in the order
    // in which they lie)
    __device__ __forceinline__ u32x4 across(int jk, int t, int lm, int g) const {
        if constexpr (sizeof(E) == 2) {
            const char *a = p + (g * 4 + (lm >> 2)) * kRow + ((lm & 3) ^ (kMoved ? g : 0)) * 8 + jk * 32 * kRow + t * 32;
            const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(a));
            const u32x2 hi = lds_read_tr(reinterpret_cast<const uint16_t *>(a + 16 * kRow));
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const char *a = p + g * 4 * kRow + lm * 4 + jk * 16 * kRow + t * 64;
            u32x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = *reinterpret_cast<const uint32_t *>(a + r * kRow);
            return v;
        }
    }
    // 16 bytes of a row as they come from memory
    __device__ __forceinline__ void put_piece(int row, int piece, u32x4 x) const {
        char *a = p + row * kRow;
        if constexpr (kMoved) {
            a += (piece >> 2) * 64 + ((piece & 3) ^ (row >> 2 & 3)) * 8;
            *reinterpret_cast<u32x2 *>(a) = u32x2{x[0], x[1]};
            *reinterpret_cast<u32x2 *>(a + 32) = u32x2{x[2], x[3]};
        } else {
            *reinterpret_cast<u32x4 *>(a + piece * 16) = x;
        }
    }
    // neighbouring elements of a row from column `col` on (of a tile in the order of memory)
    __device__ __forceinline__ const char *at(int row, int col) const {
        static_assert(!kMoved, "columns as they come");
        return p + row * kRow + col * (int)sizeof(E);
    }
};

// x0, x1 -> packed bf16 pair of the rounded values and packed pairs of the remainders.  A remainder x - head is one dot product of
// the packed heads with (-1, 0) or (0, -1) added to x (exact), where taking a head out of the pair and subtracting it are two.
struct Heads {
    bf16x2 first, second;
    __device__ __forceinline__ Heads() {
        // (as constants in the instruction these two pairs would be read as other values)
        uint32_t a = 0x0000bf80u, b = 0xbf800000u;
        asm("" : "+s"(a));
        asm("" : "+s"(b));
        first = __builtin_bit_cast(bf16x2, a);
        second = __builtin_bit_cast(bf16x2, b);
    }
    // PARTS packed pairs that add up to x0, x1
    template <int PARTS>
    __device__ __forceinline__ void split(float x0, float x1, uint32_t (&to)[PARTS]) const {
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            to[q] = pack_bf16(x0, x1);
            if (q + 1 == PARTS) break;
            const bf16x2 h = __builtin_bit_cast(bf16x2, to[q]);
            x0 = __builtin_amdgcn_fdot2_f32_bf16(h, first, x0, false);
            x1 = __builtin_amdgcn_fdot2_f32_bf16(h, second, x1, false);
        }
    }
};

// The steps of one chunk and where their rows lie.  Row scans: tokens first .. first + count - 1, rising or falling with the row number;
// column scans: each row its own token (first = 0).
struct Steps {
    int scan_dir, len, grid_h, grid_w;
    int s, count;                       // first step, steps
    bool back;                          // row 0 is the last step
    int first;
    bool falling;
    __device__ __forceinline__ int step_of(int i) const { return back ? s + count - 1 - i : s + i; }
    // token of row i, less `first`
    __device__ __forceinline__ int at(int i) const {
        if (scan_dir < GLA_SCAN_COL_FWD) return falling ? count - 1 - i : i;
        return scan_token(scan_dir, step_of(i), len, grid_h, grid_w);
    }
    // byte offsets of rows i0, i0 + di, ... of `step` bytes each behind `first`'s; kNowhere from `most` on
    template <int K>
    __device__ __forceinline__ void offsets(uint32_t (&o)[K], int i0, int di, uint32_t step, int most, uint32_t plus) const {
        if (scan_dir < GLA_SCAN_COL_FWD) {
            const uint32_t by = falling ? 0u - step : step;
            const uint32_t at = (falling ? (uint32_t)(count - 1) * step : 0u) + __umul24((uint32_t)i0, step) * (falling ? 0xffffffffu : 1u) + plus;
#pragma unroll
            for (int k = 0; k < K; ++k) o[k] = i0 + k * di < most ? at + (uint32_t)(k * di) * by : kNowhere;
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) o[k] = i0 + k * di < most ? __umul24((uint32_t)at(i0 + k * di), step) + plus : kNowhere;
        }
    }
};
// Rows of one sequence: what a walk visits in which order.  Chunk number ci covers steps [ci * C, min((ci + 1) * C, len)) whichever
// way it is walked; backwards row 0 is the last of them.
struct Order {
    int scan_dir, len, grid_h, grid_w;
    __device__ __forceinline__ int token(int s) const { return scan_token(scan_dir, s, len, grid_h, grid_w); }
    __device__ __forceinline__ Steps steps(int s, int count, bool back) const {
        Steps x;
        x.scan_dir = scan_dir;
        x.len = len;
        x.grid_h = grid_h;
        x.grid_w = grid_w;
        x.s = s;
        x.count = count;
        x.back = back;
        x.first = scan_dir >= GLA_SCAN_COL_FWD ? 0 : scan_dir == GLA_SCAN_ROW_FWD ? s : len - s - count;
        x.falling = back != (scan_dir == GLA_SCAN_ROW_REV);
        return x;
    }
};
__device__ __forceinline__ Order order_of(const DecayCall &c, int bh) {
    Order o;
    o.scan_dir = c.scan_dir;
    o.grid_h = c.grid_h;
    o.grid_w = c.grid_w;
    o.len = c.T;
    if (c.seq_lens != nullptr) {
        const int n = c.seq_lens[bh / c.H];
        o.len = n < 0 ? 0 : n < c.T ? n : c.T;       // (a length outside 0 .. T counts as the nearer end)
    }
    return o;
}

// Rows of a [.., d] tensor of one (batch, head): 64-bit offsets, so any length does
struct Rows {
    const char *base;
    long long step;                     // bytes between tokens
    int d;
    __device__ __forceinline__ const char *token(long long n) const { return base + n * step; }
};
template <typename E>
__device__ __forceinline__ Rows rows_of(const DecayCall &c, const void *t, int bh, int d, int size = (int)sizeof(E)) {
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
// FAST: rows are read and written through views with 32-bit offsets from the chunk's first token, where an offset that is kNowhere reads
// zeros and writes nothing; the host chooses it where every offset stays below that and rows are whole dwords (DecayCall::fast).  The
// other form takes any place and width with 64-bit addresses and branches.
__device__ __forceinline__ Rsrc chunk_view(const Rows &r, const Steps &t) { return view(r.token(t.first), kNowhere); }

__device__ __forceinline__ u32x4 load16(const char *p) {          // any alignment
    u32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// The pieces (16 bytes) of a tile that one of THREADS threads brings: issue() asks for them, commit() puts them into the tile once
// the one before has been used.  Rows from `count` on and columns from d on are zeros and are not read.
template <typename E, int W, int THREADS, bool FAST>
struct Pieces {
    static constexpr int kPerRow = W * (int)sizeof(E) / 16, kEach = 16 / (int)sizeof(E);
    static constexpr int kChunk = Elem<E>::kChunk, kCount = kChunk * kPerRow / THREADS;
    static_assert(THREADS % kPerRow == 0 && kChunk * kPerRow % THREADS == 0, "whole rows, whole pieces a thread");
    u32x4 v[kCount];
    __device__ __forceinline__ void issue(const Rows &r, int tid, const Steps &t) {
        const int col = tid % kPerRow * kEach;
        // the last piece of a row that is no whole number of pieces is read as the row's last 16 bytes and shifted in commit()
        const int at = col + kEach <= r.d ? col : r.d - kEach;
        if constexpr (FAST) {
            const Rsrc b = chunk_view(r, t);
            uint32_t o[kCount];
            t.offsets(o, tid / kPerRow, THREADS / kPerRow, (uint32_t)r.step, col < r.d ? t.count : 0, (uint32_t)at * sizeof(E));
#pragma unroll
            for (int i = 0; i < kCount; ++i) v[i] = fetch<u32x4>(b, o[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int row = i * (THREADS / kPerRow) + tid / kPerRow;
            u32x4 x = {0u, 0u, 0u, 0u};
            if (row < t.count && col < r.d) {
                const char *p = r.token((long long)t.first + t.at(row));
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
    template <Reads R>
    __device__ __forceinline__ void commit(const Rows &r, int tid, const Tile<E, W, R> &t) const {
        const int piece = tid % kPerRow, row = tid / kPerRow, over = (piece + 1) * kEach - r.d;
        constexpr int by = THREADS / kPerRow;
        const bool shifted = over > 0 && over < kEach && r.d >= kEach;
        if (r.d % kEach == 0) {
#pragma unroll
            for (int i = 0; i < kCount; ++i) t.put_piece(row + i * by, piece, v[i]);
            return;
        }
        const int bits = over * (int)sizeof(E) * 8;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            u32x4 x = v[i];
            if constexpr (FAST) {                        // half a piece
                if (shifted) x = u32x4{x[2], x[3], 0u, 0u};
            } else {
                if (shifted) x = __builtin_bit_cast(u32x4, __builtin_bit_cast(unsigned __int128, x) >> bits);
            }
            t.put_piece(row + i * by, piece, x);
        }
    }
};

// A gate, base 2.  One of exactly zero (-inf) has to stay a number: 2^-1024 is zero too, and 64 of them are 2^23 units of 2^-7; a NaN stays one.
__device__ __forceinline__ float gate_log2(float log_decay) {
    const float g = log_decay * kLog2e;
    return g < -1024.f ? -1024.f : g;
}

// What a chunk needs of the gates.  A sum of gates b (base 2) is held as a number of units of 2^-7 (`whole`) and a rest, so that differences of
// near steps keep their digits whatever lies before them: sums of units are exact, and sums of 64 rests stay below 1/4.  (With units
// of 1 the rests of gates of -0.2 added up to 18, and exp(b_i - b_j) was off by 16 * 2^-24; by 2^-25 of its own with these.)
template <int C>
struct Gates {
    float whole[C], rest[C];
    float in[C];                        // exp(b_i)
    float out[C];                       // exp(b_last - b_i)
    float tile[C];                      // exp(b_t - b_i), t the last step of the 16 that i is one of
    float last;                         // exp(b_last)
    float sum;                          // b_last, base 2
};

// One wave forms them: lane i brings gate i (natural log; 0 where there is no step)
template <int C>
__device__ inline void form_gates(Gates<C> &s, float gate, int lane) {
    const float g2 = gate_log2(gate);
    float whole = __builtin_rintf(g2 * 128.f) * 0.0078125f, rest = g2 - whole;
    whole = wave_inclusive_scan(whole);
    rest = wave_inclusive_scan(rest);
    const float wl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, whole), 63));
    const float rl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, rest), 63));
    const float wt = __shfl(whole, lane | 15), rt = __shfl(rest, lane | 15);
    if (lane < C) {
        s.tile[lane] = exp2_fast((wt - whole) + (rt - rest));
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
    static constexpr int C = Elem<E>::kChunk, kI = C / 16, kJ = C / Elem<E>::kDeep, kParts = Elem<E>::kOutParts;
    static constexpr int kBytes = kI * kJ * kParts * 1024;
    char *p;
    __device__ __forceinline__ char *at(int it, int jk, int part, int lane) const { return p + (((it * kJ + jk) * kParts + part) * 64 + lane) * 16; }
};

// One wave's part of a walk.  ZA: z's tile is one for both, so that the state's columns are counted like its rows
template <typename E, int M, int N, bool FAST, bool ZA>
struct Walker {
    static constexpr int C = Elem<E>::kChunk, kDeep = Elem<E>::kDeep, kI = C / 16, kJ = C / kDeep;
    static constexpr int kRows = M / 16, kCols = N / 64, kSteps = M / kDeep, kParts = Elem<E>::kOutParts, kStateParts = Elem<E>::kStateParts;
    f32x4 S[kRows][kCols];
    f32x4 O[kCols][kI];
    int lane, lm, g, w;

    __device__ __forceinline__ void init(int tid) {
        lane = tid & 63;
        lm = lane & 15;
        g = lane >> 4;
        w = __builtin_amdgcn_readfirstlane((tid >> 6) & 3);
    }
    __device__ __forceinline__ int col_tile(int c) const { return w * kCols + c; }
    // column of lane `lm` of tile c, and the first of the four of lane group g in what is formed transposed
    __device__ __forceinline__ int col_of(int c, int lm) const {
        return ZA ? state_row<E>(col_tile(c), lm >> 2, lm & 3) : col_tile(c) * 16 + lm;
    }
    __device__ __forceinline__ int cols_of(int c, int g) const { return ZA ? state_row<E>(col_tile(c), g, 0) : col_tile(c) * 16 + g * 4; }
    // the same lane, unknown to the optimiser: the addresses and edges of rows and states are formed where they are needed instead of
    // being held over the chunk loop (they would take more registers than the state)
    struct Lane {
        int lm, g;
    };
    __device__ __forceinline__ Lane fresh() const {
        const int l = recompute_per_chunk(lane);
        return Lane{l & 15, l >> 4};
    }

    // element (row, col) of the state at p[row * n + col], or with t at p[col * m + row]; what this lane holds of tile (a, c)
    __device__ __forceinline__ f32x4 state_at(const float *p, const Rsrc &b, int row, int col, int m, int n, bool t) const {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        if constexpr (FAST) {                            // (m is a multiple of 4)
            const bool there = col < n && row < m;
            if (t) return fetch<f32x4>(b, there ? (uint32_t)(col * m + row) * 4u : kNowhere);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = fetch<float>(b, there ? (uint32_t)((row + r) * n + col) * 4u : kNowhere);
        } else if (col < n && row < m) {
            if (t && row + 4 <= m) {
                __builtin_memcpy(&x, p + (size_t)col * m + row, 16);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (row + r < m) x[r] = t ? p[(size_t)col * m + row + r] : p[(size_t)(row + r) * n + col];
            }
        }
        return x;
    }
    __device__ __forceinline__ void load_state(const float *p, int m, int n, bool t) {
        const auto [lm, g] = fresh();
        const Rsrc b = view(p, kNowhere);
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                S[a][c] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (p != nullptr) S[a][c] = state_at(p, b, state_row<E>(a, g, 0), col_of(c, lm), m, n, t);
            }
    }
    // S = factor S + the state at p
    __device__ __forceinline__ void add_state(const float *p, int m, int n, bool t, float factor) {
        const auto [lm, g] = fresh();
        const Rsrc b = view(p, kNowhere);
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) S[a][c] = S[a][c] * factor + state_at(p, b, state_row<E>(a, g, 0), col_of(c, lm), m, n, t);
    }
    // the state that enters span sp, walked forward or (back) from the last span to the first
    __device__ __forceinline__ void enter(const DecayEntry &e, int bh, int sp, int nspans, bool back, int m, int n, bool t) {
        const size_t cells = (size_t)m * n;
        const int before = back ? nspans - 1 - sp : sp;
        if (e.chained) {
            load_state(e.local + ((size_t)bh * nspans + sp) * cells, m, n, t);
            return;
        }
        load_state(e.first == nullptr ? nullptr : e.first + (size_t)bh * cells, m, n, t);
        for (int k = 0; k < before; ++k) {
            const size_t at = (size_t)bh * nspans + (back ? nspans - 1 - k : k);
            add_state(e.local + at * cells, m, n, t, exp2_fast(e.decay[at]));
        }
    }
    __device__ __forceinline__ void store_state(float *p, int m, int n, bool t, float factor = 1.f) const {
        const auto [lm, g] = fresh();
        const Rsrc b = view(p, kNowhere);
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int row = state_row<E>(a, g, 0), col = col_of(c, lm);
                const f32x4 x = S[a][c] * factor;
                if constexpr (FAST) {
                    const bool there = col < n && row < m;
                    if (t) {
                        put(b, there ? (uint32_t)(col * m + row) * 4u : kNowhere, x);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float xr = x[r];
                            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, xr), b,
                                                                  (int)(there ? (uint32_t)((row + r) * n + col) * 4u : kNowhere), 0, 0);
                        }
                    }
                } else if (col < n && row < m) {
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
        const Rsrc b = view(p, kNowhere);
        float sum = 0.f;
#pragma unroll
        for (int a = 0; a < kRows; ++a)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const f32x4 x = state_at(p, b, state_row<E>(a, g, 0), col_of(c, lm), m, n, t);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum = fmaf(x[r], S[a][c][r], sum);
            }
        return sum;
    }

    // (1) P^T of the lower triangle, whose tiles are dealt to the waves in turn.  Products that add to one accumulator are kept apart, here and
    // below: each would wait for the one before.  With `diag` the diagonal goes there instead of into P, for add_diagonal().
    __device__ __forceinline__ void pairs(const Tile<E, M, kAlong> &x, const Tile<E, M, kBoth> &y, const Pairs<E> &P, const Gates<C> &gt,
                                          bool apart = false, float *diag = nullptr) const {
        constexpr int kTiles = kI * (kI + 1) / 2, kMine = (kTiles + 3) / 4;
        const Heads heads;
#pragma unroll
        for (int t = 0; t < kMine; ++t) {
            // tile number t * 4 + w of the triangle, row by row (the last one more than once: the same values)
            const int id = min(t * 4 + w, kTiles - 1);
            int it = 0;
#pragma unroll
            for (int k = 1; k < kI; ++k) it += id >= k * (k + 1) / 2;
            const int jt = id - it * (it + 1) / 2;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f}, odd = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks) {
                f32x4 &to = ks & 1 ? odd : acc;
                to = product<E>(y.along(jt, lm, ks, g), x.along(it, lm, ks, g), to);
            }
            acc += odd;
            const int i = it * 16 + lm, j0 = jt * 16 + g * 4;
            const float wi = gt.whole[i], ri = gt.rest[i];
            f32x4 p;
            if (jt == it) {
                const f32x4 wj = *reinterpret_cast<const f32x4 *>(&gt.whole[j0]), rj = *reinterpret_cast<const f32x4 *>(&gt.rest[j0]);
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = g * 4 + r <= lm ? acc[r] * exp2_fast((wi - wj[r]) + (ri - rj[r])) : 0.f;
                if (apart) {
                    const auto [lm, g] = fresh();
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (g * 4 + r == lm) {
                            diag[i] = acc[r];
                            p[r] = 0.f;
                        }
                }
            } else {                                     // by way of the last step of j's tile
                const float e = exp2_fast((wi - gt.whole[jt * 16 + 15]) + (ri - gt.rest[jt * 16 + 15]));
                p = acc * (*reinterpret_cast<const f32x4 *>(&gt.tile[j0]) * e);
            }
            if constexpr (sizeof(E) == 2) {
                uint32_t s0[kParts], s1[kParts];
                heads.split(p[0], p[1], s0);
                heads.split(p[2], p[3], s1);
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, q, lane) + 8 * (jt & 1)) = u32x2{s0[q], s1[q]};
                    // the upper half of a diagonal operand
                    if (jt == it && (jt & 1) == 0) *reinterpret_cast<u32x2 *>(P.at(it, jt >> 1, q, lane) + 8) = u32x2{0u, 0u};
                }
            } else {
                *reinterpret_cast<f32x4 *>(P.at(it, jt, 0, lane)) = p;
            }
        }
    }
    // (1) out^T = exp(b_i) S^T x^T of this wave's columns
    __device__ __forceinline__ void from_state(const Tile<E, M, kAlong> &x, const Gates<C> &gt) {
        const Heads heads;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int it = 0; it < kI; ++it) O[c][it] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 b[2][kI];
#pragma unroll
        for (int it = 0; it < kI; ++it) b[0][it] = x.along(it, lm, 0, g);
#pragma unroll
        for (int t = 0; t < kSteps; ++t) {
            u32x4 a[kCols][kParts];
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                if constexpr (sizeof(E) == 2) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                        {
                            uint32_t s[kParts];
                            heads.split(S[2 * t + h][c][2 * r], S[2 * t + h][c][2 * r + 1], s);
#pragma unroll
                            for (int q = 0; q < kParts; ++q) a[c][q][2 * h + r] = s[q];
                        }
                } else {
                    a[c][0] = __builtin_bit_cast(u32x4, S[t][c]);
                }
            }
            if (t + 1 < kSteps) {
#pragma unroll
                for (int k = 0; k < kI; ++k) b[(t + 1) & 1][k] = x.along(k, lm, t + 1, g);
            }
#pragma unroll
            for (int q = 0; q < kParts; ++q)
#pragma unroll
                for (int k = 0; k < kI; ++k)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) O[c][k] = product<E>(a[c][q], b[t & 1][k], O[c][k]);
        }
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const float e = gt.in[it * 16 + lm];
#pragma unroll
            for (int c = 0; c < kCols; ++c) O[c][it] *= e;
        }
    }
    // (1) The state: S = exp(b_last) S + y^T (exp(b_last - b_j) z).  zf: z's operands, which finish() takes too
    __device__ __forceinline__ void update(const Tile<E, M, kBoth> &y, const Tile<E, N, ZA ? kBoth : kAcross> &z, const Gates<C> &gt,
                                           u32x4 (&zf)[kJ][kCols]) {
        const float last = gt.last;
        const Heads heads;
        u32x4 zd[kJ][kCols][kStateParts];
#pragma unroll
        for (int jk = 0; jk < kJ; ++jk) {
#pragma unroll
            for (int c = 0; c < kCols; ++c) zf[jk][c] = z.across(jk, col_tile(c), lm, g);
            if constexpr (sizeof(E) == 2) {
                const f32x4 d0 = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 32 + g * 4]);
                const f32x4 d1 = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 32 + 16 + g * 4]);
#pragma unroll
                for (int c = 0; c < kCols; ++c)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const f32x4 &d = r < 2 ? d0 : d1;
                        uint32_t s[kStateParts];
                        heads.split(bf16_lo_as_float(zf[jk][c][r]) * d[2 * (r & 1)], bf16_hi_as_float(zf[jk][c][r]) * d[2 * (r & 1) + 1], s);
#pragma unroll
                        for (int q = 0; q < kStateParts; ++q) zd[jk][c][q][r] = s[q];
                    }
            } else {
                const f32x4 d = *reinterpret_cast<const f32x4 *>(&gt.out[jk * 16 + g * 4]);
#pragma unroll
                for (int c = 0; c < kCols; ++c) zd[jk][c][0] = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, zf[jk][c]) * d);
            }
        }
        // two tiles of state rows at a time, so that products of one accumulator are four apart, and the next operands on their way
        u32x4 yf[2][2][kJ];
        auto fetch_rows = [&](int a, u32x4(&to)[2][kJ]) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int jk = 0; jk < kJ; ++jk) to[h][jk] = y.across(jk, a + h, lm, g);
        };
        fetch_rows(0, yf[0]);
#pragma unroll
        for (int a = 0; a < kRows; a += 2) {
            if (a + 2 < kRows) fetch_rows(a + 2, yf[(a >> 1) + 1 & 1]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < kCols; ++c) S[a + h][c] *= last;
#pragma unroll
            for (int jk = 0; jk < kJ; ++jk)
#pragma unroll
                for (int q = 0; q < kStateParts; ++q)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int c = 0; c < kCols; ++c) S[a + h][c] = product<E>(yf[a >> 1 & 1][h][jk], zd[jk][c][q], S[a + h][c]);
        }
    }
    // (2) out^T += z^T P^T
    __device__ __forceinline__ void finish(const Pairs<E> &P, const u32x4 (&zf)[kJ][kCols]) {
#pragma unroll
        for (int jk = 0; jk < kJ; ++jk)
#pragma unroll
            for (int q = 0; q < kParts; ++q)
#pragma unroll
                for (int it = 0; it < kI; ++it) {
                    if (jk * kDeep > it * 16 + 15) continue;
                    const u32x4 b = *reinterpret_cast<const u32x4 *>(P.at(it, jk, q, lane));
#pragma unroll
                    for (int c = 0; c < kCols; ++c) O[c][it] = product<E>(zf[jk][c], b, O[c][it]);
                }
    }
    // out^T += z^T diag, where pairs() left the diagonal apart: a product of each tile with an operand that is the diagonal and zeros
    __device__ __forceinline__ void add_diagonal(const float *diag, const u32x4 (&zf)[kJ][kCols]) {
        const Heads heads;
        const auto [lm, g] = fresh();
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const float d = g == lm >> 2 ? diag[it * 16 + lm] : 0.f;
            if constexpr (sizeof(E) == 2) {
                uint32_t s[kParts];
                heads.split(lm & 1 ? 0.f : d, lm & 1 ? d : 0.f, s);
#pragma unroll
                for (int q = 0; q < kParts; ++q) {
                    const uint32_t lo = lm & 2 ? 0u : s[q], hi = lm & 2 ? s[q] : 0u;
                    const u32x4 b = it & 1 ? u32x4{0u, 0u, lo, hi} : u32x4{lo, hi, 0u, 0u};
#pragma unroll
                    for (int c = 0; c < kCols; ++c) O[c][it] = product<E>(zf[it >> 1][c], b, O[c][it]);
                }
            } else {
                f32x4 b;
#pragma unroll
                for (int r = 0; r < 4; ++r) b[r] = (lm & 3) == r ? d : 0.f;
#pragma unroll
                for (int c = 0; c < kCols; ++c) O[c][it] = product<E>(zf[it][c], __builtin_bit_cast(u32x4, b), O[c][it]);
            }
        }
    }
    // The rows that the outputs are multiplied with: this lane's four columns of each tile, from memory or from the tile
    struct Dots {
        uint32_t bits[kI][kCols][sizeof(E)];             // (four elements)
    };
    __device__ __forceinline__ void fetch_dots(Dots &d, const Rows &r, const Steps &st) const {
        const auto [lm, g] = fresh();
        constexpr int size = (int)sizeof(E);
        const Rsrc b = chunk_view(r, st);
        uint32_t o[kI];
        if constexpr (FAST) st.offsets(o, lm, 16, (uint32_t)r.step, st.count, 0u);
#pragma unroll
        for (int it = 0; it < kI; ++it)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int col = cols_of(c, g), i = it * 16 + lm;
                uint32_t(&bits)[size] = d.bits[it][c];
                if constexpr (FAST) {
                    // (nowhere stays nowhere with a column's offset added)
                    const uint32_t at = col < r.d ? o[it] + col * size : kNowhere;
                    if constexpr (size == 2) {
                        const u32x2 v = fetch<u32x2>(b, at);
                        bits[0] = v[0];
                        bits[1] = v[1];
                    } else {
                        const u32x4 v = fetch<u32x4>(b, at);
#pragma unroll
                        for (int j = 0; j < 4; ++j) bits[j] = v[j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < size; ++j) bits[j] = 0u;
                    if (i < st.count) {
                        const char *row = r.token((long long)st.first + st.at(i));
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (col + j < r.d) {
                                if constexpr (size == 2) bits[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[col + j] << (16 * (j & 1));
                                else bits[j] = reinterpret_cast<const uint32_t *>(row)[col + j];
                            }
                    }
                }
            }
    }
    __device__ __forceinline__ void fetch_dots(Dots &d, const Tile<E, N, kAlong> &t) const {
#pragma unroll
        for (int it = 0; it < kI; ++it)
#pragma unroll
            for (int c = 0; c < kCols; ++c) __builtin_memcpy(d.bits[it][c], t.at(it * 16 + lm, cols_of(c, g)), 4 * sizeof(E));
    }
    // out row . dot row, this wave's columns, to part[w * C + row]
    __device__ __forceinline__ void dot_rows(const Dots &d, float *part) const {
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            float sum = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float x;
                    if constexpr (sizeof(E) == 2) x = j & 1 ? bf16_hi_as_float(d.bits[it][c][j >> 1]) : bf16_lo_as_float(d.bits[it][c][j >> 1]);
                    else x = __builtin_bit_cast(float, d.bits[it][c][j]);
                    sum = fmaf(x, O[c][it][j], sum);
                }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0) part[w * C + it * 16 + lm] = sum;
        }
    }
    // rows of the chunk out of the accumulators
    __device__ __forceinline__ void store_rows(const Rows &r, int out_dtype, const Steps &st) const {
        const auto [lm, g] = fresh();
        const Rsrc b = chunk_view(r, st);
        uint32_t o[kI];
        if constexpr (FAST) st.offsets(o, lm, 16, (uint32_t)r.step, st.count, 0u);
#pragma unroll
        for (int it = 0; it < kI; ++it) {
            const int i = it * 16 + lm;
            if constexpr (FAST) {
                const uint32_t at = o[it];
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const int col = cols_of(c, g);
                    const f32x4 x = O[c][it];
                    if (out_dtype == GLA_DT_BF16)
                        put(b, col < r.d ? at + col * 2 : kNowhere, u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])});
                    else
                        put(b, col < r.d ? at + col * 4 : kNowhere, x);
                }
                continue;
            }
            if (i >= st.count) continue;
            char *row = const_cast<char *>(r.token((long long)st.first + st.at(i)));
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int col = cols_of(c, g);
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

// f(M, N, FAST) of the kernels for states of m x n
template <typename F>
hipError_t decay_sizes(int m, int n, bool fast, F f) {
    typedef std::integral_constant<int, 64> Small;
    typedef std::integral_constant<int, 128> Large;
    auto with = [&](auto quick) {
        if (m > 64) return n > 64 ? f(Large(), Large(), quick) : f(Large(), Small(), quick);
        return n > 64 ? f(Small(), Large(), quick) : f(Small(), Small(), quick);
    };
    return fast ? with(std::true_type()) : with(std::false_type());
}

}  // namespace
}  // namespace gla
