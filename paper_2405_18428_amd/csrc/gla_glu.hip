// Gated feed-forward product y = act(x Wg^T) * (x Wu^T) and its backward pass:
//   g = x Wg^T,  u = x Wu^T,   dg = dy u act'(g),  du = dy act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,  dWu = du^T x.
//
// One matrix product kernel serves all four products.  A work-group makes a BM x BN tile of the result from tiles of 128 bytes of the
// contraction (64 bf16 or 32 fp32 numbers), which go from memory to LDS directly, two of them in turn.  Operands are stored either with the
// contraction along their rows (x and the weights forward, dg and du for dx) or across them (the weights for dx, both for dW): the latter
// are transposed on their way from LDS to registers, by the 16-bit transposing read, or number by number in fp32, so that nothing is transposed in memory.
// Forward the tile's columns are some of Wg and the same ones of Wu, and a wave has both of its columns, so that the product needs no second pass.  Sums are
// fp32 MFMA accumulators; fp32 operands go through fp32 MFMA.
//
// What bounds it: the matrix units are busy 45 to 48 % of a large call.  8192 x 2048 x 8192, bf16, tiles of 256 x 256: both products with the activation, and
// their fp32 copies kept, 537 us (1024 TFLOP/s; in a row without pauses 501, without the copies 494), dx 532 (1033), both dW 502 (1095); products of these shapes by the
// vendor's library reach 1203, 1098 and 963.  Left without MFMAs dx takes 438 us, without loads 334, without LDS reads 444: tiles of the contraction come at 17 bytes a clock and compute unit,
// a fifth of their lines from beyond L2, and a tile is there when its slowest line is.  Tiles of 64 bytes, five of them under way, 650 us (lines
// are fetched twice); three tiles of A, two of B 533.  fp32, 1021 x 381 x 1531: 31 to 32 us
// a pair of products (75 TFLOP/s of the 154 that large ones reach): 768 short tiles of 64 x 64, ragged ones among them.
//
// bf16 calls round dg and du once, to bf16, as operands of the second pair of products: what they lose is as random as the rounding
// of the results and as large, so that gradients are off by 1.4 times their own rounding.  With GLA_OPT_GLU_SPLIT they are two numbers each, one segment of the contraction
// behind the other: 1.02 times and less, for a backward call of 2167 us instead of 1156 (8192 x 2048 x 8192; 1024 x 1152 x 4608 143 and 89).
#include "gla_glu.h"
#include "gla_mfma_util.h"

namespace gla {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void *lds_ptr;

constexpr int kTileBytes = 128;         // of a row of a tile, along the contraction
enum Product { kForward, kDx, kDw };

struct Activation {
    float y, slope;
};
template <bool SLOPE>
__device__ __forceinline__ Activation activation(int act, float g) {
    Activation r;
    r.slope = 0.f;
    if (act == GLA_ACT_SILU) {
        const float s = 1.f / (1.f + __builtin_amdgcn_exp2f(-1.44269504f * g));
        r.y = g * s;
        if constexpr (SLOPE) r.slope = s * fmaf(g, 1.f - s, 1.f);
    } else if (act == GLA_ACT_GELU) {
        const float phi = 0.5f * erfcf(-0.707106781f * g);
        r.y = g * phi;
        if constexpr (SLOPE) r.slope = fmaf(g * 0.398942280f, __builtin_amdgcn_exp2f(-0.721347520f * g * g), phi);
    } else {                            // g sigmoid(2 k (g + 0.044715 g^3)), k = sqrt(2 / pi)
        // (past |g| = 100, where s is 0 or 1, a larger square would only overflow; a NaN stays one by g)
        const float q = fminf(g * g, 1e4f), s = 1.f / (1.f + __builtin_amdgcn_exp2f(-2.30220819f * g * fmaf(0.044715f, q, 1.f)));
        r.y = g * s;
        // (and so would a larger g, whose slope's second term is 0 from there on)
        if constexpr (SLOPE) r.slope = s * fmaf((g < -100.f ? -100.f : g) * (1.f - s), 1.59576912f * fmaf(0.134145f, q, 1.f), 1.f);
    }
    return r;
}

struct ProductArgs {
    // operand rows: A has the result's rows, B its columns; second ones for what follows behind the first (see `Product`)
    const char *a[4], *b[2];
    int segments;                       // of the contraction, one behind the other: dx dg, du (and what is left of them), dW one (and that)
    long long lda, ldb;                 // bytes
    int M, N, K;                        // of the result (forward: N = F columns of each product) and of one contraction
    int tiles_m, tiles_n, splits;
    int act;
    void *out[2];                       // forward: [M, N]; dx: [M, N]; dW: two of [M, N]
    int out_dtype;
    float *pre, *part;
    // forward, where dg and du are wanted instead: [M, N], and two of [M, ld_f]
    const void *d_out;
    void *slope[2], *left[2];            // (left: null or what is left of them, bf16)
    int ld_f;
};

template <typename E> struct Frag;
template <> struct Frag<uint16_t> {
    u32x4 v;                            // eight numbers along the contraction
};
template <> struct Frag<float> {
    f32x4 v;                            // four
};
__device__ __forceinline__ f32x4 mma(const Frag<uint16_t> &n, const Frag<uint16_t> &m, f32x4 acc) {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, n.v), __builtin_bit_cast(bf16x8, m.v), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<float> &n, const Frag<float> &m, f32x4 acc) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n.v[j], m.v[j], acc, 0, 0, 0);
    return acc;
}

// A tile of one operand, ROWS of the result's rows or columns, in LDS, and what a lane loads and reads of it.
// Along (ACROSS = false): ROWS rows of 128 bytes, whose eight 16-byte pieces are exchanged by XOR with (row / 2) % 8, so that the 16 rows of a read meet
// all banks.  ACROSS: 64 (fp32: 32) rows of ROWS numbers, pieces exchanged by a number of the row's that differs between the rows of a read.
// PAIRED: the first half of the rows is one operand's, the second another's.
template <typename E, int ROWS, int WAVES, bool ACROSS, bool PAIRED>
struct Tile {
    static constexpr int kES = sizeof(E), kDepth = kTileBytes / kES, kBytes = ROWS * kTileBytes, kLoads = kBytes / 1024 / WAVES;
    static constexpr int kPieces = ROWS * kES / 16;              // of a row, ACROSS
    static constexpr int kReads = !ACROSS ? 1 : kES == 2 ? 2 : 4;
    uint32_t off[kLoads];               // of the lane's pieces from the operand's first one in the tile, or nowhere

    static __device__ __forceinline__ int turned(int k) { return (kES == 2 ? 2 * ((k & 3) | ((k >> 3) & 1) << 2) : 4 * ((k >> 2) & 3)) & (kPieces - 1); }
    // row of the tile and piece of the row for the i-th load of a lane
    static __device__ __forceinline__ void place(int i, int wave, int lane, int &row, int &piece) {
        const int id = (wave * kLoads + i) * 64 + lane;
        if constexpr (!ACROSS) {
            row = id >> 3;
            piece = (id & 7) ^ ((row >> 1) & 7);
        } else {
            row = id / kPieces;
            piece = (id % kPieces) ^ turned(row);
        }
    }
    static_assert(!ACROSS || (kPieces & (kPieces - 1)) == 0, "");
    static_assert(kLoads * WAVES * 1024 == kBytes && (!PAIRED || (!ACROSS && ROWS % 16 == 0)), "");
    // which of a pair a load is of
    static __device__ __forceinline__ int which(int i, int wave) { return PAIRED && (wave * kLoads + i) * (1024 / kTileBytes) >= ROWS / 2; }
    // `first`: the tile's first row or column of the result, `limit`: how many there are; `depth`: what is left of the contraction (kDepth and more:
    // a whole tile)
    __device__ __forceinline__ void plan(int wave, int lane, long long ld, int first, int limit, int depth) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int row, piece;
            place(i, wave, lane, row, piece);
            row -= which(i, wave) * (ROWS / 2);
            bool in;
            if constexpr (!ACROSS) {
                const int r = first + row;
                in = r < limit && piece * (16 / kES) < depth;
                off[i] = in ? (uint32_t)(row * ld + piece * 16) : kNowhere;
            } else {
                in = row < depth && first + piece * (16 / kES) < limit;
                off[i] = in ? (uint32_t)(row * ld + piece * 16) : kNowhere;
            }
        }
    }
    __device__ __forceinline__ void load(const char *base, const char *other, char *lds, int wave) const {
        const Rsrc one = view(base, 0x7fffffffu), two = view(PAIRED ? other : base, 0x7fffffffu);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(which(i, wave) ? two : one, (lds_ptr)(lds + (wave * kLoads + i) * 1024), 16, (int)off[i], 0, 0, 0);
    }
    // 16 rows or columns from `at` on (a multiple of 16), numbers kk of two of the contraction's halves
    static __device__ __forceinline__ Frag<E> read(const char *lds, int at, int kk, int lane) {
        const int l = lane & 15, g = lane >> 4;
        Frag<E> f;
        if constexpr (!ACROSS) {
            f.v = *reinterpret_cast<const decltype(f.v) *>(lds + (at + l) * kTileBytes + (((4 * kk + g) ^ ((l >> 1) & 7)) << 4));
        } else if constexpr (kES == 2) {
            const int k = 32 * kk + 8 * g + (l >> 2);
            const char *p = lds + k * (ROWS * 2) + ((((at >> 4) ^ (turned(k) >> 1)) << 5) | ((l & 3) << 3));
            typedef __attribute__((address_space(3))) s16x4 *lds_s4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p + 4 * ROWS * 2));
            const u32x2 x = __builtin_bit_cast(u32x2, lo), y = __builtin_bit_cast(u32x2, hi);
            f.v = u32x4{x[0], x[1], y[0], y[1]};
        } else {
            const int k = 16 * kk + 4 * g;
            const char *p = lds + k * (ROWS * 4) + ((((at >> 4) ^ g) << 6) | (l << 2));
#pragma unroll
            for (int j = 0; j < 4; ++j) f.v[j] = *reinterpret_cast<const float *>(p + j * ROWS * 4);
        }
        return f;
    }
};

// Four neighbouring results to a row of a tensor of n columns
__device__ __forceinline__ void store4(void *base, int dtype, long long row, int col, int n, f32x4 v) {
    if (dtype == GLA_DT_BF16) {
        uint16_t *p = static_cast<uint16_t *>(base) + row * n + col;
        const u32x2 b = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        if (n % 4 == 0) {
            *reinterpret_cast<u32x2 *>(p) = b;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < n) p[i] = (uint16_t)(b[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        float *p = static_cast<float *>(base) + row * n + col;
        if (n % 4 == 0) {
            *reinterpret_cast<f32x4 *>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < n) p[i] = v[i];
        }
    }
}

// Four fp32 numbers that nothing reads soon, and that are too many for the last-level cache: with it full of them, what comes after waits for their way to memory
// (8192 x 2048 x 8192: both products kept, 517 us for 585 forward, 163 for 192 where they are read)
__device__ __forceinline__ void keep4(float *base, long long row, int col, int n, f32x4 v) {
    if (n % 4 == 0) __builtin_nontemporal_store(v, reinterpret_cast<f32x4 *>(base + row * n + col));
    else store4(base, GLA_DT_F32, row, col, n, v);
}

// Eight
__device__ __forceinline__ void store8(void *base, int dtype, long long row, int col, int n, f32x4 v, f32x4 w) {
    if (dtype == GLA_DT_BF16 && n % 8 == 0) {
        if (col < n)
            *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(base) + row * n + col) =
                u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3])};
        return;
    }
    if (col < n) store4(base, dtype, row, col, n, v);
    if (col + 4 < n) store4(base, dtype, row, col + 4, n, w);
}

// dg = dy u act'(g), du = dy act(g) of four neighbouring columns, those from n on as zeros; dy [., n]
template <typename E>
__device__ __forceinline__ void slopes(int act, const E *d_out, long long row, int col, int n, f32x4 g, f32x4 u, f32x4 &dg, f32x4 &du) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const E *p = d_out + row * n + col;
    if (n % 4 == 0) {
        if (col < n) {
            if constexpr (sizeof(E) == 2) {
                const u32x2 b = *reinterpret_cast<const u32x2 *>(p);
                o = f32x4{bf16_lo_as_float(b[0]), bf16_hi_as_float(b[0]), bf16_lo_as_float(b[1]), bf16_hi_as_float(b[1])};
            } else {
                o = *reinterpret_cast<const f32x4 *>(p);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < n) {
                if constexpr (sizeof(E) == 2) o[i] = bf16_bits_to_float(p[i]);
                else o[i] = p[i];
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Activation a = activation<true>(act, g[i]);
        dg[i] = col + i < n ? o[i] * u[i] * a.slope : 0.f;
        du[i] = col + i < n ? o[i] * a.y : 0.f;
    }
}

// What a number has left when it is rounded to bf16 (nothing, where that is not finite), and four of them
__device__ __forceinline__ float left_of(float x) {
    const float r = bf16_lo_as_float(pack_bf16(x, 0.f));
    return __builtin_fabsf(r) < __builtin_inff() ? x - r : 0.f;
}
__device__ __forceinline__ f32x4 left_of(f32x4 v) { return f32x4{left_of(v[0]), left_of(v[1]), left_of(v[2]), left_of(v[3])}; }

// Tiles of a work-group: work-groups go to the eight XCDs by turns, so each XCD gets a run of tiles, and a run goes down eight rows of tiles
// before it goes on to the next column, so that what an XCD reads at a time stays in its L2.
__device__ __forceinline__ void tile_of(const ProductArgs &p, int &tm, int &tn) {
    const int count = p.tiles_m * p.tiles_n, id = blockIdx.x;
    const int xcd = id & 7, each = count >> 3, more = count & 7;
    const int t = xcd * each + min(xcd, more) + (id >> 3);
    constexpr int kDown = 8;
    const int band = t / (kDown * p.tiles_n), in = t - band * kDown * p.tiles_n;
    const int high = min(kDown, p.tiles_m - band * kDown);
    tn = in / high;
    tm = band * kDown + in - tn * high;
}

template <typename E, Product P, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(const ProductArgs p) {
    constexpr int kWaves = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    static_assert(P != kForward || NI % 2 == 0, "as many columns of each product a wave");
    constexpr int kES = sizeof(E);
    using TA = Tile<E, BM, kWaves, P == kDw, false>;
    using TB = Tile<E, BN, kWaves, P != kForward, P == kForward>;
    constexpr int kDepth = TA::kDepth;
    __shared__ __attribute__((aligned(1024))) char lds[2][TA::kBytes + TB::kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wm = wave / WN, wn = wave - wm * WN;
    int tm, tn;
    tile_of(p, tm, tn);
    // dW: tiles of the first matrix' rows, then those of the second
    const int half_tiles = p.tiles_m / 2, which = P == kDw ? tm >= half_tiles : 0;
    const int m0 = (P == kDw ? tm - which * half_tiles : tm) * BM, n0 = tn * (P == kForward ? BN / 2 : BN);

    // tiles of the contraction, those of one segment behind those of the other
    const int tiles = (p.K + kDepth - 1) / kDepth, all = P == kForward ? tiles : p.segments * tiles;
    const int each = (all + p.splits - 1) / p.splits, t0 = min((int)blockIdx.y * each, all), t1 = min(t0 + each, all);
    TA ta;
    TB tb;
    ta.plan(wave, lane, p.lda, m0, p.M, kDepth);
    tb.plan(wave, lane, p.ldb, n0, p.N, kDepth);
    auto load = [&](int t, int buf) __attribute__((always_inline)) {
        const int seg = P == kForward ? 0 : P == kDw ? t >= tiles : (t >= tiles) + (t >= 2 * tiles) + (t >= 3 * tiles), k0 = (t - seg * tiles) * kDepth;
        const char *a = p.a[P == kDw ? which + 2 * seg : seg] + (P == kDw ? k0 * p.lda + (long long)m0 * kES : m0 * p.lda + (long long)k0 * kES);
        const char *b = p.b[P == kDx ? seg & 1 : 0] + (P == kForward ? n0 * p.ldb + (long long)k0 * kES : k0 * p.ldb + (long long)n0 * kES);
        const char *other = P == kForward ? p.b[1] + n0 * p.ldb + (long long)k0 * kES : nullptr;
        char *at = lds[buf];
        if (k0 + kDepth <= p.K) {
            ta.load(a, nullptr, at, wave);
            tb.load(b, other, at + TA::kBytes, wave);
        } else {
            TA ea;
            TB eb;
            ea.plan(wave, lane, p.lda, m0, p.M, p.K - k0);
            eb.plan(wave, lane, p.ldb, n0, p.N, p.K - k0);
            ea.load(a, nullptr, at, wave);
            eb.load(b, other, at + TA::kBytes, wave);
        }
    };
    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Fragments of a tile's two halves.  The products of one half run while the other half's fragments are read: in the first phase those of the same
    // tile's second half, in the second, behind the barrier that says that the next tile has come and that this one is read, those of the next tile's
    // first half, while the tile after that is loaded over this one.
    Frag<E> fa[2][MI], fb[2][NI];
    auto read = [&](auto half, int buf) __attribute__((always_inline)) {
        constexpr int kk = decltype(half)::value;
        const char *at = lds[buf], *bt = at + TA::kBytes;
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            if constexpr (P == kForward) fb[kk][j] = TB::read(bt, j / (NI / 2) * (BN / 2) + (wn * (NI / 2) + j % (NI / 2)) * 16, kk, lane);
            else fb[kk][j] = TB::read(bt, (wn * NI + j) * 16, kk, lane);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[kk][i] = TA::read(at, (wm * MI + i) * 16, kk, lane);
    };
    auto multiply = [&](auto half) __attribute__((always_inline)) {
        constexpr int kk = decltype(half)::value;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mma(fb[kk][j], fa[kk][i], acc[i][j]);
        // a read after every few products
        constexpr int kReads = NI * TB::kReads + MI * TA::kReads, kProducts = MI * NI * (kES == 2 ? 1 : 4), kBetween = kProducts / kReads;
#pragma unroll
        for (int n = 0; n < kReads; ++n) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, kBetween, 0);
        }
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    // every wave's loads have arrived in LDS, and its reads in registers (a barrier by itself does not wait for the former)
    auto meet = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    if (t0 < t1) load(t0, 0);
    if (t0 + 1 < t1) load(t0 + 1, 1);
    meet();
    read(first, 0);
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        read(second, buf);
        multiply(first);
        meet();
        if (t + 2 < t1) load(t + 2, buf);
        read(first, buf ^ 1);            // (behind the last tile: of no use)
        multiply(second);
    }
    __syncthreads();
    // The tile goes through LDS, some rows of each wave at a time, so that a work-group stores whole rows and each result's code stands here once.
    // A lane has four neighbouring columns of one row of each 16 x 16 piece; pieces of 16 bytes are exchanged by XOR with the row.
    constexpr int kRows = (int)sizeof(lds) >= BM * BN * 4 ? BM : BM / 2, kPasses = BM / kRows, kSub = MI / kPasses;
    static_assert(kSub * kPasses == MI && kRows * BN * 4 <= (int)sizeof(lds) && BN % 64 == 0, "");
    char *const tile = lds[0];
    const int l = lane & 15, g = lane >> 4;
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
        if (pass > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < kSub; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = (wm * kSub + i) * 16 + l, piece = (wn * NI + j) * 4 + g;
                *reinterpret_cast<f32x4 *>(tile + r * (BN * 4) + ((piece ^ l) << 4)) = acc[pass * kSub + i][j];
            }
        __syncthreads();
        // four at column c of the tile
        auto at = [&](int r, int c) { return *reinterpret_cast<const f32x4 *>(tile + r * (BN * 4) + (((c >> 2) ^ (r & 15)) << 4)); };
        // columns a thread: 16 bytes of results, or of what is stored in fp32, so that a wave's store leaves no holes in lines
        auto results = [&](auto columns) __attribute__((always_inline)) {
            constexpr int kColumns = decltype(columns)::value, kThreadsARow = (P == kForward ? BN / 2 : BN) / kColumns;
#pragma unroll 1
            for (int item = threadIdx.x; item < kRows * kThreadsARow; item += 64 * kWaves) {
                const int r = item / kThreadsARow, col = item % kThreadsARow * kColumns, n = n0 + col;
                const int sub = r >> 4, m = m0 + ((sub / kSub) * MI + pass * kSub + sub % kSub) * 16 + (r & 15);
                if (m >= p.M) continue;
                if constexpr (P == kForward) {
                    const int c = col / (NI * 8) * NI * 16 + col % (NI * 8);
                    f32x4 y[kColumns / 4];
#pragma unroll
                    for (int h = 0; h < kColumns / 4; ++h) {
                        const f32x4 gt = at(r, c + 4 * h), up = at(r, c + NI * 8 + 4 * h);
                        if (kColumns == 4 && p.d_out != nullptr) {
                            if (n >= p.ld_f) continue;
                            f32x4 dg, du;
                            slopes<E>(p.act, static_cast<const E *>(p.d_out), m, n, p.N, gt, up, dg, du);
                            store4(p.slope[0], kES == 2 ? GLA_DT_BF16 : GLA_DT_F32, m, n, p.ld_f, dg);
                            store4(p.slope[1], kES == 2 ? GLA_DT_BF16 : GLA_DT_F32, m, n, p.ld_f, du);
                            if (kES == 2 && p.left[0] != nullptr) {
                                store4(p.left[0], GLA_DT_BF16, m, n, p.ld_f, left_of(dg));
                                store4(p.left[1], GLA_DT_BF16, m, n, p.ld_f, left_of(du));
                            }
                            continue;
                        }
                        if (kColumns == 4 && p.pre != nullptr && n < p.N) {
                            keep4(p.pre, m, n, p.N, gt);
                            keep4(p.pre + (long long)p.M * p.N, m, n, p.N, up);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[h][e] = activation<false>(p.act, gt[e]).y * up[e];
                    }
                    if constexpr (kColumns == 8) {
                        store8(p.out[0], p.out_dtype, m, n, p.N, y[0], y[1]);
                    } else {
                        if (p.d_out == nullptr && n < p.N) store4(p.out[0], p.out_dtype, m, n, p.N, y[0]);
                    }
                } else if constexpr (kColumns == 8) {
                    store8(p.out[which], p.out_dtype, m, n, p.N, at(r, col), at(r, col + 4));
                } else if (n < p.N) {
                    if (p.splits > 1) store4(p.part + (blockIdx.y * (P == kDw ? 2LL : 1LL) + which) * p.M * p.N, GLA_DT_F32, m, n, p.N, at(r, col));
                    else store4(p.out[which], p.out_dtype, m, n, p.N, at(r, col));
                }
            }
        };
        if (p.out_dtype == GLA_DT_BF16 && p.splits == 1 && p.pre == nullptr && p.d_out == nullptr) results(std::integral_constant<int, 8>{});
        else results(std::integral_constant<int, 4>{});
    }
}

// Forward for few rows, where the weights' reading is all: a work-group has 16 NT columns of both products, its waves a part of K each, whose weights go
// from memory to the matrix units' registers; rows of x, which all work-groups share, come from L2.  The waves' sums meet in LDS.  MT: tiles of 16 rows.
// Bound by HBM and by how short it is: one row of 2048 x 8192, bf16, 67 MB, 15.2 us from HBM, 64 sets of weights in turn (13.0 at a copy's rate), 12.4 where the
// weights are in the last-level cache; 33 rows 22.3 and 17.8; of 4096 x 16384 one row 49 us for 52, 33 rows 71.  Comparisons here and below are of short graphs with weights from
// HBM, whose starts add some 3 us a call: one row 18.6; eight pieces a wave under way instead of four 19.0, 16 rows 21.4 for 20.9.
template <typename E, int WAVES, int MT, int NT>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(const ProductArgs p) {
    constexpr int kES = sizeof(E), kAhead = MT + 2 * NT <= 8 ? 4 : 2;
    __shared__ f32x4 sums[WAVES][2 * NT * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l = lane & 15, g = lane >> 4;
    const int f0 = blockIdx.x * 16 * NT;
    const Rsrc rw[2] = {view(p.b[0] + f0 * p.ldb, 0x7fffffffu), view(p.b[1] + f0 * p.ldb, 0x7fffffffu)}, rx = view(p.a[0], 0x7fffffffu);
    // steps of 64 bytes of a row
    const int steps = (p.K * kES + 63) / 64, each = (steps + WAVES - 1) / WAVES, s0 = wave * each, s1 = min(s0 + each, steps);
    f32x4 acc[2 * NT][MT];
#pragma unroll
    for (int n = 0; n < 2 * NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = s0; s < s1; s += kAhead) {
        Frag<E> w[kAhead][2 * NT], x[kAhead][MT];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int at = (s + k) * 64 + g * 16;
            const bool in = s + k < s1 && at < p.K * kES;
#pragma unroll
            for (int n = 0; n < 2 * NT; ++n) {
                const int row = (n >> 1) * 16 + l;
                w[k][n].v = fetch<decltype(w[k][n].v)>(rw[n & 1], in && f0 + row < p.N ? (uint32_t)(row * p.ldb) + at : kNowhere);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
                x[k][m].v = fetch<decltype(x[k][m].v)>(rx, in && m * 16 + l < p.M ? (uint32_t)((m * 16 + l) * p.lda) + at : kNowhere);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < 2 * NT; ++n) acc[n][m] = mma(w[k][n], x[k][m], acc[n][m]);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < 2 * NT; ++n) sums[wave][m * 2 * NT + n][lane] = acc[n][m];
    __syncthreads();
    for (int i = wave; i < MT * NT; i += WAVES) {
        f32x4 gt = sums[0][2 * i][lane], up = sums[0][2 * i + 1][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) {
            gt += sums[k][2 * i][lane];
            up += sums[k][2 * i + 1][lane];
        }
        const int row = i / NT * 16 + l, n = f0 + i % NT * 16 + 4 * g;
        if (row >= p.M || n >= p.N) continue;
        if (p.pre != nullptr) {
            store4(p.pre, GLA_DT_F32, row, n, p.N, gt);
            store4(p.pre + (long long)p.M * p.N, GLA_DT_F32, row, n, p.N, up);
        }
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = activation<false>(p.act, gt[e]).y * up[e];
        store4(p.out[0], p.out_dtype, row, n, p.N, y);
    }
}

// dx, or both dW, from the parts of their sums, added in one order; four numbers a thread.  Bound by latency at the sizes that are summed in parts:
// 1021 x 381 from 10 parts, or two of 1531 x 381 from 3 each, 6.8 us
struct JoinArgs {
    const float *part;                  // [splits, tensors, count]
    void *out[2];
    long long count;
    int dtype, splits;
};
__global__ __launch_bounds__(256) void join_kernel(const JoinArgs p) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4, stride = p.count * gridDim.y;
    if (at >= p.count) return;
    const float *part = p.part + p.count * blockIdx.y + at;
    void *out = p.out[blockIdx.y];
    if (p.count % 4 == 0) {
        f32x4 s = *reinterpret_cast<const f32x4 *>(part);
#pragma unroll 4
        for (int i = 1; i < p.splits; ++i) s += *reinterpret_cast<const f32x4 *>(part + i * stride);
        if (p.dtype == GLA_DT_BF16) *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(out) + at) = u32x2{pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3])};
        else *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + at) = s;
        return;
    }
    const int n = (int)min(4LL, p.count - at);
    float s[4] = {};
#pragma unroll 4
    for (int i = 0; i < p.splits; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += e < n ? part[i * stride + e] : 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= n) continue;
        if (p.dtype == GLA_DT_BF16) static_cast<uint16_t *>(out)[at + e] = (uint16_t)pack_bf16(s[e], 0.f);
        else static_cast<float *>(out)[at + e] = s[e];
    }
}

// dg and du of the two products that a forward call has kept: four columns a thread, those from F to the end of a row as zeros.  Bound by HBM: 8192 x 8192, bf16,
// 940 MB, 152 us, 6.2 TB/s with what is still in the last-level cache
template <typename E>
__global__ __launch_bounds__(256) void slopes_kernel(const GluCall c, const float *pre) {
    const int pieces = c.ld_f / 4;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long m = id / pieces;
    const int f = (int)(id - m * pieces) * 4;
    if (m >= c.M) return;
    const float *g = pre + m * c.F + f, *u = g + (long long)c.M * c.F;
    f32x4 gt = {0, 0, 0, 0}, up = gt, dg, du;
    if (c.F % 4 == 0) {
        if (f < c.F) {
            gt = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(g));     // (the last that reads them: 162 -> 153 us)
            up = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(u));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (f + i < c.F) {
                gt[i] = g[i];
                up[i] = u[i];
            }
    }
    slopes<E>(c.act, static_cast<const E *>(c.d_out), m, f, c.F, gt, up, dg, du);
    store4(c.dg[0], c.dtype, m, f, c.ld_f, dg);
    store4(c.du[0], c.dtype, m, f, c.ld_f, du);
    if (sizeof(E) == 2 && c.split()) {
        store4(c.dg[1], c.dtype, m, f, c.ld_f, left_of(dg));
        store4(c.du[1], c.dtype, m, f, c.ld_f, left_of(du));
    }
}

// Rows of `cols` elements to rows of `ld`, zeros behind: three tensors in one launch, four rows a work-group at a time.  Direct loads to LDS take pieces of 16
// bytes from addresses of as many; 1021, 1531 and 1531 rows of 381 floats 5.6 us, twice in a training step of 119
struct PadArgs {
    const void *from[3];
    void *to[3];
    int rows[3], cols, ld;
};
constexpr int kPadRows = 4, kPadGroups = 1 << 16;
template <typename E>
__global__ __launch_bounds__(256) void pad_kernel(const PadArgs p) {
    const int which = blockIdx.y, rows = p.rows[which];
    const E *from = static_cast<const E *>(p.from[which]);
    E *to = static_cast<E *>(p.to[which]);
    for (long long r0 = (long long)blockIdx.x * kPadRows; r0 < rows; r0 += (long long)gridDim.x * kPadRows)
        for (int c = threadIdx.x; c < p.ld; c += 256) {
#pragma unroll
            for (int i = 0; i < kPadRows; ++i) {
                const long long r = r0 + i;
                if (r < rows) to[r * p.ld + c] = c < p.cols ? from[r * p.cols + c] : (E)0;
            }
        }
}

template <typename E, Product P, int BM, int BN, int WM, int WN>
hipError_t product(ProductArgs p, hipStream_t stream) {
    p.tiles_m = (p.M + BM - 1) / BM * (P == kDw ? 2 : 1);
    const int wide = P == kForward ? BN / 2 : BN;
    p.tiles_n = (p.N + wide - 1) / wide;
    hipLaunchKernelGGL((product_kernel<E, P, BM, BN, WM, WN>), dim3((unsigned)p.tiles_m * (unsigned)p.tiles_n, (unsigned)p.splits), dim3(64 * WM * WN), 0,
                       stream, p);
    return hipGetLastError();
}
// How a product is cut: tiles, and for dx the parts of its sum.  The cheapest by a model of rounds of tiles: microseconds a tile and step of the contraction
// (64 bf16 or 32 fp32 numbers), measured with every compute unit at work on 8192 x 2048 x 16384, and what a tile takes at its ends.  Where tiles
// of 256 x 256 leave the last round nearly empty others are ahead: 4096 x 1152 x 9216 107 us, in tiles of 256 x 192 95, of 128 x 128 101;
// 2048 rows 72, 60, 59; 1024 x 2048 x 16384 62, 87, 72.
enum { kBig, kWide, kSmall, kTiny };     // 256 x 256, 256 x 192 (forward), 128 x 128 (two on a compute unit), 64 x 64 (four)
struct Plan {
    int tile, splits;
};
Plan plan_of(Product product, long long M, long long N, long long K, int segments, int dtype) {
    constexpr int kHigh[] = {256, 256, 128, 64}, kAcross[] = {256, 192, 128, 64}, kSlots[] = {256, 256, 512, 1024};
    constexpr double kStep[2][4] = {{1.95, 1.48, 1.08, 0.75}, {7.4, 5.6, 3.9, 2.1}}, kEnds = 6, kJoin = 5, kBytesAUs = 4e6;
    const int depth = kTileBytes / (dtype == GLA_DT_BF16 ? 2 : 4);
    const long long steps = (K + depth - 1) / depth * segments;
    Plan best = {kBig, 1};
    double least = 1e300;
    for (int tile = kBig; tile <= kTiny; ++tile) {
        if (tile == kWide && product != kForward) continue;
        const long long high = (M + kHigh[tile] - 1) / kHigh[tile] * (product == kDw ? 2 : 1), tiles = high * ((N + kAcross[tile] - 1) / kAcross[tile]);
        for (int s = 1; s <= (product == kForward ? 1 : 16) && (s == 1 || steps / s >= 4); ++s) {
            const double rounds = (double)((tiles * s + kSlots[tile] - 1) / kSlots[tile]);
            const double us = rounds * ((double)((steps + s - 1) / s) * kStep[dtype == GLA_DT_BF16 ? 0 : 1][tile] + kEnds) +
                              (s > 1 ? kJoin + (double)s * M * N * (product == kDw ? 16 : 8) / kBytesAUs : 0.);
            if (us < least) {
                least = us;
                best = {tile, s};
            }
        }
    }
    return best;
}

template <Product P>
hipError_t product_of(const ProductArgs &p, int dtype, hipStream_t stream) {
    const Plan plan = plan_of(P, p.M, P == kForward ? 2LL * p.N : p.N, p.K, p.segments, dtype);
    auto run = [&](auto e) {
        using E = decltype(e);
        if constexpr (P == kForward) {
            if (plan.tile == kWide) return product<E, P, 256, 192, 4, 2>(p, stream);
        }
        if (plan.tile == kBig) return product<E, P, 256, 256, 2, 4>(p, stream);
        return plan.tile == kSmall ? product<E, P, 128, 128, 2, 2>(p, stream) : product<E, P, 64, 64, 2, 2>(p, stream);
    };
    return dtype == GLA_DT_BF16 ? run(uint16_t{}) : run(float{});
}
int element(int dtype) { return dtype == GLA_DT_BF16 ? 2 : 4; }

}  // namespace

static ProductArgs forward_args(const GluCall &c) {
    ProductArgs p = {};
    p.a[0] = static_cast<const char *>(c.x);
    p.b[0] = static_cast<const char *>(c.w_gate);
    p.b[1] = static_cast<const char *>(c.w_up);
    p.lda = (long long)c.ld_x * element(c.dtype);
    p.ldb = (long long)c.ld_w * element(c.dtype);
    p.M = c.M;
    p.N = c.F;
    p.K = c.ld_x;                        // (columns behind K are zeros)
    p.segments = 1;
    p.splits = 1;
    p.act = c.act;
    return p;
}

// Up to so many rows (2048 x 8192, bf16: 64 rows 21 us, in tiles of 128 x 128 27, 100 rows 37 and 29; fp32: 128 rows 95 and 139)
constexpr int kFewRows16 = 64, kFewRows32 = 128;
template <typename E>
static hipError_t few_rows(const ProductArgs &p, hipStream_t stream) {
    const int tiles = (p.N + 15) / 16;
    auto run = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        // two work-groups a compute unit and more; with fewer columns more waves, each with less of K (weights from HBM, 4 waves and 8: one row, 8192 x 2048 29 us
        // and 25; 2048 x 8192 18.7 and 19.0, 16 rows 20.8 and 21.8)
        if constexpr (MT == 3 || MT == 4) {              // (two tiles of columns for each reading of x: 64 rows 24 -> 20.6 us)
            if (tiles >= 512) {
                hipLaunchKernelGGL((few_rows_kernel<E, 8, MT, 2>), dim3((unsigned)(tiles + 1) / 2), dim3(512), 0, stream, p);
                return hipGetLastError();
            }
        }
        if (MT > 4 || tiles >= 512) hipLaunchKernelGGL((few_rows_kernel<E, 4, MT, 1>), dim3((unsigned)tiles), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((few_rows_kernel<E, 8, MT <= 4 ? MT : 1, 1>), dim3((unsigned)tiles), dim3(512), 0, stream, p);
        return hipGetLastError();
    };
    if (p.M <= 16) return run(std::integral_constant<int, 1>{});
    if (p.M <= 32) return run(std::integral_constant<int, 2>{});
    if (p.M <= 48) return run(std::integral_constant<int, 3>{});
    if (sizeof(E) == 2 || p.M <= 64) return run(std::integral_constant<int, 4>{});
    return run(std::integral_constant<int, sizeof(E) == 2 ? 4 : 8>{});
}

hipError_t launch_glu_fwd(const GluCall &c, void *out, int out_dtype, float *pre, hipStream_t stream) {
    ProductArgs p = forward_args(c);
    p.out[0] = out;
    p.out_dtype = out_dtype;
    p.pre = pre;
    if (c.dtype == GLA_DT_BF16 && p.M <= kFewRows16) return few_rows<uint16_t>(p, stream);
    if (c.dtype == GLA_DT_F32 && p.M <= kFewRows32) return few_rows<float>(p, stream);
    return product_of<kForward>(p, c.dtype, stream);
}

hipError_t launch_glu_slopes(const GluCall &c, const float *pre, hipStream_t stream) {
    if (pre == nullptr) {                // the two products again
        ProductArgs p = forward_args(c);
        p.d_out = c.d_out;
        p.slope[0] = c.dg[0];
        p.slope[1] = c.du[0];
        p.left[0] = c.dg[1];
        p.left[1] = c.du[1];
        p.ld_f = c.ld_f;
        return product_of<kForward>(p, c.dtype, stream);
    }
    const long long threads = (long long)c.M * (c.ld_f / 4);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (c.dtype == GLA_DT_BF16) hipLaunchKernelGGL(slopes_kernel<uint16_t>, grid, dim3(256), 0, stream, c, pre);
    else hipLaunchKernelGGL(slopes_kernel<float>, grid, dim3(256), 0, stream, c, pre);
    return hipGetLastError();
}

size_t glu_part_bytes(int M, int K, int F, int dtype, bool split) {
    const int each = split ? 2 : 1, dx = plan_of(kDx, M, K, F, 2 * each, dtype).splits, dw = plan_of(kDw, F, K, M, each, dtype).splits;
    const size_t a = dx > 1 ? (size_t)dx * M * K : 0, b = dw > 1 ? (size_t)dw * 2 * F * K : 0;
    return (a > b ? a : b) * sizeof(float);
}
// A product whose sum may be taken in parts
template <Product P>
static hipError_t in_parts(ProductArgs p, int dtype, hipStream_t stream) {
    p.splits = plan_of(P, p.M, p.N, p.K, p.segments, dtype).splits;
    const hipError_t e = product_of<P>(p, dtype, stream);
    if (e != hipSuccess || p.splits == 1) return e;
    const JoinArgs j = {p.part, {p.out[0], p.out[1]}, (long long)p.M * p.N, dtype, p.splits};
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)((j.count + 1023) / 1024), P == kDw ? 2 : 1), dim3(256), 0, stream, j);
    return hipGetLastError();
}

hipError_t launch_glu_dx(const GluCall &c, void *dx, hipStream_t stream) {
    ProductArgs p = {};
    const int each = c.split() ? 2 : 1;
    for (int i = 0; i < each; ++i) {
        p.a[2 * i] = static_cast<const char *>(c.dg[i]);
        p.a[2 * i + 1] = static_cast<const char *>(c.du[i]);
    }
    p.b[0] = static_cast<const char *>(c.w_gate);
    p.b[1] = static_cast<const char *>(c.w_up);
    p.lda = (long long)c.ld_f * element(c.dtype);
    p.ldb = (long long)c.ld_w * element(c.dtype);
    p.M = c.M;
    p.N = c.K;
    p.K = c.F;
    p.segments = 2 * each;
    p.out[0] = dx;
    p.out_dtype = c.dtype;
    p.part = c.part;
    return in_parts<kDx>(p, c.dtype, stream);
}

hipError_t launch_glu_dw(const GluCall &c, void *dw_gate, void *dw_up, hipStream_t stream) {
    ProductArgs p = {};
    const int each = c.split() ? 2 : 1;
    for (int i = 0; i < each; ++i) {
        p.a[2 * i] = static_cast<const char *>(c.dg[i]);
        p.a[2 * i + 1] = static_cast<const char *>(c.du[i]);
    }
    p.b[0] = static_cast<const char *>(c.x);
    p.lda = (long long)c.ld_f * element(c.dtype);
    p.ldb = (long long)c.ld_x * element(c.dtype);
    p.M = c.F;
    p.N = c.K;
    p.K = c.M;
    p.segments = each;
    p.out[0] = dw_gate;
    p.out[1] = dw_up;
    p.out_dtype = c.dtype;
    p.part = c.part;
    return in_parts<kDw>(p, c.dtype, stream);
}

hipError_t launch_glu_pad(const GluCall &c, const void *x, const void *w_gate, const void *w_up, hipStream_t stream) {
    const PadArgs p = {{x, w_gate, w_up}, {const_cast<void *>(c.x), const_cast<void *>(c.w_gate), const_cast<void *>(c.w_up)}, {c.M, c.F, c.F}, c.K, c.ld_x};
    const int most = c.M > c.F ? c.M : c.F, groups = (most + kPadRows - 1) / kPadRows;
    const dim3 grid((unsigned)(groups < kPadGroups ? groups : kPadGroups), 3);
    if (c.dtype == GLA_DT_BF16) hipLaunchKernelGGL(pad_kernel<uint16_t>, grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(pad_kernel<float>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace gla
