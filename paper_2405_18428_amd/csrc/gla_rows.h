// Eight neighbouring channels of a row as floats, from and to memory (gfx950 device code).
#pragma once
#include "gla_common.h"

namespace gla {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kEach = 8;             // channels of a piece

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

// Eight channels as they lie in memory
template <typename E> struct Raw;
template <> struct Raw<uint16_t> { u32x4 v; };
template <> struct Raw<float> { f32x4 v[2]; };

// Channels c0 .. c0 + 7 of a row of D, those from D on as zeros
template <typename E>
__device__ __forceinline__ Raw<E> load_raw(const char *row, int c0, int D) {
    Raw<E> x = {};
    if (c0 + kEach <= D) {
        __builtin_memcpy(&x, row + c0 * (int)sizeof(E), sizeof(x));
    } else if (c0 < D && D >= kEach) {                   // the row's last eight, moved down (element by element D = 36 took twice as long)
        __builtin_memcpy(&x, row + (D - kEach) * (int)sizeof(E), sizeof(x));
        const int over = c0 + kEach - D;
        if constexpr (sizeof(E) == 2) {
            x.v = __builtin_bit_cast(u32x4, __builtin_bit_cast(unsigned __int128, x.v) >> (16 * over));
        } else {
            float e[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) e[j] = x.v[j >> 2][j & 3];
#pragma unroll
            for (int k = 4; k > 0; k /= 2)
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    if (over & k) e[j] = j + k < kEach ? e[j + k] : 0.f;
#pragma unroll
            for (int j = 0; j < kEach; ++j) x.v[j >> 2][j & 3] = e[j];
        }
    } else if (c0 < D) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (c0 + j < D) {
                if constexpr (sizeof(E) == 2) x.v[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c0 + j] << (16 * (j & 1));
                else x.v[j >> 2][j & 3] = reinterpret_cast<const float *>(row)[c0 + j];
            }
    }
    return x;
}
template <typename E>
__device__ __forceinline__ void to_floats(const Raw<E> &r, float (&x)[kEach]) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        if constexpr (sizeof(E) == 2) x[j] = j & 1 ? __builtin_bit_cast(float, r.v[j >> 1] & 0xffff0000u) : __builtin_bit_cast(float, r.v[j >> 1] << 16);
        else x[j] = r.v[j >> 2][j & 3];
    }
}
template <typename E>
__device__ __forceinline__ void load_piece(const char *row, int c0, int D, float (&x)[kEach]) {
    to_floats<E>(load_raw<E>(row, c0, D), x);
}
__device__ __forceinline__ void store_piece(char *row, int c0, int D, int dtype, const float (&x)[kEach]) {
    if (c0 + kEach <= D) {
        if (dtype == GLA_DT_BF16) {
            const u32x4 b = {pack(x[0], x[1]), pack(x[2], x[3]), pack(x[4], x[5]), pack(x[6], x[7])};
            __builtin_memcpy(row + c0 * 2, &b, 16);
        } else {
            const f32x4 v[2] = {{x[0], x[1], x[2], x[3]}, {x[4], x[5], x[6], x[7]}};
            __builtin_memcpy(row + c0 * 4, v, 32);
        }
        return;
    }
    int from = 0;
    if (c0 + 4 <= D) {
        if (dtype == GLA_DT_BF16) {
            const u32x2 b = {pack(x[0], x[1]), pack(x[2], x[3])};
            __builtin_memcpy(row + c0 * 2, &b, 8);
        } else {
            const f32x4 v = {x[0], x[1], x[2], x[3]};
            __builtin_memcpy(row + c0 * 4, &v, 16);
        }
        from = 4;
    }
    if (c0 + from >= D) return;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (j >= from && c0 + j < D) {
            if (dtype == GLA_DT_BF16) reinterpret_cast<uint16_t *>(row)[c0 + j] = (uint16_t)pack(x[j], 0.f);
            else reinterpret_cast<float *>(row)[c0 + j] = x[j];
        }
}

}  // namespace
}  // namespace gla
