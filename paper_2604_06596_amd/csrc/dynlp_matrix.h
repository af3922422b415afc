// Fragments of matrix products and what surrounds them: v_mfma_f32_16x16x{32,4}, rows by pieces, sums over the lanes of a row, bfloat16 terms.
#pragma once

#include "dynlp_device.h"
#include "dynlp_types.h"

namespace dynlp {

// acc += left * right over a piece of each.
__device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 c, bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 c, f16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ inline f32x4 mma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mma(u32x4 a, u32x4 b, f32x4 c, float) {
    for (int k = 0; k < 4; ++k) c = mma4(__uint_as_float(a[k]), __uint_as_float(b[k]), c);
    return c;
}

// The piece at columns col .. col + n - 1 of a row of dim elements; columns from dim on are zeros.
template <typename T>
__device__ inline u32x4 load_columns(const T* row, int col, int dim) {
    constexpr int n = Piece<T>::n;
    if (col + n <= dim) return load_piece(row + col);
    u32x4 v = {};
    for (int k = 0; k < n; ++k)
        if (col + k < dim) {
            if constexpr (sizeof(T) == 2)
                v[k / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, row[col + k]) << (16 * (k & 1));
            else
                v[k] = __float_as_uint(row[col + k]);
        }
    return v;
}
template <typename T>
__device__ inline void store_columns(T* row, int col, int dim, const float (&f)[Piece<T>::n]) {
    constexpr int n = Piece<T>::n;
    if (col + n <= dim) {
        store_values<n>(row + col, f);
    } else {
        for (int k = 0; k < n; ++k)
            if (col + k < dim) row[col + k] = (T)f[k];
    }
}

// Four columns of a row: 16 bytes or 8.
template <typename T>
using Quad = Columns<T, 4>;
template <typename T>
__device__ inline Quad<T> load_quad(const T* row, int col, int dim) {
    Quad<T> v;
    if (col + 4 <= dim) {
        __builtin_memcpy(v.d, row + col, sizeof v.d);
        return v;
    }
    v.zero();
    for (int k = 0; k < 4; ++k)
        if (col + k < dim) {
            if constexpr (sizeof(T) == 2)
                v.d[k / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, row[col + k]) << (16 * (k & 1));
            else
                v.d[k] = __float_as_uint(row[col + k]);
        }
    return v;
}
// A wave's own accesses of shared memory, in order.
__device__ inline void wave_meets() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Over the four lanes that share a row.
__device__ inline float row_sum(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}
__device__ inline float row_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// e^x for x <= 0, or not a number: 2^y for y = x log2(e) as it is rounded, times 1 + ln(2) (what the rounding took).  Values below 2^-126 may be 0.
__device__ inline float exp_below_0(float x) {
    x = x < -150.f ? -150.f : x;
    const float y = x * 1.44269502f;
    const float rest = __builtin_fmaf(x, 1.44269502f, -y) + x * 1.92596299e-8f;
    const float p = __builtin_amdgcn_exp2f(y);
    return __builtin_fmaf(p, rest * 0.693147182f, p);
}

// Two values rounded to bfloat16, the first in the low half; three such terms hold all 24 bits of the values.
__device__ inline uint32_t bf16_pair(float x, float y) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}
__device__ inline void bf16_terms(float x, float y, uint32_t (&term)[3]) {
    for (int k = 0; k < 3; ++k) {
        term[k] = bf16_pair(x, y);
        x -= __uint_as_float(term[k] << 16);
        y -= __uint_as_float(term[k] & 0xffff0000u);
    }
}

}  // namespace dynlp
