// Element types of the student's operators: loads and stores of 16-byte pieces of rows at any element alignment, and the
// conversions to and from float32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dynlp {

using bf16 = __bf16;
using f16 = _Float16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// The same 16 bytes at an address that is a multiple of the element's size only (global memory takes such addresses).
typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32x4 u32x4_any4 __attribute__((aligned(4)));

template <typename T>
struct Piece {
    static constexpr int n = 16 / (int)sizeof(T);  // elements in 16 bytes
};

template <typename T>
__device__ inline u32x4 load_piece(const T* p) {
    if constexpr (sizeof(T) == 2)
        return *reinterpret_cast<const u32x4_any2*>(p);
    else
        return *reinterpret_cast<const u32x4_any4*>(p);
}

template <typename T>
__device__ inline void store_piece(T* p, u32x4 v) {
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x4_any2*>(p) = v;
    else
        *reinterpret_cast<u32x4_any4*>(p) = v;
}

__device__ inline float to_float(float x) { return x; }
__device__ inline float to_float(bf16 x) { return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, x) << 16); }
__device__ inline float to_float(f16 x) { return (float)x; }

// The piece's elements as float32.
__device__ inline void widen(u32x4 p, float (&f)[4], float) {
    for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(p[k]);
}
__device__ inline void widen(u32x4 p, float (&f)[8], bf16) {
    for (int k = 0; k < 4; ++k) {
        f[2 * k] = __uint_as_float(p[k] << 16);
        f[2 * k + 1] = __uint_as_float(p[k] & 0xffff0000u);
    }
}
__device__ inline void widen(u32x4 p, float (&f)[8], f16) {
    const f16x8 h = __builtin_bit_cast(f16x8, p);
    for (int k = 0; k < 8; ++k) f[k] = (float)h[k];
}

// V float32 values rounded to the type of the array and stored at p (any element alignment).
template <int V>
__device__ inline void store_values(float* p, const float (&f)[V]) {
    static_assert(V == 1 || V % 4 == 0, "one value, or whole pieces");
    if constexpr (V == 1) {
        *p = f[0];
    } else {
        for (int k = 0; k < V; k += 4) {
            u32x4 v;
            for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(f[k + j]);
            store_piece(p + k, v);
        }
    }
}
template <int V, typename T>
__device__ inline void store_values(T* p, const float (&f)[V]) {
    static_assert(sizeof(T) == 2 && (V == 1 || V % 4 == 0), "one value, or half a piece and more");
    if constexpr (V == 1) {
        *p = (T)f[0];
    } else {
        for (int k = 0; k < V; k += 4) {
            typedef T t4 __attribute__((ext_vector_type(4)));
            typedef t4 t4_any __attribute__((aligned(2)));
            t4 v;
            for (int j = 0; j < 4; ++j) v[j] = (T)f[k + j];
            *reinterpret_cast<t4_any*>(p + k) = v;
        }
    }
}

}  // namespace dynlp
