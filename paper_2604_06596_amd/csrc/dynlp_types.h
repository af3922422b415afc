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

// V float32 values (1, 2 or a multiple of 4) rounded to the type of the array and stored at p (any element alignment); PAST: past the caches, for
// what is not read again while it would be in them.
template <int V, bool PAST = false, typename T>
__device__ inline void store_values(T* p, const float (&f)[V]) {
    constexpr int n = V < 4 ? V : 4;
    static_assert(V % n == 0 && n != 3, "one value, two, or fours");
    if constexpr (n == 1) {
        *p = (T)f[0];
    } else {
        typedef T vec __attribute__((ext_vector_type(n)));
        typedef vec vec_any __attribute__((aligned(sizeof(T))));
        for (int k = 0; k < V; k += n) {
            vec v;
            for (int j = 0; j < n; ++j) v[j] = (T)f[k + j];
            if constexpr (PAST)
                __builtin_nontemporal_store((vec_any)v, reinterpret_cast<vec_any*>(p + k));
            else
                *reinterpret_cast<vec_any*>(p + k) = v;
        }
    }
}

// Words at an address that is a multiple of 2 or 4 bytes only, in global memory.
template <int WORDS, int ALIGN>
struct Words;
#define DYNLP_WORDS(n, a)                                                     \
    template <>                                                               \
    struct Words<n, a> {                                                      \
        typedef uint32_t vec __attribute__((ext_vector_type(n), aligned(a))); \
    };
DYNLP_WORDS(1, 2)
DYNLP_WORDS(2, 2)
DYNLP_WORDS(4, 2)
DYNLP_WORDS(1, 4)
DYNLP_WORDS(2, 4)
DYNLP_WORDS(4, 4)
#undef DYNLP_WORDS

// E consecutive elements of a row (4, 8 or 16 bytes) as they are in memory.
template <typename T, int E>
struct Columns {
    static constexpr int words = E * (int)sizeof(T) / 4;
    uint32_t d[words];
    // From `offset` bytes behind an address that is the same for all lanes (scalar registers hold it).
    __device__ inline void load(uint64_t address, uint32_t offset) {
        typedef typename Words<words, (int)sizeof(T)>::vec vec;
        typedef const __attribute__((address_space(1))) char* bytes;
        typedef const __attribute__((address_space(1))) vec* vecs;
        const vec v = *(vecs)((bytes)address + offset);
        for (int k = 0; k < words; ++k) d[k] = v[k];
    }
    __device__ inline void zero() {
        for (int k = 0; k < words; ++k) d[k] = 0u;
    }
    __device__ inline float get(int e) const {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(d[e]);
        else
            return to_float(__builtin_bit_cast(T, (uint16_t)(d[e / 2] >> (16 * (e & 1)))));
    }
};

}  // namespace dynlp
