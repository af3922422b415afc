// AdamW over many tensors in one launch, states in 32 or 8 bits.
//     m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,  p = p (1 - lr decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
// Each array is read and written once: 28 bytes an element with 32-bit states and float32 parameters and gradients, 16 with 8-bit states
// (and gradients and a copy in bfloat16).  Bound by the memory, and at it: 60 tensors, 24M elements, 32 bits: 117 us (5.8 TB/s); a table of 256M
// elements, 8 bits: 876 us (4.7 TB/s; a copy of 4 GiB runs at 4.6).  A wave takes the 256 elements that share a scale, so that the block's
// largest value is found without leaving the wave.
#pragma once

#include "dynlp_device.h"
#include "dynlp_types.h"

namespace dynlp {

constexpr int kStateBlock = 256;      // elements of an 8-bit state that share a scale: four per lane of a wave
constexpr int kAdamwTensors = 40;     // tensors of one launch: their descriptions travel in the kernel's arguments

struct AdamwTensor {
    void* param;
    const void* grad;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* copy;
    int64_t n;
    float keep;       // 1 - lr * weight_decay
    uint32_t key;     // of the dither
    int32_t types;    // param | grad << 4 | copy << 8
    int32_t block;    // first workgroup; below 0 for the rest of a tensor that a launch before this one began
};

struct AdamwBatch {
    const float* grad_scale;
    float beta1, beta2, rest1, rest2;  // rest = 1 - beta
    float step_size;                   // lr / (1 - beta1^step)
    float root;                        // 1 / sqrt(1 - beta2^step)
    float eps;
    int32_t count;
    AdamwTensor t[kAdamwTensors];
};

// 32 bits out of 32 bits.  The factors are the fractions of the golden ratio and of the square root of two.
__host__ __device__ inline uint32_t dither_mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x9E3779B9u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ (x >> 16);
}

// Four elements from i on, of which the first `have` exist; the rest are zeros.  PAST: past the caches.
template <bool PAST>
__device__ inline void load4(const void* p, int type, int64_t i, int have, float (&f)[4]) {
    if (type == 0) {
        const float* x = static_cast<const float*>(p) + i;
        if (have == 4) {
            const u32x4_any4* from = reinterpret_cast<const u32x4_any4*>(x);
            u32x4 v;
            if constexpr (PAST) v = __builtin_nontemporal_load(from);
            else v = *from;
            for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(v[k]);
        } else {
            for (int k = 0; k < 4; ++k) f[k] = k < have ? x[k] : 0.f;
        }
        return;
    }
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
    const uint16_t* x = static_cast<const uint16_t*>(p) + i;
    uint16_t b[4] = {0, 0, 0, 0};
    if (have == 4) {
        const u16x4* from = reinterpret_cast<const u16x4*>(x);
        u16x4 v;
        if constexpr (PAST) v = __builtin_nontemporal_load(from);
        else v = *from;
        for (int k = 0; k < 4; ++k) b[k] = v[k];
    } else {
        for (int k = 0; k < 4; ++k)
            if (k < have) b[k] = x[k];
    }
    for (int k = 0; k < 4; ++k) f[k] = type == 1 ? to_float(__builtin_bit_cast(bf16, b[k])) : to_float(__builtin_bit_cast(f16, b[k]));
}
template <bool PAST>
__device__ inline void store4(void* p, int type, int64_t i, int have, const float (&f)[4]) {
    if (type == 0) {
        float* x = static_cast<float*>(p) + i;
        if (have == 4)
            store_values<4, PAST>(x, f);
        else
            for (int k = 0; k < 4; ++k)
                if (k < have) x[k] = f[k];
    } else if (type == 1) {
        bf16* x = static_cast<bf16*>(p) + i;
        if (have == 4)
            store_values<4, PAST>(x, f);
        else
            for (int k = 0; k < 4; ++k)
                if (k < have) x[k] = (bf16)f[k];
    } else {
        f16* x = static_cast<f16*>(p) + i;
        if (have == 4)
            store_values<4, PAST>(x, f);
        else
            for (int k = 0; k < 4; ++k)
                if (k < have) x[k] = (f16)f[k];
    }
}
typedef uint8_t u8x4 __attribute__((ext_vector_type(4), aligned(1)));
template <bool PAST>
__device__ inline void load_codes(const void* p, int64_t i, int have, uint32_t (&c)[4]) {
    const uint8_t* x = static_cast<const uint8_t*>(p) + i;
    if (have == 4) {
        const u8x4* from = reinterpret_cast<const u8x4*>(x);
        u8x4 v;
        if constexpr (PAST) v = __builtin_nontemporal_load(from);
        else v = *from;
        for (int k = 0; k < 4; ++k) c[k] = v[k];
    } else {
        for (int k = 0; k < 4; ++k) c[k] = k < have ? x[k] : 0u;
    }
}
template <bool PAST>
__device__ inline void store_codes(void* p, int64_t i, int have, const uint32_t (&c)[4]) {
    uint8_t* x = static_cast<uint8_t*>(p) + i;
    if (have == 4) {
        u8x4 v;
        for (int k = 0; k < 4; ++k) v[k] = (uint8_t)c[k];
        if constexpr (PAST)
            __builtin_nontemporal_store(v, reinterpret_cast<u8x4*>(x));
        else
            *reinterpret_cast<u8x4*>(x) = v;
    } else {
        for (int k = 0; k < 4; ++k)
            if (k < have) x[k] = (uint8_t)c[k];
    }
}

// Values of 4 exponent and 3 mantissa bits (exponent 7 is 1; below exponent 1 in steps of 2^-9).
__device__ inline float from_code(uint32_t c) {
    const uint32_t mag = c & 127u;
    const float f = mag < 8 ? (float)mag * 0x1p-9f : __uint_as_float((mag + (120u << 3)) << 20);
    return c & 128u ? -f : f;
}
// The code of y in [0, 256), rounded up with the probability that 16 bits of dither give.
__device__ inline uint32_t to_code(float y, uint32_t dither) {
    const uint32_t normal = ((__float_as_uint(y) + (dither << 4)) >> 20) - (120u << 3);
    const uint32_t small = (uint32_t)(y * 512.f + (float)dither * 0x1p-16f);
    return y >= 0x1p-6f ? normal : small;
}

__device__ inline uint32_t wave_max_bits(uint32_t v) {
    for (int d = kWave / 2; d > 0; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d, kWave));
    return v;
}
// Scale of a block whose largest magnitude has these bits, and its inverse; zero where that is too small, not-a-number where it is not finite.
__device__ inline float block_scale(uint32_t bits, float* inverse) {
    const uint32_t top = bits >> 23;
    *inverse = top >= 8 && top < 255 ? __uint_as_float((261u - top) << 23) : 0.f;
    return top == 255 ? __uint_as_float(0x7fc00000u) : top >= 8 ? __uint_as_float((top - 7) << 23) : 0.f;
}

// One wave per block of 256 elements, four per lane.  Products and sums are rounded one by one (no fused multiply-add), so that an 8-bit state
// is a function of its inputs that does not depend on how the compiler joins them.  PAST: the step's arrays are larger than the caches.
template <bool BITS8, bool PAST>
__global__ __launch_bounds__(kBlock) void k_adamw(AdamwBatch b) {
#pragma clang fp contract(off)
    int k = 0;
    {
        int lo = 0, hi = b.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (b.t[mid].block <= (int)blockIdx.x)
                lo = mid;
            else
                hi = mid - 1;
        }
        k = lo;
    }
    const AdamwTensor& t = b.t[k];
    const int64_t block = (int64_t)((int)blockIdx.x - t.block) * (kBlock / kWave) + threadIdx.x / kWave;
    const int64_t i = block * kStateBlock + lane_id() * 4;
    if (block * kStateBlock >= t.n) return;
    const int have = (int)min(max(t.n - i, (int64_t)0), (int64_t)4);
    const float gs = b.grad_scale ? *b.grad_scale : 1.f;
    float p[4], g[4], m[4], v[4];
    load4<PAST>(t.param, t.types & 15, i, have, p);
    load4<PAST>(t.grad, t.types >> 4 & 15, i, have, g);
    if (BITS8) {
        const float ms = t.m_scale[block], vs = t.v_scale[block];
        uint32_t c[4];
        load_codes<PAST>(t.m, i, have, c);
        for (int e = 0; e < 4; ++e) m[e] = from_code(c[e]) * ms;
        load_codes<PAST>(t.v, i, have, c);
        for (int e = 0; e < 4; ++e) {
            const float r = from_code(c[e]) * vs;
            v[e] = r * r;
        }
    } else {
        load4<PAST>(t.m, 0, i, have, m);
        load4<PAST>(t.v, 0, i, have, v);
    }
    float r[4];
    uint32_t m_top = 0, r_top = 0;
    for (int e = 0; e < 4; ++e) {
        g[e] = g[e] * gs;
        m[e] = m[e] * b.beta1 + g[e] * b.rest1;
        v[e] = v[e] * b.beta2 + (g[e] * g[e]) * b.rest2;
        r[e] = sqrtf(v[e]);
        p[e] = p[e] * t.keep - b.step_size * (m[e] / (r[e] * b.root + b.eps));
        if (e < have) {
            m_top = max(m_top, __float_as_uint(m[e]) & 0x7fffffffu);
            r_top = max(r_top, __float_as_uint(r[e]) & 0x7fffffffu);
        }
    }
    store4<PAST>(t.param, t.types & 15, i, have, p);
    if (t.copy) store4<PAST>(t.copy, t.types >> 8 & 15, i, have, p);
    if (!BITS8) {
        store4<PAST>(t.m, 0, i, have, m);
        store4<PAST>(t.v, 0, i, have, v);
        return;
    }
    float m_inverse, r_inverse;
    const float ms = block_scale(wave_max_bits(m_top), &m_inverse), rs = block_scale(wave_max_bits(r_top), &r_inverse);
    uint32_t mc[4], rc[4];
    for (int e = 0; e < 4; ++e) {
        const uint64_t at = (uint64_t)(i + e);
        const uint32_t h = dither_mix((uint32_t)at ^ t.key ^ (uint32_t)(at >> 32) * 0xBB67AE85u);
        // where the inverse is zero the product is (or is not a number, and the scale says so): code 0
        const float my = m_inverse != 0.f ? fabsf(m[e]) * m_inverse : 0.f, ry = r_inverse != 0.f ? r[e] * r_inverse : 0.f;
        mc[e] = to_code(my, h & 0xffffu) | (__float_as_uint(m[e]) >> 31) << 7;
        rc[e] = to_code(ry, h >> 16);
        if (r[e] > 0.f && r_inverse != 0.f) rc[e] = max(rc[e], 1u);
    }
    store_codes<PAST>(t.m, i, have, mc);
    store_codes<PAST>(t.v, i, have, rc);
    if (lane_id() == 0) {
        t.m_scale[block] = ms;
        t.v_scale[block] = rs;
    }
}

}  // namespace dynlp
