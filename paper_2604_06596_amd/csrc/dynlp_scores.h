// What rows of logits, or of probabilities, say: log probabilities of given classes, entropy, the first classes.
//
// With m the row's largest logit, s = sum exp(x - m) and t = sum exp(x - m) (x - m):   log p = x - m - log s,   entropy = log s - t / s.
// Of rows of probabilities, which need not sum to one: s = sum x, t = sum x log x:     log p = log x - log s,   entropy = log s - t / s.
// Classes are ordered by a key of 64 bits: the value's order above the class's, so that keys differ and of equal values the lowest class is the first.
#pragma once

#include "dynlp_matrix.h"

namespace dynlp {

struct Scores {
    const int32_t* classes;  // rows x given
    float* log_given;
    float* entropy;          // or NULL
    int32_t* top_classes;    // rows x top, or NULL
    float* log_top;          // or NULL
    int32_t* rejected;       // or NULL
    int given, top;
};

// Order of a value among 32-bit numbers; what is not a number counts as -infinity, and -0 as 0.
__device__ inline uint32_t order_of(float x) {
    const uint32_t u = x != x ? 0xff800000u : __float_as_uint(x + 0.f);
    return (int)u < 0 ? ~u : u | 0x80000000u;
}
__device__ inline uint64_t key_of(float x, int column) { return (uint64_t)order_of(x) << 32 | (uint32_t)~column; }
__device__ inline int column_of_key(uint64_t key) { return (int)~(uint32_t)key; }

// Sums over a row: m and s, t as above (PROB: m is not used).
struct RowSums {
    float m, s, t;
    __device__ static RowSums none() { return {-INFINITY, 0.f, 0.f}; }
};
template <bool PROB>
__device__ inline void add_value(RowSums& a, float x) {
    if constexpr (PROB) {
        a.s += x;
        a.t += x == 0.f ? 0.f : x * logf(x);
    } else {
        if (x > a.m) {
            const float d = a.m - x, f = a.m == -INFINITY ? 0.f : expf(d);
            a.t = a.m == -INFINITY ? a.t : f * (a.t + a.s * d);
            a.s *= a.m == -INFINITY ? 1.f : f;
            a.m = x;
        }
        const float d = x - a.m, e = expf(d);
        if (x != -INFINITY) a.s += e, a.t += e == 0.f ? 0.f : e * d;
    }
}
// Sums of two parts of a row.
template <bool PROB>
__device__ inline RowSums joined(const RowSums& a, const RowSums& b) {
    if constexpr (PROB) return {0.f, a.s + b.s, a.t + b.t};
    RowSums r{fmaxf(a.m, b.m), 0.f, 0.f};
    for (const RowSums* x : {&a, &b}) {
        const float d = x->m - r.m;
        if (x->m == -INFINITY) {
            r.s += x->s, r.t += x->t;  // nothing, or not a number
        } else {
            const float f = expf(d);
            r.s += f * x->s;
            r.t += f == 0.f ? 0.f : f * (x->t + x->s * d);
        }
    }
    return r;
}
// Log probability of value x of a row.  A row of nothing but -infinity (zeros) has 1/C everywhere.
template <bool PROB>
__device__ inline float log_of(float x, const RowSums& a, float log_s, int dim) {
    if (a.s == 0.f) return -logf((float)dim);
    return PROB ? logf(x) - log_s : (x - a.m) - log_s;
}
template <bool PROB>
__device__ inline float entropy_of(const RowSums& a, float log_s, int dim) {
    return a.s == 0.f ? logf((float)dim) : log_s - a.t / a.s;
}

template <typename V, typename F>
__device__ inline V over_block(V v, V* space, F f) {
    for (int d = 1; d < kWave; d <<= 1) {
        constexpr int n = sizeof(V) / 4;
        int word[n];
        __builtin_memcpy(word, &v, sizeof v);
        for (int k = 0; k < n; ++k) word[k] = __shfl_xor(word[k], d, kWave);
        V o;
        __builtin_memcpy(&o, word, sizeof o);
        v = lane_id() & d ? f(o, v) : f(v, o);
    }
    __syncthreads();
    if (lane_id() == 0) space[threadIdx.x / kWave] = v;
    __syncthreads();
    v = space[0];
    for (int w = 1; w < (int)blockDim.x / kWave; ++w) v = f(v, space[w]);
    return v;
}

// A workgroup per row.
template <typename T, bool PROB>
__global__ __launch_bounds__(kBlock) void k_row_scores(const T* x, int64_t ld, int64_t rows, int dim, Scores o, int64_t row0) {
    __shared__ RowSums sums[kBlock / kWave];
    __shared__ uint64_t best[kBlock / kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* p = x + row * ld;
        RowSums a = RowSums::none();
        for (int c = threadIdx.x; c < dim; c += kBlock) add_value<PROB>(a, to_float(p[c]));
        a = over_block(a, sums, [](const RowSums& u, const RowSums& v) { return joined<PROB>(u, v); });
        const float log_s = logf(a.s);
        const int64_t to = row0 + row;
        if (threadIdx.x == 0 && o.entropy) o.entropy[to] = entropy_of<PROB>(a, log_s, dim);
        for (int k = threadIdx.x; k < o.given; k += kBlock) {
            const int c = o.classes[to * o.given + k];
            if (c >= dim && o.rejected) atomicAdd(o.rejected, 1);
            o.log_given[to * o.given + k] = c >= 0 && c < dim ? log_of<PROB>(to_float(p[c]), a, log_s, dim) : 0.f;
        }
        uint64_t last = ~uint64_t(0);
        for (int k = 0; k < o.top; ++k) {
            uint64_t mine = 0;
            for (int c = threadIdx.x; c < dim; c += kBlock) {
                const uint64_t key = key_of(to_float(p[c]), c);
                if (key < last && key > mine) mine = key;
            }
            last = over_block(mine, best, [](uint64_t u, uint64_t v) { return u > v ? u : v; });
            if (threadIdx.x == 0) {
                const int c = column_of_key(last);
                if (o.top_classes) o.top_classes[to * o.top + k] = c;
                if (o.log_top) o.log_top[to * o.top + k] = log_of<PROB>(to_float(p[c]), a, log_s, dim);
            }
        }
    }
}

}  // namespace dynlp
