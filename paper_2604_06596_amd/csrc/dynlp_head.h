// The class head: logits, class distributions, cross entropy and its gradients.  Dense products on the matrix cores.
//
// Fragments of v_mfma_f32_16x16x{32,4}: lane l = 16 q + r (q = 0 .. 3, r = 0 .. 15) gives row r of the left operand, column r of the right
// one and holds rows 4 q .. 4 q + 3 of column r of the result.  Which k of the product a lane's operand elements stand for is free as
// long as both operands agree, and so is which columns of a matrix stand behind the 16 rows or columns of a tile; both are chosen
// here so that every lane reads 16 consecutive bytes and the result of one product is, as it lies in the registers, an operand of the
// next:
//   logits   z^T = W h^T.   Lane (q, r): W of class r, h of row r, a piece of n columns from k0 + n q on (64 bytes of a row per access).
//            Result: row r's logits of classes 16 t + 4 q + i.
//   dh       dh^T = W^T dz^T.  The right operand (k = class, column = row r) is what the lane holds after the softmax.  The left one
//            needs W by columns: pieces of W's rows, for two-byte types transposed between registers.  Result: row r, n consecutive columns.
//   dweight  dz^T h.  Both operands are read row by row of h and dz, h in pieces, transposed between registers where needed.
// Precision: products of bfloat16 and float16 values are exact in the matrix cores, sums are float32; dz, which is float32, is taken in three
// bfloat16 terms, which hold all of it, or the product is made in float32 (float32 and float16 heads).
// Terms in float16 would need scales of their own: dz, with a grad_scale of one in a million rows, lies below what float16 holds.  The float32 instruction has
// an eighth of the rate (153 TFLOP/s, 1,190 in bfloat16), which bounds float16 heads: 1M x 256, 50 classes, 816 us, 410 in bfloat16 in the same run.
// What bounds it: h is read once (from memory; for dweight again, from the L2) and dh written once.  1M rows x 256 bfloat16, 50 classes, with soft
// targets: 385 us (3.2 TB/s of what has to move; the first kernels, with dz through memory and h read twice, 905 us).  100,000 x 64 float32, 10
// classes: 24 us, of which each workgroup spends half on its start and end.
#pragma once

#include "dynlp_device.h"
#include "dynlp_types.h"

namespace dynlp {

constexpr int kMaxTiles = 4;  // of 16 classes

struct Head {
    const void* h;
    const void* weight;
    const float* bias;
    int64_t ld_h, ld_w;
    int64_t rows;
    int dim, classes;
};

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
// Column t of eight rows' quads, as an operand with these rows for k.
__device__ inline u32x4 column_of(const Quad<bf16> (&x)[8], int t) {
    u32x4 v;
    for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(x[2 * j + 1].d[t >> 1], x[2 * j].d[t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
    return v;
}

// The head's rows where they are, or a copy in shared memory that is padded with zeros to whole tiles of classes and columns.
template <typename T>
struct WeightRows {
    const T* w;
    const float* bias;
    int64_t ld;
    int dim, classes;
    // Bias of classes c .. c + 3; -infinity, which makes the logit so whatever h holds, for what is not a class.
    __device__ inline f32x4 bias4(int c) const {
        f32x4 b;
        for (int i = 0; i < 4; ++i) b[i] = c + i >= classes ? -INFINITY : bias ? bias[c + i] : 0.f;
        return b;
    }
    __device__ inline u32x4 piece(int c, int col) const {
        return c < classes && col < dim ? load_columns(w + (int64_t)c * ld, col, dim) : u32x4{0u, 0u, 0u, 0u};
    }
    __device__ inline Quad<T> quad(int c, int col) const {
        if (c < classes && col < dim) return load_quad(w + (int64_t)c * ld, col, dim);
        Quad<T> v;
        v.zero();
        return v;
    }
};
template <typename T>
struct SharedWeight {
    const T* w;
    const float* bias;
    int ld;
    __device__ inline f32x4 bias4(int c) const { return *reinterpret_cast<const f32x4*>(bias + c); }
    __device__ inline u32x4 piece(int c, int col) const { return *reinterpret_cast<const u32x4*>(w + c * ld + col); }
    __device__ inline Quad<T> quad(int c, int col) const {
        Quad<T> v;
        if constexpr (sizeof(T) == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(w + c * ld + col);
            v.d[0] = x.x, v.d[1] = x.y;
        } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(w + c * ld + col);
            for (int k = 0; k < 4; ++k) v.d[k] = x[k];
        }
        return v;
    }
};
// The same rows, but addresses made from them are not kept in registers from one step of a loop to the next.
template <typename T>
__device__ inline WeightRows<T> anew(const WeightRows<T>& w) {
    return w;
}
template <typename T>
__device__ inline SharedWeight<T> anew(SharedWeight<T> w) {
    asm volatile("" : "+s"(w.ld));
    return w;
}
// Columns of the copy: whole pieces of a wave (16 lanes x n columns, and the 8 n of a step over the logits), and 16 bytes so that the 16 rows
// of a tile begin in different banks.
template <typename T>
__host__ __device__ inline int shared_ld(int dim) {
    constexpr int n = Piece<T>::n;
    return (dim + 16 * n - 1) / (16 * n) * (16 * n) + n;
}
template <typename T, int CT>
__device__ inline SharedWeight<T> share_weight(const Head& a, T* to) {
    constexpr int n = Piece<T>::n;
    const int ld = shared_ld<T>(a.dim), pieces = ld / n;
    const WeightRows<T> w{static_cast<const T*>(a.weight), a.bias, a.ld_w, a.dim, a.classes};
    float* bias = reinterpret_cast<float*>(to + 16 * CT * ld);
    if ((int)threadIdx.x < 4 * CT) *reinterpret_cast<f32x4*>(bias + 4 * threadIdx.x) = w.bias4(4 * threadIdx.x);
    for (int at = threadIdx.x; at < 16 * CT * pieces; at += blockDim.x)
        *reinterpret_cast<u32x4*>(to + at * n) = w.piece(at / pieces, at % pieces * n);
    __syncthreads();
    return SharedWeight<T>{to, bias, ld};
}
// Bytes of that copy, a multiple of 16.
template <typename T, int CT>
__host__ __device__ inline int shared_bytes(int dim) {
    return 16 * CT * (shared_ld<T>(dim) * (int)sizeof(T) + 4);
}

// z[m][t] = logits of rows first + 16 m + r, classes 16 t + 4 q + i, bias added; -infinity beyond the classes.  S steps' parts of h are asked for
// before the first's products.
template <typename T, int CT, int NT, int S, typename W>
__device__ inline void head_logits(const Head& a, const W& w, int64_t first, f32x4 (&z)[NT][CT]) {
    constexpr int n = Piece<T>::n;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* h[NT];
    for (int m = 0; m < NT; ++m) {
        h[m] = static_cast<const T*>(a.h) + min(first + 16 * m + r, a.rows - 1) * a.ld_h;
        for (int t = 0; t < CT; ++t) z[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int mine = q * n;
#pragma unroll 1
    for (int k0 = 0; k0 < a.dim; k0 += S * 8 * n) {
        const W rows = anew(w);
        u32x4 v[S][NT][2];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int c = k0 + s * 8 * n;
            if (c + 8 * n <= a.dim) {
                for (int m = 0; m < NT; ++m)
                    for (int e = 0; e < 2; ++e) v[s][m][e] = load_piece(h[m] + c + mine + e * 4 * n);
            } else if (c < a.dim) {
                for (int m = 0; m < NT; ++m)
                    for (int e = 0; e < 2; ++e) v[s][m][e] = load_columns(h[m], c + mine + e * 4 * n, a.dim);
            }
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int c = k0 + s * 8 * n;
            if (c < a.dim)
                for (int e = 0; e < 2; ++e)
                    for (int t = 0; t < CT; ++t) {
                        const u32x4 wv = rows.piece(16 * t + r, c + mine + e * 4 * n);
                        for (int m = 0; m < NT; ++m) z[m][t] = mma(wv, v[s][m][e], z[m][t], T());
                    }
        }
    }
    for (int t = 0; t < CT; ++t) {
        const f32x4 b = w.bias4(16 * t + 4 * q);
        for (int m = 0; m < NT; ++m)
            for (int i = 0; i < 4; ++i) z[m][t][i] = b[i] == -INFINITY ? b[i] : z[m][t][i] + b[i];
    }
}

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

// z becomes exp(z - max); returns the sum, and the largest logit.  A NaN among the logits makes the sum one.
template <int CT>
__device__ inline float head_exp(f32x4 (&z)[CT], float* top) {
    float m = -INFINITY;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) m = fmaxf(m, z[t][i]);
    m = row_max(m);
    float sum = 0.f;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) {
            // a row of nothing but -infinity keeps sum 0; +infinity - +infinity is not a number, as it should be
            z[t][i] = z[t][i] == -INFINITY ? 0.f : exp_below_0(z[t][i] - m);
            sum += z[t][i];
        }
    *top = m;
    return row_sum(sum);
}

constexpr int kLabelRows = 16 * (kBlock / kWave);   // rows of a workgroup's tile for labels
constexpr int kHeadTiles = 2;                       // tiles of 16 rows per wave where loss and gradients are not made in one pass
constexpr int kHeadRows = kHeadTiles * 16 * (kBlock / kWave);  // rows per workgroup

// One tile of 16 rows per wave from W as it is, or (SHARED) any number of them from a copy of W in shared memory.  Bound by reading h, with enough of it
// under way: 300,007 x 200 float16, 29 classes: 37 us (4.2 TB/s), where tiles of 32 rows and half as many steps ahead took 53 us.
template <typename T, int CT, bool SHARED>
__global__ __launch_bounds__(kBlock) void k_head_labels(Head a, float* soft, int32_t* hard) {
    constexpr int NT = 1;
    extern __shared__ char space[];
    const int q = lane_id() >> 4, r = lane_id() & 15;
    auto tile = [&](const auto& w, int64_t first) {
        f32x4 z[NT][CT];
        head_logits<T, CT, NT, 4>(a, w, first, z);
        for (int m = 0; m < NT; ++m) {
            const int64_t row = first + 16 * m + r;
            if (hard) {
                float best = -INFINITY;
                int at = a.classes;
                for (int t = 0; t < CT; ++t)
                    for (int i = 0; i < 4; ++i)
                        if (z[m][t][i] > best) best = z[m][t][i], at = 16 * t + 4 * q + i;
                for (int d = 16; d < kWave; d <<= 1) {
                    const float other = __shfl_xor(best, d, kWave);
                    const int other_at = __shfl_xor(at, d, kWave);
                    if (other > best || (other == best && other_at < at)) best = other, at = other_at;
                }
                if (q == 0 && row < a.rows) hard[row] = at < a.classes ? at : 0;
            }
            if (soft) {
                float top;
                const float sum = head_exp(z[m], &top), inverse = 1.f / sum;
                if (row < a.rows)
                    for (int t = 0; t < CT; ++t) {
                        float f[4];
                        for (int i = 0; i < 4; ++i) f[i] = sum == 0.f ? 1.f / (float)a.classes : z[m][t][i] * inverse;
                        if (16 * t + 4 * q < a.classes) store_columns(soft + row * a.classes, 16 * t + 4 * q, a.classes, f);
                    }
            }
        }
    };
    const int64_t first = (threadIdx.x / kWave) * (NT * 16);
    if constexpr (SHARED) {
        const SharedWeight<T> w = share_weight<T, CT>(a, reinterpret_cast<T*>(space));
        for (int64_t at = (int64_t)blockIdx.x * kLabelRows; at + first < a.rows; at += (int64_t)gridDim.x * kLabelRows) tile(w, at + first);
    } else {
        const WeightRows<T> w{static_cast<const T*>(a.weight), a.bias, a.ld_w, a.dim, a.classes};
        if ((int64_t)blockIdx.x * kLabelRows + first < a.rows) tile(w, (int64_t)blockIdx.x * kLabelRows + first);
    }
}

struct Loss {
    const float* soft;
    const int32_t* hard;
    const float* row_weight;
    int32_t* rejected;
    float grad_scale;
    float* loss;
    void* dh;        // or NULL
    int64_t ld_dh;
    float* dz;       // rows x (16 tiles), or NULL; rows that are left out: zeros
    uint8_t* kept;   // rows: 0 if left out
};

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

// dh of the tile's rows from their dz, 64 columns at a time.  Quads of W's rows are the left operand; in bfloat16 a lane's 8 x 4 block (8 classes, 4
// columns) is transposed by v_perm.
template <int CT, int NT, typename T>
__device__ inline void store_dh(const Head& a, int64_t first, int base, const f32x4 (&acc)[NT][4], const bool (&kept)[NT], T* dh, int64_t ld_dh) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    constexpr int n = Piece<T>::n;
    const bool whole = first + 16 * NT <= a.rows && base + 64 <= a.dim;  // nothing to look at lane by lane
    for (int m = 0; m < NT; ++m) {
        const int64_t row = first + 16 * m + r;
        // a lane holds 16 consecutive columns
        for (int k = 0; k < 16; k += n) {
            const int to = base + 16 * q + k;
            float f[n];
            for (int e = 0; e < n; ++e) f[e] = kept[m] ? acc[m][(k + e) & 3][(k + e) >> 2] : 0.f;
            if (whole)
                store_values<n>(dh + row * ld_dh + to, f);
            else if (row < a.rows && to < a.dim)
                store_columns(dh + row * ld_dh, to, a.dim, f);
        }
    }
}
// dz of a lane's row and classes 16 t + 4 q + i in bfloat16 terms: pairs (i = 0, 1) and (2, 3).
template <int CT>
struct DzTerms {
    uint32_t v[CT][2][3];
    __device__ inline void make(const f32x4 (&dz)[CT]) {
        for (int t = 0; t < CT; ++t)
            for (int k = 0; k < 2; ++k) bf16_terms(dz[t][2 * k], dz[t][2 * k + 1], v[t][k]);
    }
    // Operand whose k = 8 q + j stands for class 16 (2 p + j / 4) + 4 q + j % 4.
    __device__ inline u32x4 operand(int p, int term) const {
        const bool two = 2 * p + 1 < CT;
        const int o = two ? 2 * p + 1 : 0;
        return u32x4{v[2 * p][0][term], v[2 * p][1][term], two ? v[o][0][term] : 0u, two ? v[o][1][term] : 0u};
    }
};
// Two terms would leave out 2^-17 of dz, which shows in dh where classes cancel, as what W's rows have in common always does (dz sums to nothing over
// the classes of a row).  The third costs 1 to 3% of a step: 1M x 256, 50 classes, 399 us with two, 410 with three.
template <int CT, int NT, typename W>
__device__ inline void head_dh(const Head& a, const W& w, int64_t first, const DzTerms<CT> (&dz)[NT], const bool (&kept)[NT], bf16* dh,
                               int64_t ld_dh) {
    constexpr int P = (CT + 1) / 2;
    const int q = lane_id() >> 4, r = lane_id() & 15;
#pragma unroll 1
    for (int base = 0; base < a.dim; base += 64) {
        const W rows = anew(w);
        f32x4 acc[NT][4];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < P; ++p) {
            Quad<bf16> x[8];
            for (int j = 0; j < 8; ++j) {
                const int t = 2 * p + (j >> 2);
                if (t < CT)
                    x[j] = rows.quad(16 * t + 4 * q + (j & 3), base + 4 * r);
                else
                    x[j].zero();
            }
            for (int t = 0; t < 4; ++t) {
                const u32x4 left = column_of(x, t);
                for (int m = 0; m < NT; ++m)
                    for (int k = 2; k >= 0; --k) acc[m][t] = mma(left, dz[m].operand(p, k), acc[m][t], bf16());
            }
        }
        store_dh<CT, NT>(a, first, base, acc, kept, dh, ld_dh);
    }
}
template <int CT, int NT, typename W, typename T>
__device__ inline void head_dh(const Head& a, const W& w, int64_t first, const f32x4 (&dz)[NT][CT], const bool (&kept)[NT], T* dh, int64_t ld_dh) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
#pragma unroll 1
    for (int base = 0; base < a.dim; base += 64) {
        const W rows = anew(w);
        f32x4 acc[NT][4];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int ct = 0; ct < CT; ++ct)
            for (int i = 0; i < 4; ++i) {
                const Quad<T> x = rows.quad(16 * ct + 4 * q + i, base + 4 * r);
                for (int t = 0; t < 4; ++t)
                    for (int m = 0; m < NT; ++m) acc[m][t] = mma4(x.get(t), dz[m][ct][i], acc[m][t]);
            }
        store_dh<CT, NT>(a, first, base, acc, kept, dh, ld_dh);
    }
}

// What a lane needs of row `row` beside its logits, asked for before them.
template <int CT>
struct RowTarget {
    f32x4 y[CT];
    float weight;
    bool use;
    // inner (the same for all lanes): 64 rows follow, so that a whole tile of classes may be read from every row.
    __device__ inline void ask(const Head& a, const Loss& g, int64_t row, bool inner) {
        const int q = lane_id() >> 4;
        const bool inside = row < a.rows;
        const int64_t at = inside ? row : a.rows - 1;
        weight = g.row_weight ? g.row_weight[at] : 1.f;
        use = inside;
        if (g.hard) {
            const int label = g.hard[at];
            if (inside && q == 0 && label >= a.classes && g.rejected) atomicAdd(g.rejected, 1);
            use = use && label >= 0 && label < a.classes;
            for (int t = 0; t < CT; ++t)
                for (int i = 0; i < 4; ++i) y[t][i] = 16 * t + 4 * q + i == label ? 1.f : 0.f;
        } else if (inner) {
            for (int t = 0; t < CT; ++t) y[t] = __builtin_bit_cast(f32x4, load_piece(g.soft + at * a.classes + 16 * t + 4 * q));
            for (int i = 0; i < 4; ++i) y[CT - 1][i] = 16 * (CT - 1) + 4 * q + i < a.classes ? y[CT - 1][i] : 0.f;
        } else {
            for (int t = 0; t < CT; ++t) {
                const int c = 16 * t + 4 * q;
                y[t] = __builtin_bit_cast(f32x4, c < a.classes ? load_columns(g.soft + at * a.classes, c, a.classes) : u32x4{0u, 0u, 0u, 0u});
            }
        }
    }
};

// From the logits z of row `row` of a lane (first + 16 m + r): its loss is stored, z becomes dz.  Returns whether the row takes part.
template <int CT>
__device__ inline bool head_dz(const Loss& g, int64_t row, int64_t rows, const RowTarget<CT>& target, f32x4 (&z)[CT]) {
    f32x4 e[CT];
    for (int t = 0; t < CT; ++t) e[t] = z[t];
    float top;
    const float sum = head_exp(e, &top);
    const bool use = target.use && target.weight != 0.f && sum != 0.f;
    const float lse = logf(sum);  // of the shifted logits
    float total = 0.f, loss = 0.f;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) {
            const float y = target.y[t][i];
            total += y;
            loss += y != 0.f ? y * (lse - (z[t][i] - top)) : 0.f;
        }
    total = row_sum(total);
    loss = row_sum(loss);
    const float scale = g.grad_scale * target.weight, part = total / sum;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) z[t][i] = use ? scale * (part * e[t][i] - target.y[t][i]) : 0.f;
    if (row < rows && lane_id() < 16 && g.loss) g.loss[row] = use ? target.weight * loss : 0.f;
    return use;
}

// Loss, dz and dh of a tile of rows: logits, softmax and the product with W, without leaving the registers.  For heads whose W and dweight do
// not fit a workgroup, and where no dweight is asked for.  Rows from row0 on.
template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_head_loss(Head a, Loss g, int64_t row0) {
    constexpr int NT = kHeadTiles;
    const int64_t first = row0 + (int64_t)blockIdx.x * kHeadRows + (threadIdx.x / kWave) * (NT * 16);
    if (first >= a.rows) return;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const WeightRows<T> w{static_cast<const T*>(a.weight), a.bias, a.ld_w, a.dim, a.classes};
    f32x4 z[NT][CT];
    RowTarget<CT> target[NT];
    bool kept[NT];
    for (int m = 0; m < NT; ++m) target[m].ask(a, g, first + 16 * m + r, first + 16 * NT + 64 <= a.rows);
    head_logits<T, CT, NT, 2>(a, w, first, z);
    for (int m = 0; m < NT; ++m) {
        const int64_t row = first + 16 * m + r;
        kept[m] = head_dz(g, row, a.rows, target[m], z[m]);
        if (row < a.rows && g.dz) {
            if (q == 0) g.kept[row] = kept[m] ? 1 : 0;
            for (int t = 0; t < CT; ++t) *reinterpret_cast<f32x4*>(g.dz + row * (16 * CT) + 16 * t + 4 * q) = z[m][t];
        }
    }
    if (!g.dh) return;
    if constexpr (__is_same(T, bf16)) {
        DzTerms<CT> terms[NT];
        for (int m = 0; m < NT; ++m) terms[m].make(z[m]);
        head_dh<CT, NT>(a, w, first, terms, kept, static_cast<T*>(g.dh), g.ld_dh);
    } else {
        head_dh<CT, NT>(a, w, first, z, kept, static_cast<T*>(g.dh), g.ld_dh);
    }
}

// ---- dweight = dz^T h, dbias ------------------------------------------------------------------------------------------

struct Outer {
    const void* h;
    const float* dz;
    const uint8_t* kept;
    float* part;      // [split][classes][dim + 1]: the last column is dbias
    int64_t ld_h;
    int64_t rows;
    int64_t per_wave; // rows of a wave, a multiple of 32
    int dim, classes;
};

// Columns base + n r + t of a wave's part of dweight: acc[ct][t].  Rows are taken 16 (one product over 4 rows for each column of a piece) or,
// for bfloat16, 32 at a time.
template <int CT>
__device__ inline void outer_rows(const Outer& o, int64_t first, int64_t end, int col, f32x4 (&acc)[CT][8], float (&sum)[CT], bf16) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const bf16* h = static_cast<const bf16*>(o.h);
    for (int64_t n0 = first; n0 < end; n0 += 32) {
        u32x4 x[8];
        f32x4 a[CT][2];
        for (int j = 0; j < 8; ++j) {
            const int64_t row = n0 + 8 * q + j;
            const bool use = row < end && o.kept[min(row, o.rows - 1)];
            x[j] = u32x4{0u, 0u, 0u, 0u};
            if (use && col < o.dim) x[j] = load_columns(h + row * o.ld_h, col, o.dim);
            for (int t = 0; t < CT; ++t) a[t][j >> 2][j & 3] = use ? o.dz[row * (16 * CT) + 16 * t + r] : 0.f;
        }
        // dz in three bfloat16 terms, which hold all 24 bits of it: dweight is a float32 sum over all rows
        u32x4 term[3][CT];
        for (int t = 0; t < CT; ++t)
            for (int j = 0; j < 8; j += 2) {
                const float v0 = a[t][j >> 2][j & 3], v1 = a[t][j >> 2][(j & 3) + 1];
                sum[t] += v0;
                sum[t] += v1;
                uint32_t three[3];
                bf16_terms(v0, v1, three);
                for (int k = 0; k < 3; ++k) term[k][t][j >> 1] = three[k];
            }
        for (int t = 0; t < 8; ++t) {
            u32x4 right;
            for (int j = 0; j < 4; ++j)
                right[j] = __builtin_amdgcn_perm(x[2 * j + 1][t >> 1], x[2 * j][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
            for (int k = 2; k >= 0; --k)
                for (int ct = 0; ct < CT; ++ct) acc[ct][t] = mma(term[k][ct], right, acc[ct][t], bf16());
        }
    }
}
template <int CT, int N, typename T>
__device__ inline void outer_rows(const Outer& o, int64_t first, int64_t end, int col, f32x4 (&acc)[CT][N], float (&sum)[CT], T) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* h = static_cast<const T*>(o.h);
    for (int64_t n0 = first; n0 < end; n0 += 16) {
        u32x4 x[4];
        float a[4][CT];
        for (int j = 0; j < 4; ++j) {
            const int64_t row = n0 + 4 * j + q;
            const bool use = row < end && o.kept[min(row, o.rows - 1)];
            x[j] = u32x4{0u, 0u, 0u, 0u};
            if (use && col < o.dim) x[j] = load_columns(h + row * o.ld_h, col, o.dim);
            for (int t = 0; t < CT; ++t) a[j][t] = use ? o.dz[row * (16 * CT) + 16 * t + r] : 0.f;
        }
        for (int j = 0; j < 4; ++j) {
            float f[N];
            widen(x[j], f, T());
            for (int ct = 0; ct < CT; ++ct) {
                sum[ct] += a[j][ct];
                for (int t = 0; t < N; ++t) acc[ct][t] = mma4(a[j][ct], f[t], acc[ct][t]);
            }
        }
    }
}

template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_head_outer(Outer o) {
    constexpr int N = Piece<T>::n, kCols = 16 * N;
    __shared__ float joined[16 * CT][kCols + 1];
    const int q = lane_id() >> 4, r = lane_id() & 15, wave = threadIdx.x / kWave;
    const int64_t first = ((int64_t)blockIdx.x * (kBlock / kWave) + wave) * o.per_wave;
    const int64_t end = min(first + o.per_wave, o.rows);
    const int base = (int)blockIdx.y * kCols;
    f32x4 acc[CT][N];
    float sum[CT];
    for (int ct = 0; ct < CT; ++ct) {
        sum[ct] = 0.f;
        for (int t = 0; t < N; ++t) acc[ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    outer_rows(o, first, end, base + N * r, acc, sum, T());
    for (int ct = 0; ct < CT; ++ct) sum[ct] = row_sum(sum[ct]);
    for (int w = 0; w < kBlock / kWave; ++w) {
        if (w == wave)
            for (int ct = 0; ct < CT; ++ct) {
                for (int t = 0; t < N; ++t)
                    for (int i = 0; i < 4; ++i) {
                        float& to = joined[16 * ct + 4 * q + i][N * r + t];
                        to = w ? to + acc[ct][t][i] : acc[ct][t][i];
                    }
                if (q == 0) {
                    float& to = joined[16 * ct + r][kCols];
                    to = w ? to + sum[ct] : sum[ct];
                }
            }
        __syncthreads();
    }
    float* part = o.part + (int64_t)blockIdx.x * o.classes * (o.dim + 1);
    for (int at = threadIdx.x; at < o.classes * (kCols + 1); at += kBlock) {
        const int c = at / (kCols + 1), k = at - c * (kCols + 1);
        if (k < kCols && base + k < o.dim) part[(int64_t)c * (o.dim + 1) + base + k] = joined[c][k];
        if (k == kCols && blockIdx.y == 0) part[(int64_t)c * (o.dim + 1) + o.dim] = joined[c][k];
    }
}

// ---- everything in one pass over h ------------------------------------------------------------------------------------

constexpr int kFusedColumns = 64;  // of a group: a wave's part of dweight
constexpr int kFusedMost = kFusedColumns * 8;

// Waves of a workgroup, 16 rows each: eight up to 32 classes, four on a SIMD; beyond that four, two on a SIMD.  us with eight and with four waves:
//   up to 16 classes (128 registers are enough): 100,000 x 64, 10 classes: float32 28.0 and 31.1, bfloat16 22.0 and 25.4; 1M x 256 bfloat16 262 and 280
//   17 to 32 (8, 44 and 100 bytes a lane go to scratch in float16, float32 and bfloat16): 1M x 256, 29 classes: bfloat16 325 and 310, float32 667 and 687,
//     float16 444 and 464; 1M x 64 float32, 20 classes: 226 and 241
//   beyond 32: 1M x 256, 50 classes: bfloat16 436 and 410, float16 879 and 816, but float32 1,037 and 1,303; 200,000 x 128 float32, 64 classes: 167 and 145
// Where more than 256 columns make a wave of the four hold two groups of dweight's columns, one wave is on a SIMD: 500,000 x 512 bfloat16, 50 classes,
// 571 us, which eight waves would take 392 for.
__host__ __device__ constexpr int fused_waves(int class_tiles) { return class_tiles <= 2 ? 8 : 4; }
__host__ __device__ constexpr int fused_rows(int class_tiles) { return 16 * fused_waves(class_tiles); }  // of a tile

// dz of a tile in shared memory: [row][class], padded so that the four rows that a wave reads at once lie in different banks.
template <typename T, int CT>
struct SharedDz {
    static constexpr int ld = 16 * CT + 16, bytes = fused_rows(CT) * ld * 4;
    float* p;
    __device__ inline void put(int row, int t, int q, const f32x4& z) { *reinterpret_cast<f32x4*>(p + row * ld + 16 * t + 4 * q) = z; }
    // Sum of a class over 16 rows.
    __device__ inline float rows_of(int c, int from) const {
        float s = 0.f;
        for (int k = 0; k < 16; ++k) s += p[(from + k) * ld + c];
        return s;
    }
};
// For bfloat16 in three terms, which hold all 24 bits (dweight is a float32 sum over all rows): [term][class][row].
template <int CT>
struct SharedDz<bf16, CT> {
    static constexpr int ld = fused_rows(CT) + 8, bytes = 3 * 16 * CT * ld * 2;
    float* p;
    __device__ inline bf16* at(int term, int c, int row) const { return reinterpret_cast<bf16*>(p) + (term * 16 * CT + c) * ld + row; }
    __device__ inline void put(int row, int q, const DzTerms<CT>& z) {
        for (int t = 0; t < CT; ++t)
            for (int k = 0; k < 2; ++k)
                for (int term = 0; term < 3; ++term) {
                    const uint32_t v = z.v[t][k][term];
                    *at(term, 16 * t + 4 * q + 2 * k, row) = __builtin_bit_cast(bf16, (uint16_t)v);
                    *at(term, 16 * t + 4 * q + 2 * k + 1, row) = __builtin_bit_cast(bf16, (uint16_t)(v >> 16));
                }
    }
    __device__ inline float rows_of(int c, int from) const {
        float s = 0.f;
        for (int term = 2; term >= 0; --term)
            for (int k = 0; k < 16; k += 8) {
                float f[8];
                widen(*reinterpret_cast<const u32x4*>(at(term, c, from + k)), f, bf16());
                for (int e = 0; e < 8; ++e) s += f[e];
            }
        return s;
    }
};

// dweight's right operand: quads of h's rows, K of them per lane (8 q + j, or 4 j + q), which the workgroup has just read: this time they come from the L2.
// They are asked for a step ahead, and the rows that are left out are blanked when they are used.
template <typename T>
struct OuterRows {
    static constexpr bool two = __is_same(T, bf16);
    static constexpr int K = two ? 8 : 4, step = two ? 32 : 16;
    uint64_t h;        // the tile's first row, the same for all lanes
    uint32_t pitch;    // bytes from one row to the next
    uint32_t column;   // bytes of this lane's first column
    uint32_t last;     // bytes of the last row of the tile that is there
    int room;          // columns from this lane's first one on
    bool whole;        // every lane has four (the same for all lanes)
    __device__ inline static int row_of(int j) {
        const int q = lane_id() >> 4;
        return two ? 8 * q + j : 4 * j + q;
    }
    __device__ inline void ask(int k0, Quad<T> (&x)[K]) const {
        if (whole) {
            for (int j = 0; j < K; ++j) x[j].load(h, min((uint32_t)(k0 + row_of(j)) * pitch, last) + column);
        } else {
            for (int j = 0; j < K; ++j)
                x[j] = load_quad(reinterpret_cast<const T*>(h + min((uint32_t)(k0 + row_of(j)) * pitch, last) + column), 0, room);
        }
    }
    // kept: a bit per row of the tile, 32 to a word.
    __device__ inline static void blank(const uint32_t* kept, int k0, Quad<T> (&x)[K]) {
        const int word = (int)kept[k0 >> 5] >> (k0 & 31);
        for (int j = 0; j < K; ++j) {
            const uint32_t mask = (uint32_t)__builtin_amdgcn_sbfe(word, row_of(j), 1);
            for (int e = 0; e < Quad<T>::words; ++e) x[j].d[e] &= mask;
        }
    }
};

// acc[ct][t] += dz^T h for the rows k0 .. k0 + step - 1 of the tile.
template <int CT>
__device__ inline void outer_step(const SharedDz<bf16, CT>& dz, int k0, const Quad<bf16> (&x)[8], f32x4 (&acc)[CT][4]) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    u32x4 right[4];
    for (int t = 0; t < 4; ++t) right[t] = column_of(x, t);
    for (int ct = 0; ct < CT; ++ct)
        for (int k = 2; k >= 0; --k) {
            const u32x4 term = *reinterpret_cast<const u32x4*>(dz.at(k, 16 * ct + r, k0 + 8 * q));
            for (int t = 0; t < 4; ++t) acc[ct][t] = mma(term, right[t], acc[ct][t], bf16());
        }
}
template <int CT, typename T>
__device__ inline void outer_step(const SharedDz<T, CT>& dz, int k0, const Quad<T> (&x)[4], f32x4 (&acc)[CT][4]) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    for (int j = 0; j < 4; ++j)
        for (int ct = 0; ct < CT; ++ct) {
            const float left = dz.p[(k0 + 4 * j + q) * SharedDz<T, CT>::ld + 16 * ct + r];
            for (int t = 0; t < 4; ++t) acc[ct][t] = mma4(left, x[j].get(t), acc[ct][t]);
        }
}

// How many waves share the rows of a tile for one group of columns of dweight: those that the groups leave, but a wave has whole steps.
template <typename T>
__host__ __device__ inline int fused_splits(int groups, int waves) {
    const int most = 16 * waves / (__is_same(T, bf16) ? 32 : 16);
    int splits = waves;
    while (splits > 1 && (splits > most || splits * groups > waves)) splits >>= 1;
    return splits;
}

// Logits, loss, dz, dh and dweight of a tile of rows, one after the other: switched off one at a time (1M x 256, 50 classes, then 379 us, with dh from two terms
// of dz), dweight was worth 83 us, dh 103, the logits 63: with two waves to a SIMD they hardly overlap, and registers (238) and shared memory (62 KB) leave room
// for no third.
// Workgroups stay: W is copied to shared memory once, and a wave keeps its columns of dweight (GPW groups of 64, a quad for each of 16 lanes) in registers
// over all tiles of 64 or 128 rows.  Where there are fewer groups of columns than waves, several waves share the rows.
template <typename T, int CT, int GPW>
__global__ __launch_bounds__(kWave * fused_waves(CT), CT <= 2 ? 4 : 3 - GPW) void k_head_fused(Head a, Loss g, float* part) {
    constexpr int kCols = kFusedColumns, kWaves = fused_waves(CT), NT = 1, kFusedRows = fused_rows(CT);
    extern __shared__ char space[];
    const int q = lane_id() >> 4, r = lane_id() & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const SharedWeight<T> w = share_weight<T, CT>(a, reinterpret_cast<T*>(space));
    char* behind = space + shared_bytes<T, CT>(a.dim);
    SharedDz<T, CT> dz{reinterpret_cast<float*>(behind)};
    uint32_t* kept = reinterpret_cast<uint32_t*>(behind + SharedDz<T, CT>::bytes);  // a bit per row of the tile
    uint16_t* kept16 = reinterpret_cast<uint16_t*>(kept);
    const int groups = (a.dim + kCols - 1) / kCols, splits = fused_splits<T>(groups, kWaves);
    const int my_group = wave / splits, my_split = wave % splits;
    const int from = my_split * (kFusedRows / splits), to = from + kFusedRows / splits;
    f32x4 acc[GPW][CT][4];
    for (int p = 0; p < GPW; ++p)
        for (int ct = 0; ct < CT; ++ct)
            for (int t = 0; t < 4; ++t) acc[p][ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int my_class = threadIdx.x % (16 * CT), my_rows = threadIdx.x / (16 * CT) * 16;  // of dbias: 16 rows of the tile
    float sum = 0.f;
    using Right = OuterRows<T>;
    const int mine = wave * (16 * NT);
#pragma unroll 1
    for (int64_t tile = (int64_t)blockIdx.x * kFusedRows; tile < a.rows; tile += (int64_t)gridDim.x * kFusedRows) {
        {
            f32x4 z[NT][CT];
            RowTarget<CT> target[NT];
            bool use[NT];
            for (int m = 0; m < NT; ++m) target[m].ask(a, g, tile + mine + 16 * m + r, tile + kFusedRows + 64 <= a.rows);
            head_logits<T, CT, NT, 2>(a, w, tile + mine, z);
            for (int m = 0; m < NT; ++m) {
                const int row = mine + 16 * m + r;
                use[m] = head_dz(g, tile + row, a.rows, target[m], z[m]);
                const uint16_t bits = (uint16_t)__ballot(use[m]);
                if (lane_id() == 0) kept16[wave * NT + m] = bits;
                if constexpr (!__is_same(T, bf16))
                    for (int t = 0; t < CT; ++t) dz.put(row, t, q, z[m][t]);
            }
            if constexpr (__is_same(T, bf16)) {
                DzTerms<CT> terms[NT];
                for (int m = 0; m < NT; ++m) {
                    terms[m].make(z[m]);
                    dz.put(mine + 16 * m + r, q, terms[m]);
                }
                if (g.dh) head_dh<CT, NT>(a, w, tile + mine, terms, use, static_cast<T*>(g.dh), g.ld_dh);
            } else if (g.dh) {
                head_dh<CT, NT>(a, w, tile + mine, z, use, static_cast<T*>(g.dh), g.ld_dh);
            }
        }
        const int last = (int)min((int64_t)kFusedRows, a.rows - tile) - 1;
#pragma unroll
        for (int p = 0; p < GPW; ++p) {
            const int col = (my_group + kWaves * p) * kCols + 4 * r;
            const bool owner = my_group + kWaves * p < groups;
            const uint32_t pitch = (uint32_t)(a.ld_h * sizeof(T));
            const Right right{reinterpret_cast<uint64_t>(static_cast<const T*>(a.h) + tile * a.ld_h), pitch,
                              (uint32_t)min(col, a.dim - 1) * (uint32_t)sizeof(T), (uint32_t)last * pitch, a.dim - col, (my_group + kWaves * p + 1) * kCols <= a.dim};
            Quad<T> x[Right::K], next[Right::K];
            if (owner) right.ask(from, next);
            if (p == 0) {
                __syncthreads();
                for (int at = my_rows; at < kFusedRows; at += kWave * kWaves / (16 * CT) * 16) sum += dz.rows_of(my_class, at);
            }
            if (owner)
#pragma unroll 1
                for (int k0 = from; k0 < to; k0 += Right::step) {
                    for (int j = 0; j < Right::K; ++j) x[j] = next[j];
                    if (k0 + Right::step < to) right.ask(k0 + Right::step, next);
                    Right::blank(kept, k0, x);
                    outer_step(dz, k0, x, acc[p]);
                }
        }
        __syncthreads();
    }
    part += (int64_t)blockIdx.x * a.classes * (a.dim + 1);
    float* bias = reinterpret_cast<float*>(behind);
    bias[threadIdx.x] = sum;
    __syncthreads();
    if ((int)threadIdx.x < a.classes) {
        float v = 0.f;
        for (int k = threadIdx.x; k < kWave * kWaves / (16 * CT) * (16 * CT); k += 16 * CT) v += bias[k];
        part[(int64_t)threadIdx.x * (a.dim + 1) + a.dim] = v;
    }
    // dweight: the parts of waves that shared a group's rows, halves of them at a time; in place of everything else in shared memory
    f32x4* slots = reinterpret_cast<f32x4*>(space);
    for (int half = splits >> 1; half > 0; half >>= 1) {
        __syncthreads();
        if (my_group < groups && my_split >= half && my_split < 2 * half)
            for (int ct = 0; ct < CT; ++ct)
                for (int t = 0; t < 4; ++t) slots[((my_group * half + my_split - half) * CT * 4 + ct * 4 + t) * kWave + lane_id()] = acc[0][ct][t];
        __syncthreads();
        if (my_group < groups && my_split < half)
            for (int ct = 0; ct < CT; ++ct)
                for (int t = 0; t < 4; ++t) acc[0][ct][t] += slots[((my_group * half + my_split) * CT * 4 + ct * 4 + t) * kWave + lane_id()];
    }
    if (my_split != 0) return;
#pragma unroll
    for (int p = 0; p < GPW; ++p) {
        const int col = (my_group + kWaves * p) * kCols + 4 * r;
        for (int ct = 0; ct < CT; ++ct)
            for (int i = 0; i < 4; ++i) {
                const int c = 16 * ct + 4 * q + i;
                const float f[4] = {acc[p][ct][0][i], acc[p][ct][1][i], acc[p][ct][2][i], acc[p][ct][3][i]};
                if (c < a.classes && col < a.dim) store_columns(part + (int64_t)c * (a.dim + 1), col, a.dim, f);
            }
    }
}

// Bytes of shared memory of k_head_fused.
template <typename T, int CT>
inline int64_t fused_bytes(int dim) {
    // in the end, the parts of half the waves: with one group of columns, all of them share its rows
    const int64_t slots = (fused_waves(CT) / 2) * 16 * CT * kFusedColumns * 4, all = shared_bytes<T, CT>(dim) + SharedDz<T, CT>::bytes + fused_rows(CT) / 8;
    return all > slots ? all : slots;
}

// Sums the parts: 16 neighbouring elements per turn of a workgroup, 16 groups of lanes taking turns on the parts, then joined in order.
__global__ __launch_bounds__(kBlock) void k_head_join(const float* part, int splits, int classes, int dim, float* dweight, float* dbias) {
    __shared__ float sums[16][17];
    const int e = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t size = (int64_t)classes * (dim + 1);
    for (int64_t first = (int64_t)blockIdx.x * 16; first < size; first += (int64_t)gridDim.x * 16) {
        const int64_t at = first + e;
        float s = 0.f;
        if (at < size)
#pragma unroll 8
            for (int k = g; k < splits; k += 16) s += part[k * size + at];
        sums[g][e] = s;
        __syncthreads();
        if (g == 0 && at < size) {
            for (int k = 1; k < 16; ++k) s += sums[k][e];
            const int c = (int)(at / (dim + 1)), k = (int)(at - (int64_t)c * (dim + 1));
            if (k < dim) {
                if (dweight) dweight[(int64_t)c * dim + k] = s;
            } else if (dbias) {
                dbias[c] = s;
            }
        }
        __syncthreads();
    }
}

}  // namespace dynlp
