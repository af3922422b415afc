// The class head: logits, class distributions, cross entropy and its gradients.  Dense products on the matrix cores.
//
// Fragments of v_mfma_f32_16x16x{32,4}: lane l = 16 q + r (q = 0 .. 3, r = 0 .. 15) gives row r of the left operand, column r of the right
// one and holds rows 4 q .. 4 q + 3 of column r of the result.  Which k of the product a lane's operand elements stand for is free as
// long as both operands agree, and so is which columns of a matrix stand behind the 16 rows or columns of a tile; both are chosen
// here so that every lane reads 16 consecutive bytes and the result of one product is, as it lies in the registers, an operand of the
// next:
//   logits   z^T = W h^T.   Lane (q, r): W of class r, h of row r, columns k0 + 2 n q ... of a piece of n elements (a lane's two pieces
//            fill its part of a 128-byte line).  Result: row r's logits of classes 16 t + 4 q + i.
//   dh       dh^T = W^T dz^T.  The right operand (k = class, column = row r) is what the lane holds after the softmax.  The left one
//            needs W by columns: pieces of W's rows, for two-byte types transposed between registers.  Result: row r, n consecutive columns.
//   dweight  dz^T h.  Both operands are read row by row of h and dz, h in pieces, transposed between registers where needed.
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
template <typename T>
__device__ inline void store_quad(T* row, int col, int dim, const float (&f)[4]) {
    if (col + 4 <= dim) {
        store_values<4>(row + col, f);
    } else {
        for (int k = 0; k < 4; ++k)
            if (col + k < dim) row[col + k] = (T)f[k];
    }
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
    int64_t ld;
    int dim, classes;
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
    int ld;
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
    const WeightRows<T> w{static_cast<const T*>(a.weight), a.ld_w, a.dim, a.classes};
    for (int at = threadIdx.x; at < 16 * CT * pieces; at += kBlock)
        *reinterpret_cast<u32x4*>(to + at * n) = w.piece(at / pieces, at % pieces * n);
    __syncthreads();
    return SharedWeight<T>{to, ld};
}

// z[m][t] = logits of rows first + 16 m + r, classes 16 t + 4 q + i, bias added; -infinity beyond the classes.  The next step's part of h is
// asked for before this step's products.
template <typename T, int CT, int NT, typename W>
__device__ inline void head_logits(const Head& a, const W& w, int64_t first, f32x4 (&z)[NT][CT]) {
    constexpr int n = Piece<T>::n;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* h = static_cast<const T*>(a.h);
    const T* hr[NT];
    for (int m = 0; m < NT; ++m) {
        hr[m] = h + min(first + 16 * m + r, a.rows - 1) * a.ld_h;
        for (int t = 0; t < CT; ++t) z[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    u32x4 now[NT][2], next[NT][2];
    auto ask = [&](int k0) {
        for (int m = 0; m < NT; ++m)
            for (int s = 0; s < 2; ++s) next[m][s] = load_columns(hr[m], k0 + q * 2 * n + s * n, a.dim);
    };
    ask(0);
#pragma unroll 1
    for (int k0 = 0; k0 < a.dim; k0 += 8 * n) {
        for (int m = 0; m < NT; ++m)
            for (int s = 0; s < 2; ++s) now[m][s] = next[m][s];
        if (k0 + 8 * n < a.dim) ask(k0 + 8 * n);
#pragma unroll
        for (int s = 0; s < 2; ++s)
            for (int t = 0; t < CT; ++t) {
                const u32x4 wv = w.piece(16 * t + r, k0 + q * 2 * n + s * n);
                for (int m = 0; m < NT; ++m) z[m][t] = mma(wv, now[m][s], z[m][t], T());
            }
    }
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) {
            const int c = 16 * t + 4 * q + i;
            const float b = c < a.classes && a.bias ? a.bias[c] : 0.f;
            for (int m = 0; m < NT; ++m) z[m][t][i] = c < a.classes ? z[m][t][i] + b : -INFINITY;
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
            // (-infinity)^0: a row of nothing else keeps sum 0; +infinity - +infinity is not a number, as it should be
            z[t][i] = m == -INFINITY && z[t][i] == -INFINITY ? 0.f : expf(z[t][i] - m);
            sum += z[t][i];
        }
    *top = m;
    return row_sum(sum);
}

constexpr int kHeadTiles = 2;                       // tiles of 16 rows per wave
constexpr int kHeadRows = kHeadTiles * 16 * (kBlock / kWave);  // rows per workgroup

// One tile of rows per wave from W as it is, or (SHARED) any number of them from a copy of W in shared memory.
template <typename T, int CT, bool SHARED>
__global__ __launch_bounds__(kBlock) void k_head_labels(Head a, float* soft, int32_t* hard) {
    constexpr int NT = kHeadTiles;
    extern __shared__ char space[];
    const int q = lane_id() >> 4, r = lane_id() & 15;
    auto tile = [&](const auto& w, int64_t first) {
        f32x4 z[NT][CT];
        head_logits<T, CT, NT>(a, w, first, z);
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
                const float sum = head_exp(z[m], &top);
                if (row < a.rows)
                    for (int t = 0; t < CT; ++t) {
                        float f[4];
                        for (int i = 0; i < 4; ++i) f[i] = sum == 0.f ? 1.f / (float)a.classes : z[m][t][i] / sum;
                        if (16 * t + 4 * q < a.classes) store_columns(soft + row * a.classes, 16 * t + 4 * q, a.classes, f);
                    }
            }
        }
    };
    const int64_t first = (threadIdx.x / kWave) * (NT * 16);
    if constexpr (SHARED) {
        const SharedWeight<T> w = share_weight<T, CT>(a, reinterpret_cast<T*>(space));
        for (int64_t at = (int64_t)blockIdx.x * kHeadRows; at + first < a.rows; at += (int64_t)gridDim.x * kHeadRows) tile(w, at + first);
    } else {
        const WeightRows<T> w{static_cast<const T*>(a.weight), a.ld_w, a.dim, a.classes};
        if ((int64_t)blockIdx.x * kHeadRows + first < a.rows) tile(w, (int64_t)blockIdx.x * kHeadRows + first);
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

// x = high + low (+ what 16 or more further bits would hold), both bfloat16.
__device__ inline uint32_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (bf16)x); }

// dh of the tile's rows from their dz, 64 columns at a time.  Quads of W's rows are the left operand; in bfloat16 a lane's 8 x 4 block (8 classes, 4
// columns) is transposed by v_perm.
template <int CT, int NT, typename T>
__device__ inline void store_dh(const Head& a, int64_t first, int base, const f32x4 (&acc)[NT][4], const bool (&kept)[NT], T* dh, int64_t ld_dh) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    for (int m = 0; m < NT; ++m) {
        const int64_t row = first + 16 * m + r;
        if (row >= a.rows) continue;
        for (int i = 0; i < 4; ++i) {
            const int to = base + 4 * (4 * q + i);
            float f[4];
            for (int t = 0; t < 4; ++t) f[t] = kept[m] ? acc[m][t][i] : 0.f;
            if (to < a.dim) store_quad(dh + row * ld_dh, to, a.dim, f);
        }
    }
}
template <int CT, int NT, typename W>
__device__ inline void head_dh(const Head& a, const W& w, int64_t first, const f32x4 (&dz)[NT][CT], const bool (&kept)[NT], bf16* dh,
                               int64_t ld_dh) {
    constexpr int P = (CT + 1) / 2;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    // dz in two bfloat16 terms, which leave out 2^-17 of it: far below the rounding of dh itself
    u32x4 high[NT][P], low[NT][P];
    for (int m = 0; m < NT; ++m)
        for (int p = 0; p < P; ++p)
            for (int j = 0; j < 8; j += 2) {
                uint32_t hi = 0, lo = 0;
                for (int e = 0; e < 2; ++e) {
                    const int t = 2 * p + (j >> 2);
                    const float x = t < CT ? dz[m][t < CT ? t : 0][(j + e) & 3] : 0.f;
                    const uint32_t b = bf16_bits(x);
                    hi |= b << (16 * e);
                    lo |= bf16_bits(x - __uint_as_float(b << 16)) << (16 * e);
                }
                high[m][p][j >> 1] = hi;
                low[m][p][j >> 1] = lo;
            }
#pragma unroll 1
    for (int base = 0; base < a.dim; base += 64) {
        f32x4 acc[NT][4];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < P; ++p) {
            Quad<bf16> x[8];
            for (int j = 0; j < 8; ++j) {
                const int t = 2 * p + (j >> 2);
                if (t < CT)
                    x[j] = w.quad(16 * t + 4 * q + (j & 3), base + 4 * r);
                else
                    x[j].zero();
            }
            for (int t = 0; t < 4; ++t) {
                const u32x4 left = column_of(x, t);
                for (int m = 0; m < NT; ++m) {
                    acc[m][t] = mma(left, low[m][p], acc[m][t], bf16());
                    acc[m][t] = mma(left, high[m][p], acc[m][t], bf16());
                }
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
        f32x4 acc[NT][4];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < 4; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int ct = 0; ct < CT; ++ct)
            for (int i = 0; i < 4; ++i) {
                const Quad<T> x = w.quad(16 * ct + 4 * q + i, base + 4 * r);
                for (int t = 0; t < 4; ++t)
                    for (int m = 0; m < NT; ++m) acc[m][t] = mma4(x.get(t), dz[m][ct][i], acc[m][t]);
            }
        store_dh<CT, NT>(a, first, base, acc, kept, dh, ld_dh);
    }
}

// From the logits z of row `row` of a lane (first + 16 m + r): its loss is stored, z becomes dz.  Returns whether the row takes part.
template <int CT>
__device__ inline bool head_dz(const Head& a, const Loss& g, int64_t row, f32x4 (&z)[CT]) {
    const int q = lane_id() >> 4;
    const bool inside = row < a.rows;
    const int64_t at = inside ? row : a.rows - 1;
    const float weight = g.row_weight ? g.row_weight[at] : 1.f;
    bool use = inside && weight != 0.f;
    int label = -1;
    f32x4 target[CT];
    if (g.hard) {
        label = g.hard[at];
        if (inside && q == 0 && label >= a.classes && g.rejected) atomicAdd(g.rejected, 1);
        use = use && label >= 0 && label < a.classes;
    }
    for (int t = 0; t < CT; ++t) {
        const int c = 16 * t + 4 * q;
        if (g.hard)
            for (int i = 0; i < 4; ++i) target[t][i] = c + i == label ? 1.f : 0.f;
        else
            target[t] = __builtin_bit_cast(f32x4, c < a.classes ? load_columns(g.soft + at * a.classes, c, a.classes) : u32x4{0u, 0u, 0u, 0u});
    }
    f32x4 e[CT];
    for (int t = 0; t < CT; ++t) e[t] = z[t];
    float top;
    const float sum = head_exp(e, &top);
    use = use && sum != 0.f;
    const float lse = logf(sum);  // of the shifted logits
    float total = 0.f, loss = 0.f;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) {
            const float y = target[t][i];
            total += y;
            loss += y != 0.f ? y * (lse - (z[t][i] - top)) : 0.f;
        }
    total = row_sum(total);
    loss = row_sum(loss);
    const float scale = g.grad_scale * weight;
    for (int t = 0; t < CT; ++t)
        for (int i = 0; i < 4; ++i) z[t][i] = use ? scale * (total * (e[t][i] / sum) - target[t][i]) : 0.f;
    if (inside && q == 0 && g.loss) g.loss[row] = use ? weight * loss : 0.f;
    return use;
}

// Loss, dz and dh of a tile of rows: logits, softmax and the product with W, without leaving the registers.  For heads whose W and dweight do
// not fit a workgroup, and where no dweight is asked for.
template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_head_loss(Head a, Loss g) {
    constexpr int NT = kHeadTiles;
    const int64_t first = (int64_t)blockIdx.x * kHeadRows + (threadIdx.x / kWave) * (NT * 16);
    if (first >= a.rows) return;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const WeightRows<T> w{static_cast<const T*>(a.weight), a.ld_w, a.dim, a.classes};
    f32x4 z[NT][CT];
    bool kept[NT];
    head_logits<T, CT, NT>(a, w, first, z);
    for (int m = 0; m < NT; ++m) {
        const int64_t row = first + 16 * m + r;
        kept[m] = head_dz(a, g, row, z[m]);
        if (row < a.rows && g.dz) {
            if (q == 0) g.kept[row] = kept[m] ? 1 : 0;
            for (int t = 0; t < CT; ++t) *reinterpret_cast<f32x4*>(g.dz + row * (16 * CT) + 16 * t + 4 * q) = z[m][t];
        }
    }
    if (g.dh) head_dh<CT, NT>(a, w, first, z, kept, static_cast<T*>(g.dh), g.ld_dh);
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
                uint32_t b[3] = {0, 0, 0};
                for (int e = 0; e < 2; ++e) {
                    float v = a[t][j >> 2][(j + e) & 3];
                    sum[t] += v;
                    for (int k = 0; k < 3; ++k) {
                        const uint32_t bits = bf16_bits(v);
                        b[k] |= bits << (16 * e);
                        v -= __uint_as_float(bits << 16);
                    }
                }
                for (int k = 0; k < 3; ++k) term[k][t][j >> 1] = b[k];
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

// dz of a workgroup's 128 rows in shared memory: [row][class], padded so that the four row groups that a wave reads at once (4 j + q, or 8 q + j
// for bfloat16) lie in different banks.
template <typename T, int CT>
struct SharedDz {
    static constexpr int ld = 16 * CT + (sizeof(T) == 2 && !__is_same(T, f16) ? 2 : 16), bytes = kHeadRows * ld * 4;
    float* p;
    __device__ inline void put(int row, int t, int q, const f32x4& z) {
        float2* to = reinterpret_cast<float2*>(p + row * ld + 16 * t + 4 * q);
        to[0] = float2{z[0], z[1]};
        to[1] = float2{z[2], z[3]};
    }
    // Sum of a class over 32 rows.
    __device__ inline float rows_of(int c, int from) const {
        float s = 0.f;
        for (int k = 0; k < 32; ++k) s += p[(from + k) * ld + c];
        return s;
    }
};

// acc[ct][t] += rows from .. to of the tile, columns col + t.  h is read once more here, from the L2: the workgroup has just read it.
template <int CT>
__device__ inline void tile_outer(const Head& a, int64_t tile, int from, int to, int col, const SharedDz<bf16, CT>& dz, const uint8_t* kept,
                                  f32x4 (&acc)[CT][4]) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const bf16* h = static_cast<const bf16*>(a.h);
#pragma unroll 1
    for (int k0 = from; k0 < to; k0 += 32) {
        Quad<bf16> x[8];
        for (int j = 0; j < 8; ++j) {
            const int row = k0 + 8 * q + j;
            x[j].zero();
            if (kept[row] && col < a.dim) x[j] = load_quad(h + (tile + row) * a.ld_h, col, a.dim);
        }
        u32x4 right[4];
        for (int t = 0; t < 4; ++t) right[t] = column_of(x, t);
        for (int ct = 0; ct < CT; ++ct) {
            // dz in three bfloat16 terms, which hold all 24 bits of it: dweight is a float32 sum over all rows
            u32x4 term[3];
            for (int j = 0; j < 8; j += 2) {
                uint32_t b[3] = {0, 0, 0};
                for (int e = 0; e < 2; ++e) {
                    float v = dz.p[(k0 + 8 * q + j + e) * SharedDz<bf16, CT>::ld + 16 * ct + r];
                    for (int k = 0; k < 3; ++k) {
                        const uint32_t bits = bf16_bits(v);
                        b[k] |= bits << (16 * e);
                        v -= __uint_as_float(bits << 16);
                    }
                }
                for (int k = 0; k < 3; ++k) term[k][j >> 1] = b[k];
            }
            for (int k = 2; k >= 0; --k)
                for (int t = 0; t < 4; ++t) acc[ct][t] = mma(term[k], right[t], acc[ct][t], bf16());
        }
    }
}
template <int CT, typename T>
__device__ inline void tile_outer(const Head& a, int64_t tile, int from, int to, int col, const SharedDz<T, CT>& dz, const uint8_t* kept,
                                  f32x4 (&acc)[CT][4]) {
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* h = static_cast<const T*>(a.h);
#pragma unroll 1
    for (int k0 = from; k0 < to; k0 += 16) {
        Quad<T> x[4];
        for (int j = 0; j < 4; ++j) {
            const int row = k0 + 4 * j + q;
            x[j].zero();
            if (kept[row] && col < a.dim) x[j] = load_quad(h + (tile + row) * a.ld_h, col, a.dim);
        }
        for (int j = 0; j < 4; ++j)
            for (int ct = 0; ct < CT; ++ct) {
                const float left = dz.p[(k0 + 4 * j + q) * SharedDz<T, CT>::ld + 16 * ct + r];
                for (int t = 0; t < 4; ++t) acc[ct][t] = mma4(left, x[j].get(t), acc[ct][t]);
            }
    }
}

constexpr int kFusedColumns = 64;

// Workgroups stay: W is copied to shared memory once, and a wave keeps its columns of dweight in registers over all tiles of 128 rows.  The columns
// are cut into groups of 64 (a quad for each of 16 lanes).  One group: the four waves share the tile's rows; two: two waves
// each; more: each wave has GPW groups and all rows.
template <typename T, int CT, int GPW>
__global__ __launch_bounds__(kBlock, GPW == 1 ? 2 : 1) void k_head_fused(Head a, Loss g, float* part) {
    constexpr int NT = kHeadTiles, N = 4, kCols = kFusedColumns;
    extern __shared__ char space[];
    const int q = lane_id() >> 4, r = lane_id() & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const SharedWeight<T> w = share_weight<T, CT>(a, reinterpret_cast<T*>(space));
    char* behind = space + 16 * CT * w.ld * sizeof(T);
    SharedDz<T, CT> dz{reinterpret_cast<decltype(SharedDz<T, CT>::p)>(behind)};
    uint8_t* kept = reinterpret_cast<uint8_t*>(behind + SharedDz<T, CT>::bytes);
    const int groups = (a.dim + kCols - 1) / kCols;
    const int my_group = groups == 1 ? 0 : groups == 2 ? wave & 1 : wave;
    const int from = groups == 1 ? wave * (kHeadRows / 4) : groups == 2 ? (wave >> 1) * (kHeadRows / 2) : 0;
    const int to = groups == 1 ? from + kHeadRows / 4 : groups == 2 ? from + kHeadRows / 2 : kHeadRows;
    f32x4 acc[GPW][CT][N];
    for (int ct = 0; ct < CT; ++ct)
        for (int p = 0; p < GPW; ++p)
            for (int t = 0; t < N; ++t) acc[p][ct][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int my_class = threadIdx.x % (16 * CT), my_rows = threadIdx.x / (16 * CT) * 32;  // of dbias: 32 rows of the tile
    float sum = 0.f;
    for (int64_t tile = (int64_t)blockIdx.x * kHeadRows; tile < a.rows; tile += (int64_t)gridDim.x * kHeadRows) {
        const int mine = wave * (NT * 16);
        {
            f32x4 z[NT][CT];
            bool use[NT];
            head_logits<T, CT, NT>(a, w, tile + mine, z);
            for (int m = 0; m < NT; ++m) {
                const int row = mine + 16 * m + r;
                use[m] = head_dz(a, g, tile + row, z[m]);
                if (q == 0) kept[row] = use[m] ? 1 : 0;
                for (int t = 0; t < CT; ++t) dz.put(row, t, q, z[m][t]);
            }
            if (g.dh) head_dh<CT, NT>(a, w, tile + mine, z, use, static_cast<T*>(g.dh), g.ld_dh);
        }
        __syncthreads();
        if (my_rows < kHeadRows) sum += dz.rows_of(my_class, my_rows);
        for (int p = 0; p < GPW; ++p)
            if (my_group + 4 * p < groups) tile_outer(a, tile, from, to, (my_group + 4 * p) * kCols + N * r, dz, kept, acc[p]);
        __syncthreads();
    }
    part += (int64_t)blockIdx.x * a.classes * (a.dim + 1);
    float* bias = reinterpret_cast<float*>(behind);
    bias[threadIdx.x] = sum;
    __syncthreads();
    if ((int)threadIdx.x < a.classes) {
        float v = 0.f;
        for (int k = 0; k < kHeadRows / 32; ++k) v += bias[k * 16 * CT + threadIdx.x];
        part[(int64_t)threadIdx.x * (a.dim + 1) + a.dim] = v;
    }
    // dweight: a group of columns after the other, its waves' parts added in order
    float* joined = reinterpret_cast<float*>(behind);
    for (int k = 0; k < groups; ++k) {
        const bool owner = groups <= 2 ? my_group == k : wave == (k & 3);
        __syncthreads();
        for (int turn = 0; turn < (groups == 1 ? 4 : groups == 2 ? 2 : 1); ++turn) {
            if (owner && (groups == 1 ? wave == turn : groups == 2 ? wave >> 1 == turn : true))
                for (int p = 0; p < GPW; ++p)
                    if (p == (groups <= 2 ? 0 : k >> 2))
                        for (int ct = 0; ct < CT; ++ct)
                            for (int t = 0; t < N; ++t)
                                for (int i = 0; i < 4; ++i) {
                                    float& to_sum = joined[(16 * ct + 4 * q + i) * (kCols + 1) + N * r + t];
                                    to_sum = turn ? to_sum + acc[p][ct][t][i] : acc[p][ct][t][i];
                                }
            __syncthreads();
        }
        for (int at = threadIdx.x; at < a.classes * kCols; at += kBlock) {
            const int c = at / kCols, col = at % kCols;
            if (k * kCols + col < a.dim) part[(int64_t)c * (a.dim + 1) + k * kCols + col] = joined[c * (kCols + 1) + col];
        }
    }
}

// Bytes of shared memory of k_head_fused.
template <typename T, int CT>
inline int64_t fused_bytes(int dim) {
    const int64_t joined = 16 * CT * (kFusedColumns + 1) * 4, dz = SharedDz<T, CT>::bytes + kHeadRows;
    return (int64_t)16 * CT * shared_ld<T>(dim) * (int64_t)sizeof(T) + (joined > dz ? joined : dz);
}

// Sums the parts: 16 neighbouring elements per workgroup, 16 groups of lanes taking turns on the parts, then joined in order.
__global__ __launch_bounds__(kBlock) void k_head_join(const float* part, int splits, int classes, int dim, float* dweight, float* dbias) {
    __shared__ float sums[16][17];
    const int e = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t size = (int64_t)classes * (dim + 1);
    const int64_t at = (int64_t)blockIdx.x * 16 + e;
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
}

}  // namespace dynlp
