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

// z[m][t] = logits of rows first + 16 m + r, classes 16 t + 4 q + i, bias added; -infinity beyond the classes.
template <typename T, int CT, int NT>
__device__ inline void head_logits(const Head& a, int64_t first, f32x4 (&z)[NT][CT]) {
    constexpr int n = Piece<T>::n;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* w = static_cast<const T*>(a.weight);
    const T* h = static_cast<const T*>(a.h);
    const T* wr[CT];
    const T* hr[NT];
    for (int t = 0; t < CT; ++t) wr[t] = w + (int64_t)min(16 * t + r, a.classes - 1) * a.ld_w;
    for (int m = 0; m < NT; ++m) {
        hr[m] = h + min(first + 16 * m + r, a.rows - 1) * a.ld_h;
        for (int t = 0; t < CT; ++t) z[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int k0 = 0; k0 < a.dim; k0 += 8 * n) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int col = k0 + q * 2 * n + s * n;
            u32x4 wv[CT], hv[NT];
            for (int m = 0; m < NT; ++m) hv[m] = load_columns(hr[m], col, a.dim);
            for (int t = 0; t < CT; ++t) wv[t] = load_columns(wr[t], col, a.dim);
            for (int t = 0; t < CT; ++t)
                for (int m = 0; m < NT; ++m) z[m][t] = mma(wv[t], hv[m], z[m][t], T());
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

template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_head_labels(Head a, float* soft, int32_t* hard) {
    constexpr int NT = kHeadTiles;
    const int64_t first = (int64_t)blockIdx.x * kHeadRows + (threadIdx.x / kWave) * (NT * 16);
    if (first >= a.rows) return;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    f32x4 z[NT][CT];
    head_logits<T, CT, NT>(a, first, z);
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
            if (row < a.rows) {
                float* out = soft + row * a.classes;
                for (int t = 0; t < CT; ++t)
                    for (int i = 0; i < 4; ++i) {
                        const int c = 16 * t + 4 * q + i;
                        if (c < a.classes) out[c] = sum == 0.f ? 1.f / (float)a.classes : z[m][t][i] / sum;
                    }
            }
        }
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

// dh of the tile's rows from their dz.  Pieces of W's rows are the left operand; for two-byte types a lane's 8 x 8 block (8 classes, 8
// columns) is transposed by v_perm.
template <int CT, int NT>
__device__ inline void head_dh(const Head& a, int64_t first, const f32x4 (&dz)[NT][CT], const bool (&kept)[NT], bf16* dh, int64_t ld_dh) {
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
    const bf16* w = static_cast<const bf16*>(a.weight);
    for (int base = 0; base < a.dim; base += 128) {
        f32x4 acc[NT][8];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < 8; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int col = base + 8 * r;
        for (int p = 0; p < P; ++p) {
            u32x4 x[8];
            for (int j = 0; j < 8; ++j) {
                const int c = 16 * (2 * p + (j >> 2)) + 4 * q + (j & 3);
                x[j] = u32x4{0u, 0u, 0u, 0u};
                if (c < a.classes && col < a.dim) x[j] = load_columns(w + (int64_t)c * a.ld_w, col, a.dim);
            }
            for (int t = 0; t < 8; ++t) {
                u32x4 left;
                for (int j = 0; j < 4; ++j)
                    left[j] = __builtin_amdgcn_perm(x[2 * j + 1][t >> 1], x[2 * j][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
                for (int m = 0; m < NT; ++m) {
                    acc[m][t] = mma(left, low[m][p], acc[m][t], bf16());
                    acc[m][t] = mma(left, high[m][p], acc[m][t], bf16());
                }
            }
        }
        for (int m = 0; m < NT; ++m) {
            const int64_t row = first + 16 * m + r;
            if (row >= a.rows) continue;
            for (int i = 0; i < 4; ++i) {
                const int to = base + 8 * (4 * q + i);
                float f[8];
                for (int t = 0; t < 8; ++t) f[t] = kept[m] ? acc[m][t][i] : 0.f;
                if (to < a.dim) store_columns(dh + row * ld_dh, to, a.dim, f);
            }
        }
    }
}
template <int CT, int NT, typename T>
__device__ inline void head_dh(const Head& a, int64_t first, const f32x4 (&dz)[NT][CT], const bool (&kept)[NT], T* dh, int64_t ld_dh) {
    constexpr int n = Piece<T>::n;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    const T* w = static_cast<const T*>(a.weight);
    for (int base = 0; base < a.dim; base += 16 * n) {
        f32x4 acc[NT][n];
        for (int m = 0; m < NT; ++m)
            for (int t = 0; t < n; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int col = base + n * r;
        for (int ct = 0; ct < CT; ++ct)
            for (int i = 0; i < 4; ++i) {
                const int c = 16 * ct + 4 * q + i;
                u32x4 x = {0u, 0u, 0u, 0u};
                if (c < a.classes && col < a.dim) x = load_columns(w + (int64_t)c * a.ld_w, col, a.dim);
                float f[n];
                widen(x, f, T());
                for (int t = 0; t < n; ++t)
                    for (int m = 0; m < NT; ++m) acc[m][t] = mma4(f[t], dz[m][ct][i], acc[m][t]);
            }
        for (int m = 0; m < NT; ++m) {
            const int64_t row = first + 16 * m + r;
            if (row >= a.rows) continue;
            for (int i = 0; i < 4; ++i) {
                const int to = base + n * (4 * q + i);
                float f[n];
                for (int t = 0; t < n; ++t) f[t] = kept[m] ? acc[m][t][i] : 0.f;
                if (to < a.dim) store_columns(dh + row * ld_dh, to, a.dim, f);
            }
        }
    }
}

// Loss, dz and dh of a tile of rows: logits, softmax and the product with W, without leaving the registers.
template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_head_loss(Head a, Loss g) {
    constexpr int NT = kHeadTiles;
    const int64_t first = (int64_t)blockIdx.x * kHeadRows + (threadIdx.x / kWave) * (NT * 16);
    if (first >= a.rows) return;
    const int q = lane_id() >> 4, r = lane_id() & 15;
    f32x4 z[NT][CT];
    bool kept[NT];
    head_logits<T, CT, NT>(a, first, z);
    for (int m = 0; m < NT; ++m) {
        const int64_t row = first + 16 * m + r;
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
            target[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (g.hard) {
                for (int i = 0; i < 4; ++i) target[t][i] = c + i == label ? 1.f : 0.f;
            } else {
                for (int i = 0; i < 4; ++i)
                    if (c + i < a.classes) target[t][i] = g.soft[at * a.classes + c + i];
            }
        }
        f32x4 e[CT];
        for (int t = 0; t < CT; ++t) e[t] = z[m][t];
        float top;
        const float sum = head_exp(e, &top);
        use = use && sum != 0.f;
        const float lse = logf(sum);  // of the shifted logits
        float total = 0.f, loss = 0.f;
        for (int t = 0; t < CT; ++t)
            for (int i = 0; i < 4; ++i) {
                const float y = target[t][i];
                total += y;
                loss += y != 0.f ? y * (lse - (z[m][t][i] - top)) : 0.f;
            }
        total = row_sum(total);
        loss = row_sum(loss);
        const float scale = g.grad_scale * weight;
        for (int t = 0; t < CT; ++t)
            for (int i = 0; i < 4; ++i) z[m][t][i] = use ? scale * (total * (e[t][i] / sum) - target[t][i]) : 0.f;
        kept[m] = use;
        if (inside) {
            if (q == 0 && g.loss) g.loss[row] = use ? weight * loss : 0.f;
            if (g.dz) {
                if (q == 0) g.kept[row] = use ? 1 : 0;
                for (int t = 0; t < CT; ++t) *reinterpret_cast<f32x4*>(g.dz + row * (16 * CT) + 16 * t + 4 * q) = z[m][t];
            }
        }
    }
    if (g.dh) head_dh<CT, NT>(a, first, z, kept, static_cast<T*>(g.dh), g.ld_dh);
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
