// Heads of any number of classes: logits, their softmax, and the divergence from a teacher of which a row keeps its first classes, with its gradients.
//
// A teacher's list of a row becomes q = softmax(u / T) over its entries.  With p = softmax(z / T) over all classes:
//   loss = r T^2 sum q (log q - log p),   dz = grad_scale r T (p - q),   dh = dz W,   dweight = dz^T h,   dbias = sum of dz over rows
// Logits do not go through memory: the product h W^T is made twice, for the sums of the softmax and again for dz, of which 16-bit terms are stored for the products
// with W and h (k_wide, classes as its fast index m, rows as n).  A head's own rounding needs one term; dweight in 32 bits takes as many as hold dz.
#pragma once

#include "dynlp_teacher.h"
#include "dynlp_wide.h"

namespace dynlp {

// Rows as 16-bit terms with zeros up to ld_out, a multiple of 32.  Bfloat16 terms of 32-bit values are each the nearest to what is left, and hold all 24 bits.
template <typename T>
__device__ inline void terms_of(float x, uint16_t (&term)[3]) {
    for (int k = 0; k < 3; ++k) {
        uint16_t b = (uint16_t)bf16_pair(x, 0.f);
        float v = __uint_as_float((uint32_t)b << 16);
        if (fabsf(v) == INFINITY && fabsf(x) != INFINITY) {  // a value that rounding makes infinite is cut off instead
            b = (uint16_t)(__float_as_uint(x) >> 16);
            v = __uint_as_float((uint32_t)b << 16);
        }
        term[k] = b;
        x = fabsf(x) < INFINITY ? x - v : 0.f;
    }
}
template <typename T>
__global__ __launch_bounds__(kBlock) void k_lay_out(const T* in, int64_t ld, int64_t rows, int dim, uint16_t* out, int64_t ld_out, int64_t term) {
    const int64_t pieces = ld_out / 8, total = rows * pieces;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / pieces;
        const int col = (int)(at - row * pieces) * 8;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4*>(out + row * ld_out + col) = col < dim ? load_columns(in + row * ld, col, dim) : u32x4{0u, 0u, 0u, 0u};
        } else {
            u32x4 v[3];
            for (int k = 0; k < 8; k += 2) {
                uint16_t a[3], b[3];
                terms_of<T>(col + k < dim ? in[row * ld + col + k] : 0.f, a);
                terms_of<T>(col + k + 1 < dim ? in[row * ld + col + k + 1] : 0.f, b);
                for (int t = 0; t < 3; ++t) v[t][k / 2] = a[t] | (uint32_t)b[t] << 16;
            }
            for (int t = 0; t < 3; ++t) *reinterpret_cast<u32x4*>(out + t * term + row * ld_out + col) = v[t];
        }
    }
}

// ---- logits -----------------------------------------------------------------------------------------------------------

// The tile's bias in shared memory: -infinity, which makes a logit so whatever h holds, for what is not a class.
template <typename S>
__device__ inline const float* tile_bias(const float* bias, int first, int classes, char* space) {
    float* b = reinterpret_cast<float*>(space);
    for (int k = threadIdx.x; k < S::TM; k += kBlock) b[k] = first + k >= classes ? -INFINITY : bias ? bias[first + k] : 0.f;
    __syncthreads();
    return b;
}
__device__ inline void add_bias(const float* b, float (&v)[16]) {
    for (int k = 0; k < 16; k += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(b + k);
        for (int i = 0; i < 4; ++i) v[k + i] = x[i] == -INFINITY ? x[i] : v[k + i] + x[i];
    }
}

// Logits to memory; ld is a multiple of 16, and what lies behind the classes becomes -infinity.
struct Logits {
    float* z;
    int64_t ld;
    const float* bias;
    int rows, classes;
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        const float* b = tile_bias<S>(bias, at.tile_m * S::TM, classes, space) + at.wave_m * (16 * S::MI);
        const int q = lane_id() >> 4, r = lane_id() & 15;
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            if (n >= rows) continue;
            for (int j = 0; j < S::MI / 4; ++j) {
                const int m = at.m0 + 64 * j + 16 * q;
                if (m >= ld) continue;
                float v[16];
                sixteen(acc[i], j, v);
                add_bias(b + 64 * j + 16 * q, v);
                store_values<16>(z + n * ld + m, v);
            }
        }
    }
};

// ---- the teacher's lists ----------------------------------------------------------------------------------------------

// Lists that each name a class once (others: -1), their probabilities, sum of q log q and weight of the row (0: left out).
struct Lists {
    int32_t* classes;
    float* q;
    float* entropy;
    float* weight;
    uint32_t* largest;  // bits of the largest finite |weight|, or NULL
};

// zeros: 512 bytes of them.
__global__ __launch_bounds__(kBlock) inline void k_teach_begin(uint32_t* zeros, uint32_t* largest) {
    if (threadIdx.x < 128) zeros[threadIdx.x] = 0;
    if (threadIdx.x == 0) *largest = 0;
}

// 1 << log2 lanes per row, E entries for each.
template <int E>
__global__ __launch_bounds__(kBlock) void k_teach_lists(Teacher t, Lists out, int64_t row0, int64_t rows, int log2) {
    const int group = 1 << log2, me = threadIdx.x & (group - 1);
    const int64_t row = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> log2;
    const bool there = row < rows;
    const int64_t at = there ? row0 + row : row0;
    int c[E];
    float u[E], q[E];
    float top = -INFINITY;
    for (int e = 0; e < E; ++e) {
        const int k = e * group + me;
        c[e] = -1, u[e] = -INFINITY;
        if (there && k < t.kept) {
            c[e] = t.classes[at * t.kept + k];
            u[e] = t.logits[at * t.kept + k];
            if (c[e] >= t.count) {
                if (t.rejected) atomicAdd(t.rejected, 1);
                c[e] = -1;
            }
        }
        if (c[e] < 0) u[e] = -INFINITY;
        top = fmaxf(top, u[e]);
    }
    for (int d = 1; d < group; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, kWave));
    float sum = 0.f;
    for (int e = 0; e < E; ++e) {
        q[e] = u[e] == -INFINITY ? 0.f : expf((u[e] - top) * t.inverse);
        sum += q[e];
    }
    for (int d = 1; d < group; d <<= 1) sum += __shfl_xor(sum, d, kWave);
    const float log_sum = logf(sum);
    float entropy = 0.f;
    for (int e = 0; e < E; ++e) {
        if (sum != 0.f) q[e] /= sum;
        if (q[e] != 0.f) entropy += q[e] * ((u[e] - top) * t.inverse - log_sum);
    }
    for (int d = 1; d < group; d <<= 1) entropy += __shfl_xor(entropy, d, kWave);
    // classes that are named several times: the first gets all of it
    float all[E];
    bool first[E];
    for (int e = 0; e < E; ++e) all[e] = 0.f, first[e] = true;
    for (int k = 0; k < t.kept; ++k) {
        int other = c[0];
        float more = q[0];
        if (E > 1 && k >= group) other = c[E - 1], more = q[E - 1];
        other = __shfl(other, k & (group - 1), group);
        more = __shfl(more, k & (group - 1), group);
        for (int e = 0; e < E; ++e)
            if (other == c[e]) {
                if (k < e * group + me) first[e] = false;
                all[e] += more;
            }
    }
    if (!there) return;
    for (int e = 0; e < E; ++e) {
        const int k = e * group + me;
        if (k < t.kept) {
            out.classes[row * t.kept + k] = first[e] ? c[e] : -1;
            out.q[row * t.kept + k] = all[e];
        }
    }
    if (me == 0) {
        const float r = t.row_weight ? t.row_weight[at] : 1.f;
        const float weight = sum == 0.f ? 0.f : r;
        out.weight[row] = weight;
        out.entropy[row] = entropy;
        if (out.largest && fabsf(weight) < INFINITY) atomicMax(out.largest, __float_as_uint(fabsf(weight)));
    }
}

// A wave's part of the lists of 16 rows in shared memory: q of the wave's classes, row by row.
template <typename S>
struct ListTile {
    static constexpr int ld = 16 * S::MI + 4, bytes = 16 * ld * 4;
    float* p;
    // All zeros.
    __device__ void clear() const {
        for (int k = lane_id() * 4; k < 16 * ld; k += kWave * 4) *reinterpret_cast<f32x4*>(p + k) = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // Puts there, or takes away, what rows n .. n + 15 keep of classes m0 on.  Returns whether there is any.
    __device__ bool put(const int32_t* classes, const float* q, int kept, int n, int rows, int m0, bool away) const {
        const int r = lane_id() & 15;
        bool any = false;
        if (n + r < rows)
            for (int k = lane_id() >> 4; k < kept; k += 4) {
                const int64_t at = (int64_t)(n + r) * kept + k;
                const int c = classes[at] - m0;
                if (c >= 0 && c < 16 * S::MI && classes[at] >= 0) {
                    p[r * ld + c] = away ? 0.f : q[at];
                    any = true;
                }
            }
        return __any(any);
    }
    __device__ void get(int column, float (&v)[16]) const {
        for (int k = 0; k < 16; k += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p + (lane_id() & 15) * ld + column + k);
            for (int i = 0; i < 4; ++i) v[k + i] = x[i];
        }
    }
};
// A wave's own accesses of shared memory, in order.
__device__ inline void wave_meets() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

template <typename S>
constexpr int list_space() {
    return 4 * S::TM + 4 * ListTile<S>::bytes;
}

// Sums of the softmax: for every 16 MI classes and every row the largest logit m, sum of exp((z - m) / T), sum of q z.
struct Stats {
    const float* bias;
    const int32_t* classes;
    const float* q;
    float *top, *sum, *picked;  // [part][ld]
    int64_t ld;
    float exponent;             // log2(e) / T
    int rows, count, kept;
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        const float* b = tile_bias<S>(bias, at.tile_m * S::TM, count, space) + at.wave_m * (16 * S::MI);
        const ListTile<S> lists{reinterpret_cast<float*>(space + 4 * S::TM + (at.wave_m + S::WM * at.wave_n) * ListTile<S>::bytes)};
        lists.clear();
        const int lane_q = lane_id() >> 4, r = lane_id() & 15;
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i;
            wave_meets();
            const bool any = lists.put(classes, q, kept, n, rows, at.m0, false);
            wave_meets();
            float m = -INFINITY, pick = 0.f, z[S::MI / 4][16];
            for (int j = 0; j < S::MI / 4; ++j) {
                sixteen(acc[i], j, z[j]);
                add_bias(b + 64 * j + 16 * lane_q, z[j]);
                for (int k = 0; k < 16; ++k) m = fmaxf(m, z[j][k]);
                if (any) {
                    float y[16];
                    lists.get(64 * j + 16 * lane_q, y);
                    for (int k = 0; k < 16; ++k) pick += y[k] != 0.f ? y[k] * z[j][k] : 0.f;
                }
            }
            m = row_max(m);
            float s = 0.f;
            for (int j = 0; j < S::MI / 4; ++j)
                for (int k = 0; k < 16; ++k) s += z[j][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((z[j][k] - m) * exponent);
            s = row_sum(s);
            pick = row_sum(pick);
            if (lane_q == 0 && n + r < rows) {
                const int64_t to = (int64_t)(at.tile_m * S::WM + at.wave_m) * ld + n + r;
                top[to] = m, sum[to] = s, picked[to] = pick;
            }
            wave_meets();
            if (any) lists.put(classes, q, kept, n, rows, at.m0, true);
        }
    }
};

struct RowJoin {
    const float *top, *sum, *picked;  // [part][ld]
    int64_t ld;
    const float *entropy, *weight;    // of the lists
    const uint32_t* largest;          // of 16-bit floats with 5 bits of exponent, or NULL
    float* loss;                      // or NULL
    float* lse;                       // log2 of the sum of exp(z / T)
    float* factor;                    // weight times a power of two; 0 where the row is left out
    uint32_t* kept;                   // a bit per row
    float* undo;                      // one over that power
    float exponent, temperature;
    int rows, parts;
};
// The parts of 32 rows, by 8 threads each, in order.  The power of two brings the largest weight to 2^14 .. 2^15, so that float16 holds dz's terms.
__global__ __launch_bounds__(kBlock) inline void k_teach_rows(RowJoin g) {
    __shared__ float tops[8][32], sums[8][32], picks[8][32];
    const int r = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + r, at = min(row, g.rows - 1);
    float m = -INFINITY, s = 0.f, pick = 0.f;
    for (int p = k; p < g.parts; p += 8) {
        const float pm = g.top[p * g.ld + at], ps = g.sum[p * g.ld + at];
        pick += g.picked[p * g.ld + at];
        const float all = fmaxf(m, pm);
        s = (m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - all) * g.exponent)) + (pm == -INFINITY ? ps : ps * __builtin_amdgcn_exp2f((pm - all) * g.exponent));
        m = all;
    }
    tops[k][r] = m, sums[k][r] = s, picks[k][r] = pick;
    __syncthreads();
    if (k != 0) return;
    for (int p = 1; p < 8; ++p) {
        const float pm = tops[p][r], ps = sums[p][r], all = fmaxf(m, pm);
        pick += picks[p][r];
        s = (m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - all) * g.exponent)) + (pm == -INFINITY ? ps : ps * __builtin_amdgcn_exp2f((pm - all) * g.exponent));
        m = all;
    }
    const float weight = g.weight[at];
    const bool use = row < g.rows && weight != 0.f && s != 0.f;
    float scale = 1.f;
    if (g.largest) {
        int e;
        const float most = __uint_as_float(*g.largest);
        frexpf(most, &e);
        if (most > 0.f) scale = ldexpf(1.f, min(max(15 - e, -120), 120));
    }
    if (blockIdx.x == 0 && r == 0) *g.undo = 1.f / scale;
    const uint32_t bits = (uint32_t)__ballot(use);
    if (r == 0) g.kept[blockIdx.x] = bits;
    if (row >= g.rows) return;
    const float base = m * g.exponent, log2_s = log2f(s);
    g.lse[row] = base + log2_s;
    g.factor[row] = use ? weight * scale : 0.f;
    if (g.loss) {
        // of the largest logit's distance and not of the logits, so that large ones do not cancel
        const float t = g.temperature, part = g.entropy[row] + (m - pick) / t + log2_s * 0.693147181f;
        g.loss[row] = use ? weight * t * t * part : 0.f;
    }
}

// dz as 16-bit terms [term][row][ld], and its sums over the rows of a wave's part.
template <typename T, int TERMS>
struct Gradient {
    const float* bias;
    const int32_t* classes;
    const float* q;
    const float *lse, *factor;
    uint16_t* dz;
    int64_t ld, term;
    float* sums;  // [part][ld]
    float exponent;
    int rows, count, kept;
    __device__ static uint16_t narrow(float x) {
        if constexpr (__is_same(T, bf16)) return (uint16_t)bf16_pair(x, 0.f);
        else return __builtin_bit_cast(uint16_t, (f16)x);
    }
    __device__ static float widened(uint16_t x) { return to_float(__builtin_bit_cast(T, x)); }
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        const float* b = tile_bias<S>(bias, at.tile_m * S::TM, count, space) + at.wave_m * (16 * S::MI);
        const ListTile<S> lists{reinterpret_cast<float*>(space + 4 * S::TM + (at.wave_m + S::WM * at.wave_n) * ListTile<S>::bytes)};
        lists.clear();
        const int lane_q = lane_id() >> 4, r = lane_id() & 15;
        float total[S::MI / 4][16];
        for (int j = 0; j < S::MI / 4; ++j)
            for (int k = 0; k < 16; ++k) total[j][k] = 0.f;
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i;
            wave_meets();
            const bool any = lists.put(classes, q, kept, n, rows, at.m0, false);
            wave_meets();
            const bool there = n + r < rows;
            const float f = there ? factor[n + r] : 0.f, l = there ? lse[n + r] : 0.f;
            for (int j = 0; j < S::MI / 4; ++j) {
                const int m = at.m0 + 64 * j + 16 * lane_q;
                float v[16], y[16];
                sixteen(acc[i], j, v);
                add_bias(b + 64 * j + 16 * lane_q, v);
                if (any) {
                    lists.get(64 * j + 16 * lane_q, y);
                } else {
                    for (int k = 0; k < 16; ++k) y[k] = 0.f;
                }
                for (int k = 0; k < 16; ++k) {
                    const float p = __builtin_amdgcn_exp2f(v[k] * exponent - l);
                    v[k] = f != 0.f && m + k < count ? f * (p - y[k]) : 0.f;
                    total[j][k] += v[k];
                }
                if (there && m < ld)
                    for (int t = 0; t < TERMS; ++t) {
                        u32x4 out[2];
                        for (int k = 0; k < 16; k += 2) {
                            const uint16_t x = narrow(v[k]), y2 = narrow(v[k + 1]);
                            out[k / 8][k / 2 & 3] = x | (uint32_t)y2 << 16;
                            if (t + 1 < TERMS) v[k] -= widened(x), v[k + 1] -= widened(y2);
                        }
                        u32x4* to = reinterpret_cast<u32x4*>(dz + t * term + (n + r) * ld + m);
                        to[0] = out[0], to[1] = out[1];
                    }
            }
            wave_meets();
            if (any) lists.put(classes, q, kept, n, rows, at.m0, true);
        }
        for (int j = 0; j < S::MI / 4; ++j) {
            const int m = at.m0 + 64 * j + 16 * lane_q;
            for (int k = 0; k < 16; ++k)
                for (int d = 1; d < 16; d <<= 1) total[j][k] += __shfl_xor(total[j][k], d, kWave);
            if (r == 0 && m < ld) store_values<16>(sums + (at.tile_n * S::WN + at.wave_n) * ld + m, total[j]);
        }
    }
};

// ---- joins ------------------------------------------------------------------------------------------------------------

// dbias = alpha sum of the parts, or that added to it.
__global__ __launch_bounds__(kBlock) inline void k_teach_bias(const float* sums, int64_t ld, int parts, int classes, float alpha, const float* undo, float* dbias,
                                                              bool add) {
    __shared__ float s[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
    float v = 0.f;
    if (c < classes)
        for (int p = k; p < parts; p += 4) v += sums[p * ld + c];
    s[k][threadIdx.x & 63] = v;
    __syncthreads();
    if (k == 0 && c < classes) {
        for (int p = 1; p < 4; ++p) v += s[p][threadIdx.x];
        v *= alpha * *undo;
        dbias[c] = add ? dbias[c] + v : v;
    }
}

// out = factor times the sum of parts (rows x dim each, rows without padding), rounded; zeros for rows that are left out.
template <typename O>
__global__ __launch_bounds__(kBlock) void k_wide_join(const float* part, int splits, int64_t stride, int64_t rows, int dim, float alpha, const float* undo,
                                                      const uint32_t* kept, O* out, int64_t ld, bool add) {
    const float factor = undo ? alpha * *undo : alpha;
    const int64_t total = rows * dim;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / dim;
        float v = 0.f;
        for (int k = 0; k < splits; ++k) v += part[k * stride + at];
        v *= factor;
        if (kept && !(kept[row >> 5] >> (row & 31) & 1)) v = 0.f;
        O* to = out + row * ld + (at - row * dim);
        *to = (O)(add ? (float)*to + v : v);
    }
}

// Zeros in a matrix, for heads that learn from no rows.
template <typename O>
__global__ __launch_bounds__(kBlock) void k_teach_zeros(O* out, int64_t ld, int64_t rows, int dim) {
    const int64_t total = rows * dim;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock)
        out[at / dim * ld + at % dim] = (O)0.f;
}

}  // namespace dynlp
