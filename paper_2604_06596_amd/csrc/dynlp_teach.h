// Heads of any number of classes: logits, their softmax, and the divergence from a teacher of which a row keeps its first classes, with its gradients.
//
// A teacher's list of a row becomes q = softmax(u / T) over its entries.  With p = softmax(z / T) over all classes:
//   loss = r T^2 sum q (log q - log p),   dz = grad_scale r T (p - q),   dh = dz W,   dweight = dz^T h,   dbias = sum of dz over rows
// Logits do not go through memory: the product h W^T is made twice, for the sums of the softmax and again for dz, of which 16-bit terms are stored for the products
// with W and h (k_wide, classes as its fast index m, rows as n).  A head's own rounding needs one term (rounding dz once more, to 2^-9 of it on average, adds as much as the
// result's own rounding: 0.0023 of dh's norm where it alone is 0.0017; two are used in small calls, where few values decide); dweight in 32 bits takes as many as hold dz.
// What bounds it: the four products, 8 rows classes dim operations where 6 cannot be done without.  8,192 x 1,024 bfloat16, 50,021 classes: 3.76 ms: sums 905 us, dz 998
// (837 each without what follows the product), dh 764, dweight 935; in float16, whose dh has terms of its own, 4% more.
// Logits kept in 32 bits between the first two would move 10 bytes each at some 5 TB/s, which is a second product's time at dim = 1,000.
#pragma once

#include "dynlp_teacher.h"
#include "dynlp_wide.h"

namespace dynlp {

// Rows as 16-bit terms with zeros up to ld_out, a multiple of 32.  Bfloat16 terms of 32-bit values are each the nearest to what is left, and hold all 24 bits.  An infinite
// value is not a number there: as a term it would meet the other side's terms one by one, whose signs and zeros are not those of their sum.
__device__ inline void terms_of(float x, uint16_t (&term)[3]) {
    if (fabsf(x) == INFINITY) x = NAN;
    bool cut = false;
    for (int k = 0; k < 3; ++k) {
        uint16_t b = (uint16_t)bf16_pair(x, 0.f);
        float v = __uint_as_float((uint32_t)b << 16);
        if (cut || fabsf(v) == INFINITY) {  // a value that rounding makes infinite is cut off instead, and so is what is left of it: no sum of some terms is beyond x
            cut = true;
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
                terms_of(col + k < dim ? in[row * ld + col + k] : 0.f, a);
                terms_of(col + k + 1 < dim ? in[row * ld + col + k + 1] : 0.f, b);
                for (int t = 0; t < 3; ++t) v[t][k / 2] = a[t] | (uint32_t)b[t] << 16;
            }
            for (int t = 0; t < 3; ++t) *reinterpret_cast<u32x4*>(out + t * term + row * ld_out + col) = v[t];
        }
    }
}

// ---- logits -----------------------------------------------------------------------------------------------------------

// The tile's bias in shared memory: -infinity, which makes a logit so whatever h holds, for what is not a class.  Returns whether there is any such.
template <typename S>
__device__ inline bool tile_bias(const float* bias, int first, int classes, char* space) {
    float* b = reinterpret_cast<float*>(space);
    bool shut = false;
    for (int k = threadIdx.x; k < S::TM; k += kBlock) {
        b[k] = first + k >= classes ? -INFINITY : bias ? bias[first + k] : 0.f;
        shut |= b[k] == -INFINITY;
    }
    return __syncthreads_or(shut);
}
// Adds it to consecutive logits.
template <int N>
__device__ inline void add_bias(const float* b, bool shut, float (&v)[N]) {
    for (int k = 0; k < N; k += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(b + k);
        for (int i = 0; i < 4; ++i) v[k + i] += x[i];
        if (shut)
            for (int i = 0; i < 4; ++i) v[k + i] = x[i] == -INFINITY ? x[i] : v[k + i];
    }
}

// ---- the teacher's lists ----------------------------------------------------------------------------------------------

// Entries of 16 rows, ordered by the tile of classes that they lie in: their row and class there, and q.  A class that a row names several times is one entry.
constexpr int kListRows = 16;
struct Lists {
    uint2* entry;       // [16 rows][16 kept]: row << 8 | class, bits of q
    uint32_t* start;    // [16 rows][tiles + 1]
    float* entropy;     // sum of q log q over the classes of a row
    float* weight;      // of a row; 0: left out
    uint32_t* largest;  // bits of the largest finite |weight|, or NULL
    int kept, tiles, log2;  // tiles of 1 << log2 classes, 256 at most
};

// zeros: 512 bytes of them.
__global__ __launch_bounds__(kBlock) inline void k_teach_begin(uint32_t* zeros, uint32_t* largest) {
    if (threadIdx.x < 128) zeros[threadIdx.x] = 0;
    if (threadIdx.x == 0) *largest = 0;
}

__device__ inline float over_16(float v, bool sum) {
    for (int d = 1; d < 16; d <<= 1) {
        const float o = __shfl_xor(v, d, kWave);
        v = sum ? v + o : fmaxf(v, o);
    }
    return v;
}

// 16 rows to a workgroup, 16 lanes and E entries in each lane for a row.  8,192 rows of 32: 8 us.  Ordered, an epilogue reads the few entries of its own 16 rows and classes
// (8,192 x 50,021: sums 1,202 us and dz 1,277 with a search through all of a row's, 949 and 1,035 so when that was done).
template <int E>
__global__ __launch_bounds__(kBlock) void k_teach_lists(Teacher t, Lists out, int64_t row0, int64_t rows) {
    extern __shared__ char space[];
    uint32_t* count = reinterpret_cast<uint32_t*>(space);  // of each tile, then its next place
    __shared__ uint32_t sums[kBlock / kWave], most;
    if (threadIdx.x == 0) most = 0;
    const int me = threadIdx.x & 15, in = threadIdx.x >> 4;
    const int64_t row = (int64_t)blockIdx.x * kListRows + in;
    const bool there = row < rows;
    const int64_t at = there ? row0 + row : row0;
    for (int k = threadIdx.x; k < out.tiles; k += kBlock) count[k] = 0;
    int c[E];
    float u[E], q[E];
    float top = -INFINITY;
    for (int e = 0; e < E; ++e) {
        const int k = e * 16 + me;
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
    top = over_16(top, false);
    float sum = 0.f;
    for (int e = 0; e < E; ++e) {
        q[e] = u[e] == -INFINITY ? 0.f : expf((u[e] - top) * t.inverse);
        sum += q[e];
    }
    sum = over_16(sum, true);
    const float log_sum = logf(sum);
    for (int e = 0; e < E; ++e)
        if (sum != 0.f) q[e] /= sum;
    // a class that is named several times: the first gets all of it
    float all[E];
    bool first[E];
    for (int e = 0; e < E; ++e) all[e] = 0.f, first[e] = true;
    for (int from = 0; from < E; ++from)
        for (int k = 0; k < 16 && from * 16 + k < t.kept; ++k) {
            const int other = __shfl(c[from], k, 16);
            const float more = __shfl(q[from], k, 16);
            for (int e = 0; e < E; ++e)
                if (other == c[e]) {
                    if (from * 16 + k < e * 16 + me) first[e] = false;
                    all[e] += more;
                }
        }
    // of probabilities of classes, not of entries; an entry that has its class to itself has the logarithm of q from its logit
    float entropy = 0.f;
    for (int e = 0; e < E; ++e)
        if (c[e] >= 0 && first[e] && all[e] != 0.f) entropy += all[e] * (all[e] == q[e] ? (u[e] - top) * t.inverse - log_sum : logf(all[e]));
    entropy = over_16(entropy, true);
    __syncthreads();
    for (int e = 0; e < E; ++e)
        if (c[e] >= 0 && first[e]) atomicAdd(count + (c[e] >> out.log2), 1u);
    __syncthreads();
    // where each tile's entries begin
    const int per = (out.tiles + kBlock - 1) / kBlock;
    uint32_t mine = 0;
    for (int k = threadIdx.x * per; k < min((int)(threadIdx.x + 1) * per, out.tiles); ++k) mine += count[k];
    uint32_t before = mine;  // of the wave's threads up to this one, then of all before it
    for (int d = 1; d < kWave; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)before, d, kWave);
        if ((int)lane_id() >= d) before += o;
    }
    if (lane_id() == kWave - 1) sums[threadIdx.x / kWave] = before;
    __syncthreads();
    before -= mine;
    for (int w = 0; w < (int)threadIdx.x / kWave; ++w) before += sums[w];
    uint32_t* start = out.start + (int64_t)blockIdx.x * (out.tiles + 1);
    for (int k = threadIdx.x * per; k < min((int)(threadIdx.x + 1) * per, out.tiles); ++k) {
        const uint32_t n = count[k];
        start[k] = count[k] = before;
        before += n;
        if (k + 1 == out.tiles) start[k + 1] = before;
    }
    __syncthreads();
    uint2* entry = out.entry + (int64_t)blockIdx.x * (kListRows * t.kept);
    for (int e = 0; e < E; ++e)
        if (c[e] >= 0 && first[e])  // in whatever order: no two are for the same row and class
            entry[atomicAdd(count + (c[e] >> out.log2), 1u)] = make_uint2((uint32_t)in << 8 | (uint32_t)(c[e] & ((1 << out.log2) - 1)), __float_as_uint(all[e]));
    if (there && me == 0) {
        const float r = t.row_weight ? t.row_weight[at] : 1.f;
        const float weight = sum == 0.f ? 0.f : r;
        out.weight[row] = weight;
        out.entropy[row] = entropy;
        if (out.largest && fabsf(weight) < INFINITY) atomicMax(&most, __float_as_uint(fabsf(weight)));
    }
    if (!out.largest) return;
    __syncthreads();
    // one address takes some 10^8 of these a second: those that change nothing do not go there
    if (threadIdx.x == 0 && most > __hip_atomic_load(out.largest, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(out.largest, most);
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
    // Puts there, or takes away, a lane's entry where it is one of the wave's classes.  Returns whether any lane's is.
    __device__ bool put(uint2 entry, bool there, int wave_m, bool away) const {
        const int c = (int)(entry.x & 255) - wave_m * (16 * S::MI);
        const bool hit = there && c >= 0 && c < 16 * S::MI;
        if (hit) p[(entry.x >> 8) * ld + c] = away ? 0.f : __uint_as_float(entry.y);
        return __any(hit);
    }
    __device__ void get(int column, float (&v)[16]) const {
        for (int k = 0; k < 16; k += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p + (lane_id() & 15) * ld + column + k);
            for (int i = 0; i < 4; ++i) v[k + i] = x[i];
        }
    }
};
// The entries of a wave's rows: the first 64 of each 16 rows are asked for at once.
template <typename S>
struct WaveLists {
    ListTile<S> tile;
    const uint2* entry[S::NI];
    int count[S::NI];
    uint2 ahead[S::NI];
    int wave_m;
    __device__ WaveLists(const Lists& l, const Place& at, int rows, char* space) : wave_m(at.wave_m) {
        tile.p = reinterpret_cast<float*>(space + 4 * S::TM + (at.wave_m + S::WM * at.wave_n) * ListTile<S>::bytes);
        tile.clear();
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i;
            count[i] = 0;
            entry[i] = l.entry;
            if (n < rows) {
                const int64_t block = n / kListRows;
                const uint32_t* start = l.start + block * (l.tiles + 1) + at.tile_m;
                entry[i] = l.entry + block * (kListRows * l.kept) + start[0];
                count[i] = (int)(start[1] - start[0]);
            }
            ahead[i] = (int)lane_id() < count[i] ? entry[i][lane_id()] : make_uint2(0, 0);
        }
    }
    __device__ bool put(int i, bool away) const {
        bool any = tile.put(ahead[i], (int)lane_id() < count[i], wave_m, away);
        for (int k = kWave; k < count[i]; k += kWave) {
            const bool there = k + (int)lane_id() < count[i];
            any |= tile.put(there ? entry[i][k + lane_id()] : make_uint2(0, 0), there, wave_m, away);
        }
        wave_meets();
        return any;
    }
};

// The least that logits are taken relative to: what has none but -infinity stays at 0.
__device__ inline float base_of(float m) { return fmaxf(m, -3e38f); }

// Sums of the softmax: for every 16 MI classes and every row the largest logit m, sum of exp((z - m) / T), sum of q (z - m), sum of q.  All that is rounded is differences
// of logits, so that what they share, however large, takes no digits from p.
struct Stats {
    const float* bias;
    Lists lists;
    float *top, *sum, *picked, *share;  // [part][ld]
    int64_t ld;
    float exponent;             // log2(e) / T
    int rows, classes;
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        const bool shut = tile_bias<S>(bias, at.tile_m * S::TM, classes, space);
        const float* b = reinterpret_cast<float*>(space) + at.wave_m * (16 * S::MI);
        const WaveLists<S> wave(lists, at, rows, space);
        const int lane_q = lane_id() >> 4, r = lane_id() & 15;
        wave_meets();
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            const bool any = wave.put(i, false);
            float m = -INFINITY, z[S::MI / 4][16];
            for (int j = 0; j < S::MI / 4; ++j) {
                sixteen(acc[i], j, z[j]);
                add_bias(b + 64 * j + 16 * lane_q, shut, z[j]);
                for (int k = 0; k < 16; ++k) m = fmaxf(m, z[j][k]);
            }
            m = row_max(m);
            const float base = base_of(m);
            float s = 0.f, pick = 0.f, all = 0.f;
            for (int j = 0; j < S::MI / 4; ++j)
                for (int k = 0; k < 16; ++k) {
                    z[j][k] -= base;
                    s += __builtin_amdgcn_exp2f(z[j][k] * exponent);
                }
            s = row_sum(s);
            if (any) {
                for (int j = 0; j < S::MI / 4; ++j) {
                    float q[16];
                    wave.tile.get(64 * j + 16 * lane_q, q);
                    for (int k = 0; k < 16; ++k) {
                        pick += q[k] != 0.f ? q[k] * z[j][k] : 0.f;
                        all += q[k];
                    }
                }
                wave.put(i, true);
                pick = row_sum(pick);
                all = row_sum(all);
            }
            if (lane_q == 0 && n < rows) {
                const int64_t to = (int64_t)(at.tile_m * S::WM + at.wave_m) * ld + n;
                top[to] = m, sum[to] = s, picked[to] = pick, share[to] = all;
            }
        }
    }
};

struct RowJoin {
    const float *top, *sum, *picked, *share;  // [part][ld]
    int64_t ld;
    const float *entropy, *weight;    // of the lists
    const uint32_t* largest;          // of 16-bit floats with 5 bits of exponent, or NULL
    float* loss;                      // or NULL
    float *base, *inverse;            // the largest logit m, and one over the sum of exp((z - m) / T)
    float* factor;                    // weight times a power of two; 0 where the row is left out
    uint32_t* kept;                   // a bit per row
    float *undo_row, *ratio;          // where there is `largest`: one over the row's power, and the largest weight's power over it
    float* undo;                      // one over the largest weight's power
    float temperature, exponent;
    int rows, parts;
};
// What brings a weight to 2^14 .. 2^15, so that float16 holds the terms of its row's dz.
__device__ inline float power_to_15(float weight) {
    int e;
    frexpf(weight, &e);
    return ldexpf(1.f, min(max(15 - e, -120), 120));
}
// The parts of 32 rows, by K threads each, in order.
template <int K>
__global__ __launch_bounds__(32 * K) void k_teach_rows(RowJoin g) {
    __shared__ float tops[K][33], sums[K][33], picks[K][33], shares[K][33];
    const int r = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int row = blockIdx.x * 32 + r, at = min(row, g.rows - 1);
    float m = -INFINITY, s = 0.f, pick = 0.f, share = 0.f;
    auto take = [&](float pm, float ps, float pp, float pq) {
        const float all = fmaxf(m, pm), base = base_of(all);
        s = (m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - all) * g.exponent)) + (pm == -INFINITY ? ps : ps * __builtin_amdgcn_exp2f((pm - all) * g.exponent));
        if (share != 0.f) pick += share * (base_of(m) - base);
        if (pq != 0.f) pick += pp + pq * (base_of(pm) - base);
        share += pq;
        m = all;
    };
#pragma unroll 4
    for (int p = k; p < g.parts; p += K) take(g.top[p * g.ld + at], g.sum[p * g.ld + at], g.picked[p * g.ld + at], g.share[p * g.ld + at]);
    tops[k][r] = m, sums[k][r] = s, picks[k][r] = pick, shares[k][r] = share;
    __syncthreads();
    if (k != 0) return;
    for (int p = 1; p < K; ++p) take(tops[p][r], sums[p][r], picks[p][r], shares[p][r]);
    const float weight = g.weight[at];
    const bool use = row < g.rows && weight != 0.f && s != 0.f;
    float scale = 1.f, own = 1.f;
    if (g.largest) {
        const float most = __uint_as_float(*g.largest);
        if (most > 0.f) scale = power_to_15(most);
        own = weight != 0.f && fabsf(weight) < INFINITY ? power_to_15(fabsf(weight)) : scale;
    }
    if (blockIdx.x == 0 && r == 0) *g.undo = 1.f / scale;
    const uint32_t bits = (uint32_t)__ballot(use);
    if (r == 0) g.kept[blockIdx.x] = bits;
    if (row >= g.rows) return;
    g.base[row] = m;
    g.inverse[row] = 1.f / s;
    // a list that holds what is no number says nothing of any class
    g.factor[row] = !use ? 0.f : g.entropy[row] == g.entropy[row] ? weight * own : NAN;
    if (g.largest) g.undo_row[row] = 1.f / own, g.ratio[row] = scale / own;
    if (g.loss) {
        const float t = g.temperature, part = g.entropy[row] + (logf(s) - pick / t);
        g.loss[row] = use ? weight * (t * (t * part)) : 0.f;  // T^2 by itself may lie below what 32 bits hold
    }
}

// Two values rounded to T, the first in the low half, and what of them is left.
__device__ inline uint32_t pair_of(float x, float y, bf16) { return bf16_pair(x, y); }
__device__ inline uint32_t pair_of(float x, float y, f16) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef f16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
}
template <typename T>
__device__ inline float half_of(uint32_t pair, int k) {
    return to_float(__builtin_bit_cast(T, (uint16_t)(pair >> (16 * k))));
}

// dz as 16-bit terms [term][row][ld], and its sums over the rows of a wave's part.  Float16 has OWN terms beside them, for what is made row by row: times the row's power of
// two and not the largest weight's, so that a row of little weight keeps as many digits as any.
template <typename T, int TERMS, int OWN>
struct Gradient {
    const float* bias;
    Lists lists;
    const float *base, *inverse, *factor, *ratio;
    uint16_t *own, *dz;  // each may be NULL
    int64_t ld, term;
    float* sums;  // [part][ld]
    float exponent;
    int rows, classes;
    // 16 values of a row, as N terms.
    template <int N>
    __device__ void put(uint16_t* to, float (&v)[16]) const {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            u32x4 out[2];
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
                const uint32_t pair = pair_of(v[k], v[k + 1], T());
                out[k / 8][k / 2 & 3] = pair;
                if (t + 1 < N) v[k] -= half_of<T>(pair, 0), v[k + 1] -= half_of<T>(pair, 1);
            }
            u32x4* p = reinterpret_cast<u32x4*>(to + t * term);
            p[0] = out[0], p[1] = out[1];
        }
    }
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        const bool shut = tile_bias<S>(bias, at.tile_m * S::TM, classes, space);
        const float* b = reinterpret_cast<float*>(space) + at.wave_m * (16 * S::MI);
        const WaveLists<S> wave(lists, at, rows, space);
        const int lane_q = lane_id() >> 4, r = lane_id() & 15;
        float total[S::MI / 4][16], f[S::NI], fp[S::NI], top[S::NI], to_all[S::NI];  // f: of q; fp: of exp((z - top) / T)
        for (int j = 0; j < S::MI / 4; ++j)
            for (int k = 0; k < 16; ++k) total[j][k] = 0.f;
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            f[i] = n < rows ? factor[n] : 0.f, fp[i] = n < rows ? inverse[n] * factor[n] : 0.f, top[i] = n < rows ? base[n] : 0.f;
            if constexpr (OWN > 0) to_all[i] = n < rows ? ratio[n] : 0.f;
        }
        wave_meets();
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            const bool any = wave.put(i, false);
#pragma unroll
            for (int j = 0; j < S::MI / 4; ++j) {
                const int m = at.m0 + 64 * j + 16 * lane_q;
                float v[16];
                sixteen(acc[i], j, v);
                add_bias(b + 64 * j + 16 * lane_q, shut, v);
                for (int k = 0; k < 16; ++k) v[k] = __builtin_amdgcn_exp2f((v[k] - top[i]) * exponent) * fp[i];
                if (any) {
                    float q[16];
                    wave.tile.get(64 * j + 16 * lane_q, q);
                    for (int k = 0; k < 16; ++k) v[k] = __builtin_fmaf(-q[k], f[i], v[k]);
                }
                // a row that is left out has zeros whatever its logits, and so have the columns behind the classes
                for (int k = 0; k < 16; ++k) v[k] = f[i] != 0.f ? v[k] : 0.f;
                if (shut)
                    for (int k = 0; k < 16; ++k) v[k] = m + k < classes ? v[k] : 0.f;
                const bool there = n < rows && m < ld;
                if constexpr (OWN > 0) {
                    float x[16];
                    for (int k = 0; k < 16; ++k) x[k] = v[k], v[k] *= to_all[i];
                    if (there && own) put<OWN>(own + n * ld + m, x);
                }
                for (int k = 0; k < 16; ++k) total[j][k] += v[k];
                if (there && dz) put<TERMS>(dz + n * ld + m, v);
            }
            if (any) wave.put(i, true);
        }
        for (int j = 0; j < S::MI / 4; ++j) {
            const int m = at.m0 + 64 * j + 16 * lane_q;
            for (int k = 0; k < 16; ++k) {
                uint32_t v = __float_as_uint(total[j][k]);
                auto add = [](uint32_t x, int y) { return __float_as_uint(__uint_as_float(x) + __uint_as_float((uint32_t)y)); };
                v = add(v, __builtin_amdgcn_update_dpp((int)v, (int)v, 0x121, 0xf, 0xf, false));  // of 16 lanes, rotated by 1, 2, 4, 8
                v = add(v, __builtin_amdgcn_update_dpp((int)v, (int)v, 0x122, 0xf, 0xf, false));
                v = add(v, __builtin_amdgcn_update_dpp((int)v, (int)v, 0x124, 0xf, 0xf, false));
                v = add(v, __builtin_amdgcn_update_dpp((int)v, (int)v, 0x128, 0xf, 0xf, false));
                total[j][k] = __uint_as_float(v);
            }
            if (r == 0 && m < ld) store_values<16>(sums + (at.tile_n * S::WN + at.wave_n) * ld + m, total[j]);
        }
    }
};

// ---- joins ------------------------------------------------------------------------------------------------------------

// dbias = alpha sum of the parts, or that added to it; `each` of them at a time, to one row of dbias (ld elements) for each.
constexpr int kBiasParts = 64;
__global__ __launch_bounds__(kBlock) inline void k_teach_bias(const float* sums, int64_t ld, int parts, int each, int classes, float alpha, const float* undo, float* dbias,
                                                              bool add) {
    __shared__ float s[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6, first = blockIdx.y * each, end = min(first + each, parts);
    float v = 0.f;
    if (c < classes)
#pragma unroll 4
        for (int p = first + k; p < end; p += 4) v += sums[p * ld + c];
    s[k][threadIdx.x & 63] = v;
    __syncthreads();
    if (k == 0 && c < classes) {
        for (int p = 1; p < 4; ++p) v += s[p][threadIdx.x];
        v *= undo ? alpha * *undo : alpha;
        float* to = dbias + blockIdx.y * ld + c;
        *to = add ? *to + v : v;
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
