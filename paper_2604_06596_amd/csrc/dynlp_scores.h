// What rows of logits, or of probabilities, say: log probabilities of given classes, entropy, the first classes.
//
// With m the row's largest logit, s = sum exp(x - m) and t = sum exp(x - m) (x - m):   log p = x - m - log s,   entropy = log s - t / s.
// Of rows of probabilities, which need not sum to one: s = sum x, t = sum x log x:     log p = log x - log s,   entropy = log s - t / s.
// Classes are ordered by a key of 64 bits: the value's order above the class's, so that keys differ and of equal values the lowest class is the first.
// What bounds it: 4,099 x 100,003 bfloat16, the first 32: 185 us (4.4 TB/s, a copy 4.7), one pass over the rows with a threshold that some k values pass (k searches through
// a row: 16,969).  1M x 50 float32 probabilities, the first 4: 75 us (3.1 TB/s), half of it arithmetic: the logarithms and 20 operations a value for the order.
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

__device__ inline float value_of(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float((int)o < 0 ? o & 0x7fffffffu : ~o);
}

// f over 16 lanes, by moves between them; the result is in every lane.
template <typename F>
__device__ inline uint32_t over_16_lanes(uint32_t v, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, true));  // rotated by 1, 2, 4, 8
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, true));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, true));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true));
    return v;
}
// f over the 64 lanes.
template <typename F>
__device__ inline uint32_t over_wave(uint32_t v, F f) {
    v = over_16_lanes(v, f);
    const uint32_t a = f((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    const uint32_t b = f((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48));
    return f(a, b);
}
struct MaxFloat {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
};
struct AddFloat {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
};
struct Larger {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct Smaller {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a < b ? a : b; }
};
__device__ inline float lanes_max(float v) { return __uint_as_float(over_wave(__float_as_uint(v), MaxFloat())); }
__device__ inline float lanes_sum(float v) { return __uint_as_float(over_wave(__float_as_uint(v), AddFloat())); }
__device__ inline uint32_t lanes_max(uint32_t v) { return over_wave(v, Larger()); }
__device__ inline uint32_t lanes_min(uint32_t v) { return over_wave(v, Smaller()); }
__device__ inline int lanes_before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// ---- sums -------------------------------------------------------------------------------------------------------------

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// m: the largest x; with y = (x - m) log2(e), s = sum 2^y, t = sum 2^y y.  PROB: s = sum x, t = sum x log2(x), and m is not used.  (One operation less, x log2(e) - m', leaves
// the rounding of m' = m log2(e) in every y, which is more than 32 bits hold where m is large, as masks are.)
struct RowSums {
    float m, s, t;
    __device__ static RowSums none() { return {-INFINITY, 0.f, 0.f}; }
    // Values v, of which those that are not there are -infinity, and their largest.  What is -infinity adds nothing, what is not a number makes s so.
    template <bool PROB, int N>
    __device__ void add(const float (&v)[N], float top) {
        if constexpr (PROB) {
            for (int k = 0; k < N; ++k) add_probability(v[k]);
        } else {
            rescale(fmaxf(m, top));
            const float from = base();
            for (int k = 0; k < N; ++k) add_power((v[k] - from) * kLog2e);
        }
    }
    // The instruction's logarithm takes a denormal for 0: those, and 0, have that of 2^-126, which is near enough beside a sum of 2^-60 (power_of() sees to others).
    __device__ void add_probability(float v) {
        const float x = v == -INFINITY ? 0.f : v;
        s += x;
        t = __builtin_fmaf(x, __builtin_amdgcn_logf(fmaxf(x, 1.17549435e-38f)), t);
    }
    // A power of two for rows of probabilities whose sum is so small, or so large, that s or t does not hold it: they are summed once more, times that.  1 for all others.
    __device__ float power_of() const { return s > 0.f && s < 0x1p-60f ? 0x1p90f : s > 0x1p100f ? 0x1p-60f : 1.f; }
    // A row of nothing but -infinity stays at 0.
    __device__ float base() const { return m == -INFINITY ? 0.f : m; }
    __device__ void add_power(float y) {
        const float e = __builtin_amdgcn_exp2f(y);
        s += e;
        t = __builtin_fmaf(e, fmaxf(y, -1e30f), t);
    }
    __device__ void rescale(float top) {
        const float y = (m - top) * kLog2e;
        if (m == -INFINITY) {
            // nothing yet, or not a number
        } else if (y != 0.f) {
            const float f = __builtin_amdgcn_exp2f(y);
            t = f * (t + s * fmaxf(y, -1e30f));
            s *= f;
        }
        m = top;
    }
    template <bool PROB>
    __device__ void over_lanes() {
        if constexpr (!PROB) rescale(lanes_max(m));
        s = lanes_sum(s);
        t = lanes_sum(t);
    }
    template <bool PROB>
    __device__ void join(RowSums o) {
        if constexpr (!PROB) {
            const float top = fmaxf(m, o.m);
            rescale(top);
            o.rescale(top);
        }
        s += o.s;
        t += o.t;
    }
};
template <int N>
__device__ inline float largest_of(const float (&v)[N]) {
    float top = v[0];
    for (int k = 1; k < N; ++k) top = fmaxf(top, v[k]);
    return top;
}
// What the sums of a whole row (of probabilities: times `power`) say.  A row of nothing but -infinity (zeros) has 1/C everywhere.
template <bool PROB>
struct RowLog {
    float m, log_s, entropy, uniform;
    bool none;
    __device__ RowLog(const RowSums& a, int dim, float power = 1.f) {
        m = a.m;
        none = a.s == 0.f;
        log_s = logf(a.s);
        uniform = none ? logf((float)dim) : 0.f;
        entropy = none ? uniform : log_s - a.t / a.s * kLn2;
        if constexpr (PROB) {
            if (power != 1.f) log_s = a.s == INFINITY ? NAN : log_s - (power > 1.f ? 90.f : -60.f) * kLn2;
        }
    }
    __device__ float of(float x) const { return none ? -uniform : PROB ? logf(x) - log_s : (x - m) - log_s; }
};

// ---- the first classes ------------------------------------------------------------------------------------------------

// A number such that at least k of the wave's `order(j)`, j < n, are not below it, and seldom many more: the interval between the least and the largest is halved up to
// `most` times.  Orders that are not there are 0; there are k others.  U of them are looked at at a time (n is a multiple of U, or order(j) is 0 beyond it).
template <int U, typename O>
__device__ inline uint32_t threshold(int n, int k, int most, O order) {
    const uint32_t least = order_of(-INFINITY);
    uint32_t high = 0, low = ~0u;
    int count = 0;
    for (int j = 0; j < n; j += U) {
        uint32_t o[U];
        for (int u = 0; u < U; ++u) o[u] = order(j + u);
        for (int u = 0; u < U; ++u) {
            high = max(high, o[u]);
            low = min(low, o[u] > least ? o[u] : ~0u);
            count += __popcll(__ballot(o[u] > least));
        }
    }
    if (count < k) return least;
    high = lanes_max(high);
    low = lanes_min(low);
    for (int step = 0; step < most && low < high; ++step) {
        const uint32_t middle = low + ((high - low) >> 1) + 1;
        count = 0;
        for (int j = 0; j < n; j += U) {
            uint32_t o[U];
            for (int u = 0; u < U; ++u) o[u] = order(j + u);
            for (int u = 0; u < U; ++u) count += __popcll(__ballot(o[u] >= middle));
        }
        if (count >= k) low = middle;
        else high = middle - 1;
        if (count == k) break;
    }
    return low;
}

// A wave's candidates in shared memory, in no order; those that cannot be among the first k are no longer there.
struct Candidates {
    uint64_t* key;
    int count;       // the same for all lanes
    uint32_t above;  // what is not above it in order is none
    float over;      // the same as a value, for a first look: what is not above it is none.  Not a number where all have to be looked at
    __device__ void none(uint64_t* space) {
        key = space;
        count = 0;
        above = 0;
        over = NAN;
    }
    __device__ void raise(uint32_t order) {
        above = order;
        const float v = value_of((uint64_t)order << 32);
        over = order <= order_of(-INFINITY) ? NAN : v == 0.f ? -1e-37f : v;  // -0 comes before 0
    }
    __device__ void put(float x, int column, bool there) {
        if (!__any(!(x <= over))) return;
        const uint32_t o = order_of(x);
        const bool hit = there && o > above;
        const uint64_t mask = __ballot(hit);
        if (hit) key[count + lanes_before(mask)] = (uint64_t)o << 32 | (uint32_t)~column;
        count += __popcll(mask);
    }
    // Leaves those whose key is not below `least`.
    __device__ void keep(uint64_t least) {
        int to = 0;
        for (int at = 0; at < count; at += kWave) {
            const int i = at + lane_id();
            const uint64_t k = i < count ? key[i] : 0;
            const bool stays = i < count && k >= least;
            const uint64_t mask = __ballot(stays);
            if (stays) key[to + lanes_before(mask)] = k;
            to += __popcll(mask);
        }
        count = to;
    }
    // Leaves k at least and `most` at most; k <= most.
    __device__ void cut(int k, int most) {
        if (count <= k) return;
        const int n = (count + kWave - 1) / kWave;
        uint32_t least = threshold<2>(n, k, 14, [&](int j) { return (int)(j * kWave + lane_id()) < count ? (uint32_t)(key[j * kWave + lane_id()] >> 32) : 0u; });
        keep((uint64_t)least << 32);
        if (count > most) {  // equal or nearly equal values: exactly k, bit by bit
            const int left = (count + kWave - 1) / kWave;
            uint64_t exact = 0;
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t next = exact | uint64_t(1) << bit;
                int above_it = 0;
                for (int j = 0; j < left; ++j) {
                    const int i = j * kWave + lane_id();
                    above_it += __popcll(__ballot(i < count && key[i] >= next));
                }
                if (above_it >= k) exact = next;
            }
            keep(exact);
            raise((uint32_t)(exact >> 32));  // those that come have higher columns
        } else {
            raise(max(least, 1u) - 1u);
        }
    }
};

constexpr int kCandidates = 384;  // that a wave has at most when its part is done
// Candidates beyond which the list is cut: a cut costs as much as some twenty candidates, and each lets fewer through (100,003 values, the first 32: cut
// at 160 candidates 266 us for 4,099 rows).
__device__ inline int most_of(int top) { return top + max(top, 32); }

// One wave's part of a row: turns of P pieces per lane, `waves` of them taking turns.
template <typename T, bool PROB, int P>
struct RowScan {
    static constexpr int E = Piece<T>::n, N = P * E, turn = N * kWave;
    __device__ static void load(const T* row, int from, int dim, float (&v)[N]) {
        u32x4 piece[P];
        if (from + turn <= dim) {
            for (int p = 0; p < P; ++p) piece[p] = load_piece(row + from + (p * kWave + lane_id()) * E);
        } else {
            for (int p = 0; p < P; ++p) {
                const int col = from + (p * kWave + lane_id()) * E;
                piece[p] = col < dim ? load_columns(row, col, dim) : u32x4{0u, 0u, 0u, 0u};
            }
        }
        for (int p = 0; p < P; ++p) {
            float f[E];
            widen(piece[p], f, T());
            for (int e = 0; e < E; ++e) v[p * E + e] = f[e];
        }
        if (from + turn > dim)
            for (int p = 0; p < P; ++p)
                for (int e = 0; e < E; ++e)
                    if (from + (p * kWave + (int)lane_id()) * E + e >= dim) v[p * E + e] = -INFINITY;
    }
    // The sums alone, of values times a power of two.
    __device__ static RowSums again(const T* row, int dim, int wave, int waves, float power) {
        RowSums sums = RowSums::none();
#pragma unroll 1
        for (int from = wave * turn; from < dim; from += waves * turn) {
            float v[N];
            load(row, from, dim, v);
            for (int k = 0; k < N; ++k) sums.add_probability(v[k] * power);
        }
        sums.over_lanes<true>();
        return sums;
    }
    __device__ static void run(const T* row, int dim, int wave, int waves, int top, RowSums& sums, Candidates& c) {
#pragma unroll 1
        for (int from = wave * turn; from < dim; from += waves * turn) {
            float v[N];
            load(row, from, dim, v);
            float tops[P];
            for (int p = 0; p < P; ++p) {
                tops[p] = v[p * E];
                for (int e = 1; e < E; ++e) tops[p] = fmaxf(tops[p], v[p * E + e]);
            }
            const float best = largest_of(tops);
            sums.add<PROB>(v, best);
            if (top == 0) continue;
            if (from == wave * turn) {
                // of 128 groups of values the k-th largest maximum: k values are not below it
                float half = v[0];
                for (int k = 1; k < (N + 1) / 2; ++k) half = fmaxf(half, v[k]);
                float other = v[N / 2];
                for (int k = N / 2 + 1; k < N; ++k) other = fmaxf(other, v[k]);
                const uint32_t order[2] = {order_of(half), order_of(other)};
                c.raise(max(threshold<2>(2, top, 14, [&](int j) { return order[j]; }), 1u) - 1u);
            }
            if (!__any(!(best <= c.over))) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (!__any(!(tops[p] <= c.over))) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int col = from + (p * kWave + (int)lane_id()) * E + e;
                    c.put(v[p * E + e], col, col < dim);
                }
                if (c.count > most_of(top)) c.cut(top, most_of(top));
            }
        }
    }
};

// The first classes of a wave's candidates to the outputs: the place of a candidate is how many come before it.
template <bool PROB>
__device__ inline void write_top(Candidates& c, const Scores& o, int64_t row, const RowLog<PROB>& log) {
    c.cut(o.top, kCandidates);
    for (int at = 0; at < c.count; at += kWave) {
        const int i = at + lane_id();
        const uint64_t key = i < c.count ? c.key[i] : 0;
        int place = 0;
        for (int j = 0; j < c.count; ++j) place += c.key[j] > key;
        if (i < c.count && place < o.top) {
            if (o.top_classes) o.top_classes[row * o.top + place] = column_of_key(key);
            if (o.log_top) o.log_top[row * o.top + place] = log.of(value_of(key));
        }
    }
}

constexpr int row_lists(int waves) { return waves == 1 ? kBlock / kWave : waves; }
template <typename T>
constexpr int row_space(int waves) {
    return row_lists(waves) * ((kCandidates + kWave * Piece<T>::n) * 8 + (int)sizeof(RowSums) + 4);
}
// WAVES waves for each row; four rows to a workgroup where it is one.
template <typename T, bool PROB, int P, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kBlock : WAVES * kWave) void k_row_scores(const T* x, int64_t ld, int64_t rows, int dim, Scores o) {
    using Scan = RowScan<T, PROB, P>;
    constexpr int kLists = row_lists(WAVES), kSpace = kCandidates + kWave * Scan::E;
    extern __shared__ char space[];
    uint64_t* keys = reinterpret_cast<uint64_t*>(space);
    RowSums* parts = reinterpret_cast<RowSums*>(keys + kLists * kSpace);
    int* counts = reinterpret_cast<int*>(parts + kLists);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t first = WAVES == 1 ? (int64_t)blockIdx.x * kLists + wave : blockIdx.x, step = WAVES == 1 ? (int64_t)gridDim.x * kLists : gridDim.x;
    for (int64_t row = first; row < rows; row += step) {
        const T* p = x + row * ld;
        RowSums sums = RowSums::none();
        Candidates c;
        c.none(keys + wave * kSpace);
        Scan::run(p, dim, WAVES == 1 ? 0 : wave, WAVES, o.top, sums, c);
        sums.over_lanes<PROB>();
        if constexpr (WAVES > 1) {
            if (o.top) c.cut(o.top, kCandidates);
            if (lane_id() == 0) parts[wave] = sums, counts[wave] = c.count;
            uint64_t mine[kCandidates / kWave];
            for (int j = 0; j < kCandidates / kWave; ++j) mine[j] = j * kWave + (int)lane_id() < c.count ? c.key[j * kWave + lane_id()] : 0;
            __syncthreads();
            sums = parts[0];
            for (int w = 1; w < WAVES; ++w) sums.join<PROB>(parts[w]);
            int before = 0, all = 0;
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) before += counts[w];
                all += counts[w];
            }
            for (int j = 0; j < kCandidates / kWave; ++j)
                if (j * kWave + (int)lane_id() < c.count) keys[before + j * kWave + lane_id()] = mine[j];
            __syncthreads();
            c.key = keys;
            c.count = all;
        }
        float power = 1.f;
        if constexpr (PROB) {
            power = sums.power_of();  // the same for all waves of the row
            if (power != 1.f) {
                sums = Scan::again(p, dim, WAVES == 1 ? 0 : wave, WAVES, power);
                if constexpr (WAVES > 1) {
                    if (lane_id() == 0) parts[wave] = sums;
                    __syncthreads();
                    sums = parts[0];
                    for (int w = 1; w < WAVES; ++w) sums.join<PROB>(parts[w]);
                }
            }
        }
        const RowLog<PROB> log(sums, dim, power);
        if (threadIdx.x % (WAVES * kWave) == 0 && o.entropy) o.entropy[row] = log.entropy;
        for (int k = threadIdx.x % (WAVES * kWave); k < o.given; k += WAVES * kWave) {
            const int g = o.classes[row * o.given + k];
            if (g >= dim && o.rejected) atomicAdd(o.rejected, 1);
            o.log_given[row * o.given + k] = g >= 0 && g < dim ? log.of(to_float(p[g])) : 0.f;
        }
        if (o.top && (WAVES == 1 || wave == 0)) write_top<PROB>(c, o, row, log);
        if constexpr (WAVES > 1) __syncthreads();
    }
}

// Many rows of up to 64 values, of which up to K classes are asked for: a lane for each row, from a copy of 64 rows in shared memory.  A lane keeps its first
// K in order, so that a value is compared with K others.  1M rows of 50, the first 4: probabilities 75 us, logits 77, in 16 bits 69; with 16 lanes for a row (k_short_scores) 173, 166
// and 150; 70,000 rows of 10, the first 2: 15.5 and 16.5.
template <typename T, bool PROB, int K>
__global__ __launch_bounds__(kWave) void k_lane_scores(const T* x, int64_t ld, int64_t rows, int dim, Scores o) {
    extern __shared__ char space[];
    float* copy = reinterpret_cast<float*>(space);
    const int pitch = dim | 1, lane = threadIdx.x;  // rows begin in different banks
#pragma unroll 1
    for (int64_t first = (int64_t)blockIdx.x * kWave; first < rows; first += (int64_t)gridDim.x * kWave) {
        const T* p = x + first * ld;
        const int here = (int)min(rows - first, (int64_t)kWave);
        constexpr int kAhead = 16;
        for (int from = 0; from < here; from += kAhead) {
            uint32_t v[kAhead];  // bits: as values of 16 bits two would share a register, and each load wait for the one before it
            for (int k = 0; k < kAhead; ++k) {
                const T one = p[min(from + k, here - 1) * ld + min(lane, dim - 1)];
                if constexpr (sizeof(T) == 2) v[k] = __builtin_bit_cast(uint16_t, one);
                else v[k] = __float_as_uint(one);
            }
            for (int k = 0; k < kAhead; ++k)
                if (lane < dim) {
                    if constexpr (sizeof(T) == 2) copy[min(from + k, here - 1) * pitch + lane] = to_float(__builtin_bit_cast(T, (uint16_t)v[k]));
                    else copy[min(from + k, here - 1) * pitch + lane] = __uint_as_float(v[k]);
                }
        }
        wave_meets();
        const float* mine = copy + min(lane, here - 1) * pitch;
        RowSums a = RowSums::none();
        float value[K];
        int at[K];
        for (int k = 0; k < K; ++k) value[k] = NAN, at[k] = 0;  // not a number: nothing yet
        if constexpr (!PROB) {
            float top = -INFINITY;
            for (int c = 0; c < dim; ++c) top = fmaxf(top, mine[c]);
            a.m = top;
        }
        const float base = a.base();
#pragma unroll 2
        for (int c = 0; c < dim; ++c) {
            const float x1 = mine[c];
            if constexpr (PROB) {
                a.add_probability(x1);
            } else {
                a.add_power((x1 - base) * kLog2e);
            }
            const float u = fmaxf(x1, -INFINITY);  // what is not a number counts as that
            bool before[K];
            for (int k = 0; k < K; ++k) before[k] = !(u <= value[k]);
            for (int k = K - 1; k >= 0; --k) {
                const float own = before[k] ? u : value[k];
                const int own_at = before[k] ? c : at[k];
                value[k] = k > 0 && before[k - 1] ? value[k - 1] : own;
                at[k] = k > 0 && before[k - 1] ? at[k - 1] : own_at;
            }
        }
        float power = 1.f;
        if constexpr (PROB) {
            power = a.power_of();
            if (power != 1.f) {
                a = RowSums::none();
                for (int c = 0; c < dim; ++c) a.add_probability(mine[c] * power);
            }
        }
        const RowLog<PROB> log(a, dim, power);
        const int64_t row = first + lane;
        if (lane < here) {
            if (o.entropy) o.entropy[row] = log.entropy;
            for (int k = 0; k < o.given; ++k) {
                const int g = o.classes[row * o.given + k];
                if (g >= dim && o.rejected) atomicAdd(o.rejected, 1);
                o.log_given[row * o.given + k] = g >= 0 && g < dim ? log.of(mine[g]) : 0.f;
            }
            for (int k = 0; k < K; ++k)
                if (k < o.top) {
                    if (o.top_classes) o.top_classes[row * o.top + k] = at[k];
                    if (o.log_top) o.log_top[row * o.top + k] = log.of(value[k]);
                }
        }
        wave_meets();
    }
}

// Rows of up to 64 values: 16 lanes for each, four values in a lane.  The first classes are taken one after the other; lane k mod 16 keeps the k-th until 16 are together.
template <typename T, bool PROB>
__global__ __launch_bounds__(kBlock) void k_short_scores(const T* x, int64_t ld, int64_t rows, int dim, Scores o) {
    const int r = threadIdx.x & 15, col = 4 * r;
    const int64_t step = (int64_t)gridDim.x * (kBlock / 16);
    Columns<T, 4> ahead;
    auto ask = [&](int64_t row) {
        const T* p = x + min(row, rows - 1) * ld;
        if (col + 4 <= dim) {
            __builtin_memcpy(ahead.d, p + col, sizeof ahead.d);
        } else {
            const Quad<T> some = load_quad(p, min(col, dim), dim);
            for (int k = 0; k < Columns<T, 4>::words; ++k) ahead.d[k] = some.d[k];
        }
    };
    ask((int64_t)blockIdx.x * (kBlock / 16) + threadIdx.x / 16);
#pragma unroll 1
    for (int64_t first = (int64_t)blockIdx.x * (kBlock / 16); first < rows; first += step) {
        const int64_t row = first + threadIdx.x / 16;
        const bool there = row < rows;
        const T* p = x + min(row, rows - 1) * ld;
        float v[4];
        for (int k = 0; k < 4; ++k) v[k] = col + k < dim ? ahead.get(k) : -INFINITY;
        if (first + step < rows) ask(row + step);
        RowSums a = RowSums::none();
        float top = largest_of(v);
        if constexpr (!PROB) top = __uint_as_float(over_16_lanes(__float_as_uint(top), MaxFloat()));
        a.add<PROB>(v, top);
        auto join = [&] {
            a.s = __uint_as_float(over_16_lanes(__float_as_uint(a.s), AddFloat()));
            a.t = __uint_as_float(over_16_lanes(__float_as_uint(a.t), AddFloat()));
        };
        join();
        float power = 1.f;
        if constexpr (PROB) {
            power = a.power_of();
            if (__any(power != 1.f)) {  // the wave's other rows have the same sums again
                a = RowSums::none();
                for (int k = 0; k < 4; ++k) a.add_probability(v[k] * power);
                join();
            }
        }
        const RowLog<PROB> log(a, dim, power);
        if (there && r == 0 && o.entropy) o.entropy[row] = log.entropy;
        if (there)
            for (int k = r; k < o.given; k += 16) {
                const int g = o.classes[row * o.given + k];
                if (g >= dim && o.rejected) atomicAdd(o.rejected, 1);
                o.log_given[row * o.given + k] = g >= 0 && g < dim ? log.of(to_float(p[g])) : 0.f;
            }
        if (o.top == 0) continue;
        uint32_t order[4];
        for (int k = 0; k < 4; ++k) order[k] = col + k < dim ? order_of(v[k]) : 0u;
        for (int from = 0; from < o.top; from += 16) {
            uint32_t my_order = 0, my_class = 0;
            const int here = min(o.top - from, 16);
            for (int place = 0; place < here; ++place) {
                const uint32_t best = over_16_lanes(max(max(order[0], order[1]), max(order[2], order[3])), Larger());
                uint32_t at = 64;
                for (int k = 3; k >= 0; --k) at = order[k] == best ? col + k : at;
                at = over_16_lanes(at, Smaller());
                for (int k = 0; k < 4; ++k) order[k] = (int)at == col + k ? 0u : order[k];
                my_order = r == place ? best : my_order;
                my_class = r == place ? at : my_class;
            }
            if (there && r < here) {
                if (o.top_classes) o.top_classes[row * o.top + from + r] = (int)my_class;
                if (o.log_top) o.log_top[row * o.top + from + r] = log.of(value_of((uint64_t)my_order << 32));
            }
        }
    }
}

}  // namespace dynlp
