// Products of matrices for heads of any number of classes, on the matrix cores, with what follows them done to the result where it lies in registers.
//
//   out[n][m] = sum over k of B(n, k) A(m, k),   m the fast index of the result
// Either operand lies in memory with k running along its rows ("along": operand[m][k]) or across them ("across": operand[k][m]).  Both come into shared
// memory by loads that do not pass through registers, 32 of k at a time in three turns, and are read from there as fragments of
// v_mfma_f32_16x16x32: along in 16-byte pieces, across by the reads that transpose 4 x 16 blocks of 16-bit elements on their way.  Pieces
// of a row change places by an XOR with bits of the row's number, so that neither kind of read meets another lane's bank.
// Fragments: lane l = 16 q + r holds columns (n) r and rows (m) 4 q .. 4 q + 3 of a result.  Which rows of A stand behind the 16 rows of a fragment is free: for results of 16
// bits four fragments share 64 of them (WOVEN) so that a lane has the 16 consecutive elements m = 16 q .. 16 q + 15 of row n, and four lanes a whole line of memory;
// for results of 32 bits the four consecutive elements of a fragment do.
// Sums are float32, products of 16-bit values are exact.  Operands in 32 bits come as bfloat16 terms that hold all 24 bits, and the sum runs over pairs of terms: six of
// the nine, the others lie below 2^-24 of the whole.  (Two terms of float16 would take three products, but only with a power of two for each matrix or row, under which a
// row of values of very different sizes loses its small ones.)
// What bounds it: 50,021 x 8,192 x 1,024 bfloat16 837 to 872 us without what follows (1,000 TFLOP/s; the library's product 1,029), 8,192^3 1,023 (library 1,400).
// The matrix cores are busy 41% of the time then, the requests to the L2 (64 bytes of a row per step) at 40% of its rate and shared memory at 40%.  Two workgroups to
// a CU, so that one's end and beginning fall into the other's sums; fragments of the next step read ahead, a fourth stage's worth of prefetch and s_setprio around the
// products changed nothing (837 / 848 / 839 us).
#pragma once

#include "dynlp_matrix.h"

namespace dynlp {

constexpr int kStep = 32;    // of k
constexpr int kStages = 3;   // steps in shared memory: one is read, two are under way
constexpr int kMostPairs = 6;

// One product.
struct Wide {
    const void *a, *b;          // first terms
    int64_t ld_a, ld_b;         // elements
    int64_t term_a, term_b;     // bytes from one term to the next
    int32_t m, n, k;            // along: rows of the operand that are there; across: k is
    int32_t steps;              // of one pair of terms
    int32_t pairs;
    uint32_t pair;              // 4 bits each: term of a, term of b << 2
    int32_t tiles_m, tiles_n;
    int32_t whole;              // tiles whose sum one workgroup makes; the others' are split
    int32_t splits, per_split;  // of the others; steps of each, over all pairs
    const uint32_t* kept;       // a bit per k: whether A's row k takes part (across), or NULL
    const void* zeros;          // 512 bytes of zeros in device memory, where kept is
};

// 64 lanes x 16 bytes from base + their offset to consecutive places of shared memory from `to` on (both the same for all lanes).  The compiler
// does not count these loads: whoever reads them waits by arrived().
__device__ inline void load_shared(const char* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" ::"s"(base), "v"(offset), "s"(to) : "memory", "m0");
}
__device__ inline void load_shared(const char* address, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(address), "s"(to) : "memory", "m0");
}
// All but the last N of a wave's loads are in shared memory.
template <int N>
__device__ inline void arrived() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All waves are here, and what they asked of shared memory is done.
__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

typedef __attribute__((address_space(3))) char* SharedBytes;
__device__ inline uint32_t shared_address(const void* p) { return (uint32_t)reinterpret_cast<uint64_t>((SharedBytes)p); }

// One operand's part of a stage: R rows (along) or columns (across), 64 R bytes.  WOVEN: four fragments share 64 rows.
template <int R, bool ACROSS, bool WOVEN>
struct Side {
    static constexpr int bytes = R * kStep * 2;
    static constexpr int loads = (R / 16 + 3) / 4;  // of a wave; where there are fewer than waves, several fetch the same
    uint32_t offset[loads];
    // What is added to a place in a row of pieces.
    __device__ static uint32_t key(int row) {
        if constexpr (!ACROSS) return WOVEN ? (row >> 4) & 3 : (row >> 2) & 3;
        else if constexpr (WOVEN) return R >= 128 ? (row & 1) | (row & 2) << 2 : (row >> 1) & 1;
        else return R >= 64 ? (row & 3) << 1 : 0;
    }
    __device__ static int load_of(int j, int wave) { return (wave + 4 * j) % (R / 16); }
    // Row of the operand, from the first one of the step on (across), or of the tile (along), of a lane's piece.
    __device__ static int row_of(int u) {
        const int at = u * 1024 + lane_id() * 16;
        return ACROSS ? at / (2 * R) : at / 64;
    }
    __device__ static int piece_of(int u) {
        const int at = u * 1024 + lane_id() * 16;
        const int row = row_of(u);
        return ACROSS ? (int)((at % (2 * R) / 16) ^ key(row)) : (int)((at % 64 / 16) ^ key(row));
    }
    // first: of the tile; there: rows (along) or columns, a multiple of 8 (across), that the operand has.
    __device__ void place(int wave, int first, int there, int64_t ld) {
        for (int j = 0; j < loads; ++j) {
            const int u = load_of(j, wave);
            if constexpr (ACROSS)
                offset[j] = (uint32_t)row_of(u) * (uint32_t)(2 * ld) + 2u * (uint32_t)min(8 * piece_of(u), there - first - 8);
            else
                offset[j] = (uint32_t)min(row_of(u), there - first - 1) * (uint32_t)(2 * ld) + 16u * (uint32_t)piece_of(u);
        }
    }
    // Asks for a step.  base: the tile's first element of the step; left: rows from the step's first on (across).
    __device__ void ask(int wave, const char* base, int64_t ld, int left, uint32_t to) const {
        if (ACROSS && left < kStep) {
            for (int j = 0; j < loads; ++j) {
                const int u = load_of(j, wave), row = row_of(u);
                load_shared(base, offset[j] - (uint32_t)max(row - (left - 1), 0) * (uint32_t)(2 * ld), to + 1024 * u);
            }
        } else {
            for (int j = 0; j < loads; ++j) load_shared(base, offset[j], to + 1024 * load_of(j, wave));
        }
    }
    // The same where rows may be left out, whose bits in `word` are zero: zeros come in their place.
    __device__ void ask(int wave, const char* base, int64_t ld, uint32_t word, const char* zeros, uint32_t to) const {
        if (word == 0xffffffffu) {
            for (int j = 0; j < loads; ++j) load_shared(base, offset[j], to + 1024 * load_of(j, wave));
        } else {
            for (int j = 0; j < loads; ++j) {
                const int u = load_of(j, wave);
                load_shared(word >> row_of(u) & 1 ? base + offset[j] : zeros, to + 1024 * u);
            }
        }
    }
    // Where a lane's part of fragment 0 lies in a stage, for the wave's rows from `first` on; of the others, see read().
    __device__ static u32x4 read(const char* stage, int first, int f) {
        const int q = lane_id() >> 4, r = lane_id() & 15;
        if constexpr (!ACROSS) {
            const int row = first + (WOVEN ? 64 * (f >> 2) + 16 * (r >> 2) + 4 * (f & 3) + (r & 3) : 16 * f + r);
            return *reinterpret_cast<const u32x4*>(stage + row * 64 + ((q ^ (r >> 2)) * 16));
        } else {
            u32x4 v;
            for (int half = 0; half < 2; ++half) {
                const int row = 8 * q + 4 * half + (r >> 2);
                const int piece = WOVEN ? (first + 64 * (f >> 2)) / 8 + 2 * (r & 3) + ((f & 3) >> 1) : (first + 16 * f) / 8 + ((r & 3) >> 1);
                const int at = row * (2 * R) + (int)((uint32_t)piece ^ key(row)) * 16 + (WOVEN ? f & 1 : r & 1) * 8;
                typedef short s16x4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) s16x4* Quads;
                const uint2 two = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Quads)(SharedBytes)(stage + at)));
                v[2 * half] = two.x, v[2 * half + 1] = two.y;
            }
            return v;
        }
    }
};

// Sizes of a workgroup's tile: TM x TN results, WM x WN waves.  256 x 128 has the fewest reads of shared memory per product that leave two workgroups room on a CU (72 KB each).
template <int TM_, int TN_, int WM_, int WN_, bool TA_, bool TB_, bool WOVEN_>
struct Shape {
    static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_;
    static constexpr bool TA = TA_, TB = TB_, WOVEN = WOVEN_;
    static constexpr int MI = TM / WM / 16, NI = TN / WN / 16;
    static constexpr int stage = (TM + TN) * kStep * 2;
    static_assert(WM * WN == 4 && MI % 4 == 0 && NI >= 1, "four waves, 64 rows of A at least for each");
};

// Where a wave's results belong.
struct Place {
    int m0, n0;     // first m and n of the wave
    int tile_m, tile_n, wave_m, wave_n;
    int tile, split;  // split: -1 where the tile's sum is whole
};

// A tile's sums over its steps.
template <typename T, typename S>
__device__ inline void wide_sums(const Wide& g, const Place& at, int tile_m0, int tile_n0, char* space, f32x4 (&acc)[S::NI][S::MI]) {
    using A = Side<S::TM, S::TA, S::WOVEN>;
    using B = Side<S::TN, S::TB, false>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    A a;
    B b;
    a.place(wave, tile_m0, g.m, g.ld_a);
    b.place(wave, tile_n0, g.n, g.ld_b);
    for (int i = 0; i < S::NI; ++i)
        for (int j = 0; j < S::MI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int first = at.split < 0 ? 0 : at.split * g.per_split, count = at.split < 0 ? g.pairs * g.steps : min(g.per_split, g.pairs * g.steps - first);
    // the step that is asked for next
    int pair = first / g.steps, step = first - pair * g.steps;
    const int64_t move_a = S::TA ? 2 * kStep * g.ld_a : 2 * kStep, move_b = S::TB ? 2 * kStep * g.ld_b : 2 * kStep;
    const char* origin_a = static_cast<const char*>(g.a) + (S::TA ? 2 * (int64_t)tile_m0 : 2 * tile_m0 * g.ld_a);
    const char* origin_b = static_cast<const char*>(g.b) + (S::TB ? 2 * (int64_t)tile_n0 : 2 * tile_n0 * g.ld_b);
    const uint32_t shared = __builtin_amdgcn_readfirstlane(shared_address(space));
    auto ask = [&](int slot) {
        const uint32_t code = g.pair >> (4 * pair);
        const char* pa = origin_a + (code & 3) * g.term_a + step * move_a;
        const char* pb = origin_b + (code >> 2 & 3) * g.term_b + step * move_b;
        const uint32_t to = shared + slot * S::stage;
        const int left = g.k - step * kStep;
        if (S::TA && g.kept) a.ask(wave, pa, g.ld_a, g.kept[step], static_cast<const char*>(g.zeros), to);
        else a.ask(wave, pa, g.ld_a, left, to);
        b.ask(wave, pb, g.ld_b, left, to + A::bytes);
        if (++step == g.steps) step = 0, ++pair;
    };
    constexpr int loads = A::loads + B::loads;
    const int wm = at.wave_m * (16 * S::MI), wn = at.wave_n * (16 * S::NI);
    ask(0);
    if (count > 1) ask(1);
    int slot = 0;
#pragma unroll 1
    for (int s = 0; s < count; ++s) {
        if (s + 1 < count) arrived<loads>();
        else arrived<0>();
        meet();
        const int next = slot == 0 ? 2 : slot - 1;  // (slot + 2) % 3
        if (s + 2 < count) ask(next);
        const char* stage = space + slot * S::stage;
        u32x4 x[S::MI], y[S::NI];
        for (int i = 0; i < S::NI; ++i) y[i] = B::read(stage + A::bytes, wn, i);
        for (int j = 0; j < S::MI; ++j) x[j] = A::read(stage, wm, j);
        for (int j = 0; j < S::MI; ++j)
            for (int i = 0; i < S::NI; ++i) acc[i][j] = mma(x[j], y[i], acc[i][j], T());
        slot = slot == 2 ? 0 : slot + 1;
    }
    meet();  // the stages are free
}

// Tiles in an order in which those that run at the same time on one of the eight dies share rows: 8 neighbours along n, then along m.
__device__ inline void tile_place(const Wide& g, int t, int* tile_m, int* tile_n) {
    const int group = 8 * g.tiles_m, first = t / group * 8, wide = min(g.tiles_n - first, 8), in = t - first * g.tiles_m;
    *tile_n = first + in % wide;
    *tile_m = in / wide;
}
// Workgroups go to the dies in turn: each die gets a range of `total` of them.
__device__ inline int of_die(int t, int total) {
    if (total < 64) return t;
    const int die = t & 7, each = total >> 3, rest = total & 7;
    return die * each + min(die, rest) + (t >> 3);
}
__device__ inline void wide_tile(const Wide& g, Place* at) {
    const int t = blockIdx.x, others = g.tiles_m * g.tiles_n - g.whole;
    if (t < g.whole) {
        at->tile = of_die(t, g.whole);
        at->split = -1;
    } else {
        const int k = of_die(t - g.whole, (int)gridDim.x - g.whole);
        at->split = k / others;
        at->tile = g.whole + k - at->split * others;
    }
    tile_place(g, at->tile, &at->tile_m, &at->tile_n);
}

// E does what follows: e.finish<S>(g, at, acc, space), with space to itself.
template <typename T, typename S, typename E>
__global__ __launch_bounds__(kBlock, 2) void k_wide(Wide g, E e) {
    extern __shared__ char space[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    Place at;
    wide_tile(g, &at);
    at.wave_m = wave % S::WM;
    at.wave_n = wave / S::WM;
    at.m0 = at.tile_m * S::TM + at.wave_m * (16 * S::MI);
    at.n0 = at.tile_n * S::TN + at.wave_n * (16 * S::NI);
    f32x4 acc[S::NI][S::MI];
    wide_sums<T, S>(g, at, at.tile_m * S::TM, at.tile_n * S::TN, space, acc);
    e.template finish<S>(g, at, acc, space);
}

// The 16 results of a lane for columns m .. m + 15 of row n, from fragments 4 j .. 4 j + 3.
template <int MI>
__device__ inline void sixteen(const f32x4 (&acc)[MI], int j, float (&v)[16]) {
    for (int t = 0; t < 4; ++t)
        for (int i = 0; i < 4; ++i) v[4 * t + i] = acc[4 * j + t][i];
}

// N values to columns col .. col + N - 1 of a row that has dim.
template <int N, typename O>
__device__ inline void store_some(O* row, int col, int dim, const float (&v)[N]) {
    if (col + N <= dim) {
        store_values<N>(row + col, v);
    } else {
        for (int k = 0; k < N; ++k)
            if (col + k < dim) row[col + k] = (O)v[k];
    }
}

// What becomes of a product's sums: times alpha (and *scale, and the row's own), rounded to O; rows that are left out are zeros; added to what is there.
template <typename O>
struct Output {
    O* out;
    int64_t ld;
    int rows, dim;
    float alpha;
    const float* scale;     // or NULL
    const float* of_row;    // a factor per row n, or NULL
    const uint32_t* kept;   // a bit per row n, or NULL
    bool add;
    __device__ float factor() const { return scale ? alpha * *scale : alpha; }
    __device__ float factor(int n, float of_all) const { return of_row ? of_all * of_row[n] : of_all; }
    template <int N>
    __device__ void put(int n, int m, float factor, float (&v)[N]) const {
        const bool zero = kept && !(kept[n >> 5] >> (n & 31) & 1);
        O* row = out + n * ld;
        for (int k = 0; k < N; ++k) v[k] = zero ? 0.f : v[k] * factor;
        if (add)
            for (int k = 0; k < N; ++k) v[k] += m + k < dim ? (float)row[m + k] : 0.f;
        store_some<N>(row, m, dim, v);
    }
};

// A product to its output; parts of split sums to memory, a tile after the other.
template <typename O>
struct Store {
    Output<O> to;
    float* part;
    template <typename S>
    __device__ void finish(const Wide& g, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char*) const {
        const int q = lane_id() >> 4, r = lane_id() & 15;
        if (at.split >= 0) {
            float* p = part + ((int64_t)(at.tile - g.whole) * g.splits + at.split) * (S::TM * S::TN);
#pragma unroll
            for (int i = 0; i < S::NI; ++i)
#pragma unroll
                for (int j = 0; j < S::MI; ++j) {
                    const int n = (at.wave_n * S::NI + i) * 16 + r;
                    const int m = 16 * S::MI * at.wave_m + (S::WOVEN ? 64 * (j >> 2) + 16 * q + 4 * (j & 3) : 16 * j + 4 * q);
                    *reinterpret_cast<f32x4*>(p + n * S::TM + m) = acc[i][j];
                }
            return;
        }
        const float of_all = to.factor();
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            if (n >= to.rows) continue;
            const float factor = to.factor(n, of_all);
            if constexpr (S::WOVEN) {
#pragma unroll
                for (int j = 0; j < S::MI / 4; ++j) {
                    const int m = at.m0 + 64 * j + 16 * q;
                    float v[16];
                    sixteen(acc[i], j, v);
                    if (m < to.dim) to.put(n, m, factor, v);
                }
            } else {
#pragma unroll
                for (int j = 0; j < S::MI; ++j) {
                    const int m = at.m0 + 16 * j + 4 * q;
                    float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    if (m < to.dim) to.put(n, m, factor, v);
                }
            }
        }
    }
};

// The tiles whose sums were split: their parts, in order.
template <typename O>
__global__ __launch_bounds__(kBlock) void k_wide_join(Wide g, int tm, int tn, const float* part, Output<O> to) {
    const int pieces = tm * tn / 4;
    const int64_t total = (int64_t)(g.tiles_m * g.tiles_n - g.whole) * pieces;
    const float factor = to.factor();
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
        const int tile = (int)(at / pieces), in = (int)(at - (int64_t)tile * pieces) * 4;
        int tile_m, tile_n;
        tile_place(g, g.whole + tile, &tile_m, &tile_n);
        const int n = tile_n * tn + in / tm, m = tile_m * tm + in % tm;
        if (n >= to.rows || m >= to.dim) continue;
        const float* p = part + (int64_t)tile * g.splits * (tm * tn) + in;
        f32x4 sum = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
        for (int k = 1; k < g.splits; ++k) sum += *reinterpret_cast<const f32x4*>(p + (int64_t)k * (tm * tn));
        float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        to.put(n, m, to.factor(n, factor), v);
    }
}

// A matrix rounded to O.
template <typename O>
__global__ __launch_bounds__(kBlock) void k_round(const float* in, int64_t rows, int dim, O* out, int64_t ld) {
    const int64_t total = rows * dim;
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < total; at += (int64_t)gridDim.x * kBlock) {
        const int64_t row = at / dim;
        out[row * ld + (at - row * dim)] = (O)in[at];
    }
}

}  // namespace dynlp
