// Scores of the head's answers.
//
// Up to 64 classes: logits and what they say, in registers (k_few_scores).  More: a product makes logits (k_wide, or k_thin_logits for up to 16 rows) and leaves with them
// what each group of classes of a row adds to its sums, and its largest logit.  The k-th largest of these is not above the row's k-th largest logit, so
// that k_group_scores looks at some k groups of a row again and not at all of it.
// What bounds it: 8,192 x 1,024 bfloat16, 32,768 classes: 756 us in two turns, whose products take 693 (770 TFLOP/s with 1.04 GB of logits stored; without stores and sums 930)
// and 39 (256 rows), the groups 48 and 16.
// 64 x 1,024, 131,072 classes: 78 us: the head once, 63 (4.3 TB/s), the groups 16, a wave for each row.  20,011 x 200 float16, 29 classes: 15 us, the host's call; 9 on the GPU.
#pragma once

#include "dynlp_head.h"
#include "dynlp_scores.h"
#include "dynlp_teach.h"

namespace dynlp {

// A group's sums, as in RowSums.
struct __attribute__((aligned(16))) GroupSums {
    float m, s, t, none;
};

// Of the lanes q that share a row r: their sums, joined.
__device__ inline RowSums joined_lanes(RowSums a) {
    a.rescale(row_max(a.m));
    a.s = row_sum(a.s);
    a.t = row_sum(a.t);
    return a;
}

// Logits to memory, of row n at n * ld, a multiple of 16; what lies behind the classes becomes -infinity.  Sums of 16 MI classes each.
struct Logits {
    float* z;
    int64_t ld;
    GroupSums* sums;  // [row][groups]
    int groups;
    const float* bias;
    int rows, classes;
    template <typename S>
    __device__ void finish(const Wide&, const Place& at, const f32x4 (&acc)[S::NI][S::MI], char* space) const {
        static_assert(!S::WOVEN, "fours");
        const bool shut = tile_bias<S>(bias, at.tile_m * S::TM, classes, space);
        const float* b = reinterpret_cast<float*>(space) + at.wave_m * (16 * S::MI);
        const int q = lane_id() >> 4, r = lane_id() & 15, group = at.tile_m * S::WM + at.wave_m;
#pragma unroll
        for (int i = 0; i < S::NI; ++i) {
            const int n = at.n0 + 16 * i + r;
            float v[S::MI * 4];
#pragma unroll
            for (int j = 0; j < S::MI; ++j) {
                const int m = at.m0 + 16 * j + 4 * q;
                float x[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                add_bias(b + 16 * j + 4 * q, shut, x);
                if (n < rows && m < ld) store_values<4>(z + n * ld + m, x);
                for (int k = 0; k < 4; ++k) v[4 * j + k] = x[k];
            }
            RowSums a = RowSums::none();
            a.add<false>(v, largest_of(v));
            a = joined_lanes(a);
            if (q == 0 && n < rows && group < groups) sums[(int64_t)n * groups + group] = GroupSums{a.m, a.s, a.t, 0.f};
        }
    }
};

// The same for up to 16 rows, without shared memory: 16 CT classes for each wave, whose loads are all under way at once.
template <typename T, int CT>
__global__ __launch_bounds__(kBlock) void k_thin_logits(Head a, Logits o) {
    const int group = __builtin_amdgcn_readfirstlane(blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave), first = group * 16 * CT;
    if (first >= a.classes) return;
    const WeightRows<T> w{static_cast<const T*>(a.weight) + first * a.ld_w, a.bias ? a.bias + first : nullptr, a.ld_w, a.dim, a.classes - first};
    f32x4 z[1][CT];
    head_logits<T, CT, 1, 4>(a, w, 0, z);
    const int q = lane_id() >> 4, r = lane_id() & 15;
    float v[4 * CT];
    for (int t = 0; t < CT; ++t) {
        const int m = first + 16 * t + 4 * q;
        float x[4] = {z[0][t][0], z[0][t][1], z[0][t][2], z[0][t][3]};
        if (r < a.rows && m < o.ld) store_values<4>(o.z + r * o.ld + m, x);
        for (int k = 0; k < 4; ++k) v[4 * t + k] = x[k];
    }
    RowSums sums = RowSums::none();
    sums.add<false>(v, largest_of(v));
    sums = joined_lanes(sums);
    if (q == 0 && r < a.rows) o.sums[(int64_t)r * o.groups + group] = GroupSums{sums.m, sums.s, sums.t, 0.f};
}

constexpr int kTurns = 8;  // of 64 heaps of groups, whose largest logits are in registers

// A wave for each row.  `merge` groups, a power of two, make a heap, of 1 << log2 fours of classes; there are up to 64 kTurns.
__global__ __launch_bounds__(kWave) inline void k_group_scores(const float* z, int64_t ld, const GroupSums* groups, int count, int merge, int log2, int64_t rows, int dim,
                                                               Scores o, int64_t row0) {
    constexpr int kAhead = 4;
    __shared__ uint64_t keys[kCandidates + kWave * 4];
    __shared__ int chosen[kTurns * kWave];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const float* p = z + row * ld;
        const int64_t to = row0 + row;
        RowSums sums = RowSums::none();
        uint32_t order[kTurns];
        for (int j = 0; j < kTurns; ++j) order[j] = 0;
#pragma unroll 2
        for (int part = 0; part < merge; ++part) {
            f32x4 s[kTurns];
#pragma unroll
            for (int j = 0; j < kTurns; ++j)
                s[j] = *reinterpret_cast<const f32x4*>(groups + row * count + min((j * kWave + (int)lane_id()) * merge + part, count - 1));
#pragma unroll
            for (int j = 0; j < kTurns; ++j)
                if ((j * kWave + (int)lane_id()) * merge + part < count) {
                    sums.join<false>(RowSums{s[j][0], s[j][1], s[j][2]});
                    order[j] = max(order[j], order_of(s[j][0]));
                }
        }
        sums.over_lanes<false>();
        const RowLog<false> log(sums, dim);
        if (lane_id() == 0 && o.entropy) o.entropy[to] = log.entropy;
        for (int k = lane_id(); k < o.given; k += kWave) {
            const int g = o.classes[to * o.given + k];
            if (g >= dim && o.rejected) atomicAdd(o.rejected, 1);
            o.log_given[to * o.given + k] = g >= 0 && g < dim ? log.of(p[g]) : 0.f;
        }
        if (o.top == 0) continue;
        Candidates c;
        c.none(keys);
        const uint32_t least = threshold<kTurns>(kTurns, o.top, 14, [&](int j) { return order[j]; });
        int found = 0;
        for (int j = 0; j < kTurns; ++j) {
            const bool hit = order[j] != 0 && order[j] >= least;
            const uint64_t mask = __ballot(hit);
            if (hit) chosen[found + lanes_before(mask)] = j * kWave + lane_id();
            found += __popcll(mask);
        }
        wave_meets();
        const int fours = found << log2;
#pragma unroll 1
        for (int from = 0; from < fours; from += kWave * kAhead) {
            f32x4 v[kAhead];
            int col[kAhead];
            for (int j = 0; j < kAhead; ++j) {
                const int k = from + j * kWave + lane_id();
                col[j] = k < fours ? ((chosen[k >> log2] << log2) + (k & ((1 << log2) - 1))) * 4 : dim;
                v[j] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if (col[j] < dim) v[j] = *reinterpret_cast<const f32x4*>(p + col[j]);
            }
            if (from == 0) {
                // of 128 pairs of fours the k-th largest maximum, as in RowScan
                uint32_t best[2];
                for (int j = 0; j < 2; ++j) {
                    float top = -INFINITY;
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(v[2 * j][e], v[2 * j + 1][e]));
                    best[j] = order_of(top);
                }
                c.raise(max(threshold<2>(2, o.top, 14, [&](int j) { return best[j]; }), 1u) - 1u);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                for (int e = 0; e < 4; ++e) c.put(v[j][e], col[j] + e, col[j] + e < dim);
                if (c.count > most_of(o.top)) c.cut(o.top, most_of(o.top));
            }
        }
        write_top<false>(c, o, to, log);
        wave_meets();
    }
}

// Up to 64 classes: 16 rows for each wave, four lanes to a row.
template <typename T, int CT, bool SHARED>
__global__ __launch_bounds__(kBlock) void k_few_scores(Head a, Scores o) {
    extern __shared__ char space[];
    const int q = lane_id() >> 4, r = lane_id() & 15;
    auto tile = [&](const auto& w, int64_t first) {
        f32x4 z[1][CT];
        head_logits<T, CT, 1, 4>(a, w, first, z);
        const int64_t row = first + r;
        const bool there = row < a.rows;
        float v[4 * CT];
        for (int t = 0; t < CT; ++t)
            for (int i = 0; i < 4; ++i) v[4 * t + i] = z[0][t][i];
        RowSums sums = RowSums::none();
        sums.add<false>(v, largest_of(v));
        sums = joined_lanes(sums);
        const RowLog<false> log(sums, a.classes);
        if (there && q == 0 && o.entropy) o.entropy[row] = log.entropy;
        for (int k = 0; k < o.given; ++k) {
            const int g = there ? o.classes[row * o.given + k] : -1;
            if (q == 0 && g >= a.classes && o.rejected) atomicAdd(o.rejected, 1);
            float x = 0.f;
            for (int t = 0; t < CT; ++t)
                for (int i = 0; i < 4; ++i) x = 16 * t + 4 * q + i == g ? v[4 * t + i] : x;
            x = row_sum(x);  // one lane's, zeros of the others
            if (there && q == 0) o.log_given[row * o.given + k] = g >= 0 && g < a.classes ? log.of(x) : 0.f;
        }
        if (o.top == 0) return;
        uint32_t order[4 * CT];
        for (int t = 0; t < CT; ++t)
            for (int i = 0; i < 4; ++i) order[4 * t + i] = 16 * t + 4 * q + i < a.classes ? order_of(v[4 * t + i]) : 0u;
        for (int place = 0; place < o.top; ++place) {
            uint32_t best = 0;
            int at = 4 * q;
            for (int t = 0; t < CT; ++t)
                for (int i = 0; i < 4; ++i)
                    if (order[4 * t + i] > best) best = order[4 * t + i], at = 16 * t + 4 * q + i;
            for (int d = 16; d < kWave; d <<= 1) {
                const uint32_t other = __shfl_xor(best, d, kWave);
                const int other_at = __shfl_xor(at, d, kWave);
                if (other > best || (other == best && other_at < at)) best = other, at = other_at;
            }
            for (int t = 0; t < CT; ++t)
                for (int i = 0; i < 4; ++i) order[4 * t + i] = 16 * t + 4 * q + i == at ? 0u : order[4 * t + i];
            if (there && q == (place & 3)) {
                if (o.top_classes) o.top_classes[row * o.top + place] = at;
                if (o.log_top) o.log_top[row * o.top + place] = log.of(value_of((uint64_t)best << 32));
            }
        }
    };
    const int64_t first = (threadIdx.x / kWave) * 16;
    if constexpr (SHARED) {
        const SharedWeight<T> w = share_weight<T, CT>(a, reinterpret_cast<T*>(space));
        for (int64_t at = (int64_t)blockIdx.x * kLabelRows; at + first < a.rows; at += (int64_t)gridDim.x * kLabelRows) tile(w, at + first);
    } else {
        const WeightRows<T> w{static_cast<const T*>(a.weight), a.bias, a.ld_w, a.dim, a.classes};
        if ((int64_t)blockIdx.x * kLabelRows + first < a.rows) tile(w, (int64_t)blockIdx.x * kLabelRows + first);
    }
}

}  // namespace dynlp
