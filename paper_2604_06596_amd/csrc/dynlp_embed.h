// Rows of items from a table of token rows, and the table's gradient.
//
// Both directions are one sum over a list of (key, source, factor) sorted by key:
//     out[key] = scale * sum of factor * rows[source]
// Forward the key is the item of a token and the source its id (the list is in order as it stands); backward the key is the id
// (the list is sorted by a stable radix sort) and the source the item.  Each row of `out` is written once; each row of `rows` is
// read once per token, from the caches as far as they hold it, and that is what bounds long lists: how many lines a CU can have
// under way, times how long the L2 (28 TB/s over the chip, measured with random rows of 256 bytes) or what lies behind it (7 TB/s) takes.
// Measured: 8.4M tokens, rows of 512 bytes: 390 us forward (11 TB/s; 43% of the requests hit the L2), 660 us backward for
// the sum alone (6.5 TB/s, all rows from behind the L2).  Forward 2.4 of 4.3 GB come from behind the L2: 6.1 TB/s, beside what it holds.
#pragma once

#include "dynlp_device.h"
#include "dynlp_types.h"

namespace dynlp {

// A lane's part of a row: V = Piece<T>::n elements in one 16-byte access, or V = 1 for rows shorter than that.
template <typename T, int V>
struct Lane {
    u32x4 raw;
    __device__ inline void load(const T* p) { raw = load_piece(p); }
    __device__ inline void keep(bool ok) {
        for (int k = 0; k < 4; ++k) raw[k] = ok ? raw[k] : 0u;
    }
    __device__ inline void get(float (&f)[V]) const { widen(raw, f, T()); }
};
template <typename T>
struct Lane<T, 1> {
    T raw;
    __device__ inline void load(const T* p) { raw = *p; }
    __device__ inline void keep(bool ok) { raw = ok ? raw : (T)0.f; }
    __device__ inline void get(float (&f)[1]) const { f[0] = to_float(raw); }
};

// The first column of lane-column c: pieces start at multiples of V, the last one at dim - V, so that rows whose length is no
// multiple of V need no tail (the columns two pieces share get the same value twice).
template <int V>
__device__ inline int piece_column(int c, int dim) {
    return min(c * V, dim - V);
}

struct TokenList {
    const void* ids;
    const int64_t* offsets;
    const float* weights;
    int32_t* rejected;
    int64_t count;
    int64_t items;
    int64_t limit;  // rows of the table
    float scale;
    bool wide;  // ids are int64

    // The id, or -1 for padding and for ids that are not below the table's rows.
    __device__ inline int32_t id(int64_t i, bool* out_of_range) const {
        const int64_t v = wide ? static_cast<const int64_t*>(ids)[i] : (int64_t) static_cast<const int32_t*>(ids)[i];
        *out_of_range = v >= limit;
        return v < 0 || v >= limit ? -1 : (int32_t)v;
    }
    __device__ inline int32_t id(int64_t i) const {
        bool ignored;
        return id(i, &ignored);
    }
    // The ids of tokens i, i + 64, ... below `end`, all asked for at once; -1 for what id() says so of, and beyond the end.
    template <int N>
    __device__ inline void ids_from(int64_t i, int64_t end, int32_t (&to)[N]) const {
        int64_t v[N];
        if (wide) {
            for (int u = 0; u < N; ++u) v[u] = i + u * kWave < end ? static_cast<const int64_t*>(ids)[i + u * kWave] : -1;
        } else {
            for (int u = 0; u < N; ++u) v[u] = i + u * kWave < end ? static_cast<const int32_t*>(ids)[i + u * kWave] : -1;
        }
        for (int u = 0; u < N; ++u) to[u] = v[u] < 0 || v[u] >= limit ? -1 : (int32_t)v[u];
    }
    // Bounds of item b within the list.
    __device__ inline void bounds(int64_t b, int64_t* begin, int64_t* end) const {
        *begin = min(max(offsets[b], (int64_t)0), count);
        *end = min(max(offsets[b + 1], *begin), count);
    }
    // The last item in [lo, hi] whose tokens begin at or before i, given that lo's do (or lo is -1).
    __device__ inline int64_t item_from(int64_t i, int64_t lo, int64_t hi) const {
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) >> 1;
            if (offsets[mid] <= i)
                lo = mid;
            else
                hi = mid - 1;
        }
        return lo;
    }
    // The same over all items by a whole wave, 64 offsets at a time: as many reads one after the other as 64 has to be multiplied by itself.
    __device__ inline int64_t item_by_wave(int64_t i) const {
        int64_t lo = -1, hi = items;  // the answer is in [lo, hi]
        while (lo < hi) {
            const int64_t step = (hi - lo + kWave - 1) / kWave;
            const int64_t at = lo + step * (lane_id() + 1);
            const unsigned long long m = __ballot(at <= hi && offsets[min(at, hi)] <= i);
            const int n = (int)__popcll(m);  // offsets do not decrease: these are the first n lanes
            hi = min(lo + step * (n + 1) - 1, hi);
            lo = lo + step * n;
        }
        return lo;
    }
    // The item of token i, -1 if it is in none.
    __device__ inline int32_t item(int64_t i) const {
        if (!offsets) return (int32_t)i;
        const int64_t b = item_from(i, -1, items);
        return b < items ? (int32_t)b : -1;
    }
};

__device__ inline void count_rejected(int32_t* rejected, bool bad) {
    const unsigned long long m = __ballot(bad);
    if (m && rejected && lane_id() == __ffsll(m) - 1) atomicAdd(rejected, (int)__popcll(m));
}

// Counts the ids that are not below the table's rows, where nothing else looks at them: without items, or without rows.
__global__ __launch_bounds__(kBlock) void k_count_rejected(TokenList t) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < t.count; i += (int64_t)gridDim.x * kBlock) {
        bool bad;
        t.id(i, &bad);
        count_rejected(t.rejected, bad);
    }
}

// ---- one row per token -----------------------------------------------------------------------------------------------

// out[i] = scale * weight * table[id]: a copy with a factor, bound by the memory: 65,536 rows of 1,000 float16 from a table of 250,007: 46 to 48 us
// (3.9 TB/s of what has to move, with one piece per thread 50 us).  Four 16-byte pieces per thread, asked for at once; `pieces` of them make a row.
constexpr int kRowsAhead = 4;
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_embed_rows(TokenList t, const T* table, int64_t ld, T* out, int64_t out_ld, int dim,
                                                       int pieces) {
    const int64_t first = (int64_t)blockIdx.x * (kBlock * kRowsAhead);
    const int64_t row0 = first / pieces;             // the same for all threads
    const uint32_t rest = (uint32_t)(first - row0 * pieces);
    Lane<T, V> x[kRowsAhead];
    float s[kRowsAhead];
    int64_t row[kRowsAhead];
    int col[kRowsAhead];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
        const uint32_t at = rest + (uint32_t)(k * kBlock) + threadIdx.x, r = at / (uint32_t)pieces, c = at - r * (uint32_t)pieces;
        row[k] = row0 + r;
        col[k] = piece_column<V>((int)c, dim);
        s[k] = 0.f;
        if (row[k] < t.count) {
            bool bad;
            const int32_t id = t.id(row[k], &bad);
            if (bad && c == 0 && t.rejected) atomicAdd(t.rejected, 1);
            if (id >= 0) {
                s[k] = t.weights ? t.scale * t.weights[row[k]] : t.scale;
                x[k].load(table + (int64_t)id * ld + col[k]);
            }
            x[k].keep(id >= 0);
        }
    }
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k)
        if (row[k] < t.count) {
            float f[V];
            x[k].get(f);
            for (int e = 0; e < V; ++e) f[e] *= s[k];
            store_values<V>(out + row[k] * out_ld + col[k], f);
        }
}

// Zeros in the rows of `out` from `first` on that the lanes ask for, 64 at most: lane l for row first + l.  From whole waves.
template <typename T, int V>
__device__ inline void zero_rows_of_wave(bool mine, int64_t first, T* out, int64_t out_ld, int dim) {
    const float zero[V] = {};
    const int pieces = (dim + V - 1) / V;
    for (unsigned long long m = __ballot(mine); m; m &= m - 1) {
        T* row = out + (first + __ffsll(m) - 1) * out_ld;
        for (int c = lane_id(); c < pieces; c += kWave) store_values<V>(row + piece_column<V>(c, dim), zero);
    }
}

// ---- few tokens: one workgroup per item, or per distinct id ----------------------------------------------------------

// Sum of factor * rows[source] over a workgroup's list, lanes of a group across the columns, groups taking turns on the list;
// the groups' sums are joined in their order.  Lists of a few thousand at most.
template <typename T, typename O, int V, typename Entry>
__device__ inline void block_sum(const T* rows, int64_t ld, int dim, int lanes_log2, int64_t n, Entry entry, float scale, O* out) {
    __shared__ float part[kBlock * V];
    const int lanes = 1 << lanes_log2, groups = kBlock >> lanes_log2;
    const int g = threadIdx.x >> lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int pieces = (dim + V - 1) / V;
    for (int c0 = 0; c0 < pieces; c0 += lanes) {
        const int c = c0 + lane;
        const bool inside = c < pieces;
        const int col = piece_column<V>(inside ? c : pieces - 1, dim);
        float acc[V] = {};
        constexpr int U = 4;
        for (int64_t i = g; i < n; i += (int64_t)U * groups) {
            Lane<T, V> x[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                int64_t src = -1;
                w[u] = 0.f;
                if (i + (int64_t)u * groups < n) src = entry(i + (int64_t)u * groups, &w[u]);
                x[u].load(rows + max(src, (int64_t)0) * ld + col);
                x[u].keep(src >= 0);
                w[u] = src >= 0 ? w[u] : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                x[u].get(f);
                for (int k = 0; k < V; ++k) acc[k] += w[u] * f[k];
            }
        }
        for (int k = 0; k < V; ++k) part[threadIdx.x * V + k] = acc[k];
        __syncthreads();
        if (g == 0 && inside) {
            for (int o = 1; o < groups && o < n; ++o)
                for (int k = 0; k < V; ++k) acc[k] += part[(o * lanes + lane) * V + k];
            for (int k = 0; k < V; ++k) acc[k] *= scale;
            store_values<V>(out + col, acc);
        }
        __syncthreads();
    }
}

// An item per workgroup: latency is all there is (one item of 37 tokens: 3.6 us on the GPU, 9 us with the call).
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_embed_items(TokenList t, const T* table, int64_t ld, T* out, int64_t out_ld, int dim,
                                                        int lanes_log2) {
    const int64_t b = blockIdx.x;
    int64_t begin, end;
    t.bounds(b, &begin, &end);
    if (b == 0 && t.rejected)  // of the whole list: some tokens may be in no item
        for (int64_t i = threadIdx.x; i < t.count; i += kBlock) {
            bool bad;
            t.id(i, &bad);
            count_rejected(t.rejected, bad);
        }
    block_sum<T, T, V>(
        table, ld, dim, lanes_log2, end - begin,
        [&](int64_t i, float* w) -> int64_t {
            const int32_t id = t.id(begin + i);
            *w = t.weights ? t.weights[begin + i] : 1.f;
            return id;
        },
        begin < end ? t.scale : 0.f, out + b * out_ld);  // zeros without tokens, whatever the scale
}

constexpr int kFewTokens = 8192;     // 32 for each thread of a workgroup
constexpr int kZeroRows = 8192;      // rows whose presence one workgroup notes at most

// The gradient for few tokens, without a sort: a workgroup per token looks through all ids, each wave through a quarter of them.  If token i is the first
// with its id, every wave adds up the rows of those it found, four at a time, and the waves' sums are joined in order.  The workgroups before those zero the rows of
// ids that do not occur.  One launch instead of the sort's nine; the ids are read count^2 times, from the L2.  4,099 tokens,
// rows of 128 float32, a table of 30,011: 19 us (switched off one at a time, the look through the ids is worth 6, the zeros 3; the rest was not taken
// apart: workgroups are short, and 22 KB of shared memory lets seven on a CU); by the sort it would be some 45 us.
template <typename T, typename O, int V>
__global__ __launch_bounds__(kBlock) void k_embed_grad_few(TokenList t, const T* grad, int64_t ld, O* out, int64_t out_ld, int dim, int zero_rows,
                                                           int zero_blocks) {
    constexpr int kWaves = kBlock / kWave, kAhead = 8;
    __shared__ float part[kWaves][kWave * V];
    __shared__ uint16_t list[kWaves][kFewTokens / kWaves];
    __shared__ int found[kWaves];
    __shared__ uint32_t present[kZeroRows / 32];
    const int n = (int)t.count, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
    const int pieces = (dim + V - 1) / V;
    if ((int)blockIdx.x >= zero_blocks) {
        const int me = (int)blockIdx.x - zero_blocks;
        bool bad;
        const int32_t id = t.id(me, &bad);
        if (bad && threadIdx.x == 0 && t.rejected) atomicAdd(t.rejected, 1);
        if (id < 0) return;
        const int from = (int)((int64_t)n * wave / kWaves), to = (int)((int64_t)n * (wave + 1) / kWaves);
        bool earlier = false;
        int mine = 0;
        for (int i0 = from; i0 < to; i0 += kAhead * kWave) {
            int32_t ids[kAhead];
            t.ids_from<kAhead>(i0 + lane, to, ids);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = i0 + u * kWave + lane;
                const bool hit = ids[u] == id;
                const unsigned long long m = __ballot(hit);
                if (!m) continue;
                earlier |= hit && i < me;
                if (hit) list[wave][mine + (int)__popcll(m & ((1ull << lane) - 1))] = (uint16_t)i;
                mine += (int)__popcll(m);
            }
        }
        if (lane == 0) found[wave] = mine;
        if (__syncthreads_or(earlier)) return;
        int others = 0;
        for (int w = 0; w < kWaves; ++w) others += w == wave ? 0 : found[w];
        O* row = out + (int64_t)id * out_ld;
        const bool alone = __syncthreads_and(mine == 0 || others == 0);
        for (int c0 = 0; c0 < pieces; c0 += kWave) {
            const bool inside = c0 + lane < pieces;
            const int col = piece_column<V>(inside ? c0 + lane : pieces - 1, dim);
            float acc[V] = {};
            constexpr int U = 4;
            for (int k = 0; k < mine; k += U) {
                Lane<T, V> x[U];
                float w[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int pos = list[wave][min(k + u, mine - 1)];
                    const int64_t src = t.item(pos);
                    const bool ok = k + u < mine && src >= 0;
                    w[u] = t.weights ? t.weights[pos] : 1.f;
                    w[u] = ok ? w[u] : 0.f;
                    x[u].load(grad + max(src, (int64_t)0) * ld + col);
                    x[u].keep(ok);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float f[V];
                    x[u].get(f);
                    for (int e = 0; e < V; ++e) acc[e] += w[u] * f[e];
                }
            }
            if (!alone) {
                for (int e = 0; e < V; ++e) part[wave][lane * V + e] = acc[e];
                __syncthreads();
                if (wave == 0)
                    for (int w = 1; w < kWaves; ++w)
                        for (int e = 0; e < V; ++e) acc[e] += part[w][lane * V + e];
            }
            if (inside && (alone ? mine > 0 : wave == 0)) {
                for (int e = 0; e < V; ++e) acc[e] *= t.scale;
                store_values<V>(row + col, acc);
            }
            if (!alone) __syncthreads();
        }
        return;
    }
    const int64_t first = (int64_t)blockIdx.x * zero_rows;
    const int rows = (int)min((int64_t)zero_rows, t.limit - first);
    for (int k = threadIdx.x; k < (zero_rows + 31) / 32; k += kBlock) present[k] = 0;
    __syncthreads();
    for (int i0 = wave * kAhead * kWave; i0 < n; i0 += kWaves * kAhead * kWave) {
        int32_t ids[kAhead];
        t.ids_from<kAhead>(i0 + lane, n, ids);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t r = (int64_t)ids[u] - first;
            if (r >= 0 && r < rows) atomicOr(&present[r >> 5], 1u << (r & 31));
        }
    }
    __syncthreads();
    for (int r0 = wave * kWave; r0 < rows; r0 += kBlock) {
        const int r = r0 + lane;
        zero_rows_of_wave<O, V>(r < rows && !(present[r >> 5] >> (r & 31) & 1), first + r0, out, out_ld, dim);
    }
}

// ---- long lists: sums over pieces of the list, joined ----------------------------------------------------------------

// Zeros in the rows of items without tokens: block `block` looks at kBlock items.
template <typename T, int V>
__device__ inline void zero_empty_items(const TokenList& t, int64_t block, T* out, int64_t out_ld, int dim) {
    const int64_t first = block * kBlock + (threadIdx.x / kWave) * kWave, mine = first + lane_id();
    bool empty = false;
    if (mine < t.items) {
        int64_t begin, end;
        t.bounds(mine, &begin, &end);
        empty = begin == end;
    }
    zero_rows_of_wave<T, V>(empty, first, out, out_ld, dim);
}

// mark[i] = the item of token first + i, for a tile of TILE tokens of which n are there: -1 before the first item, t.items behind the last.  Each
// item that begins in the tile is noted at its first token, and a running maximum carries it on.  From all threads of the workgroup.
// Where far more items than tokens begin in the tile (a long run without tokens) each token looks for its own instead.  Rows of 16 float32, 40,000 tokens,
// 16,000 items in one tile: 49 us by a look through the items, 46 by the search; a million: 1,203 and 74.  Eight empty items to each token: 46 and 52, sixteen:
// 78 and 67.
constexpr int kItemsOfTile = 12;  // per token
template <int TILE, int NT>
__device__ inline void tile_items(const TokenList& t, int64_t first, int n, int32_t* mark, int32_t* range) {
    constexpr int per = TILE / NT;
    if (threadIdx.x < 2) range[threadIdx.x] = (int32_t)t.item_from(threadIdx.x ? first + n - 1 : first, -1, t.items);
    __syncthreads();
    const int32_t lo = range[0], hi = range[1];
    if (hi - lo > kItemsOfTile * TILE) {
        for (int i = threadIdx.x; i < n; i += NT) mark[i] = (int32_t)t.item_from(first + i, lo, hi);
        __syncthreads();
        return;
    }
    for (int i = threadIdx.x; i < TILE; i += NT) mark[i] = lo;
    __syncthreads();
    for (int64_t b = (int64_t)lo + 1 + threadIdx.x; b <= hi; b += NT) {
        const int64_t at = t.offsets[b] - first;
        if (at >= 0 && at < n) atomicMax(&mark[at], (int32_t)b);
    }
    __syncthreads();
    int32_t v[per], top = -1;
    for (int k = 0; k < per; ++k) {
        top = max(top, mark[threadIdx.x * per + k]);
        v[k] = top;
    }
    // the largest of the threads before this one: over the wave, then over the waves
    int32_t run = top;
    for (int d = 1; d < kWave; d <<= 1) {
        const int32_t o = __shfl_up(run, d, kWave);
        if (lane_id() >= d) run = max(run, o);
    }
    int32_t before = __shfl_up(run, 1, kWave);
    if (lane_id() == 0) before = -1;
    if (lane_id() == kWave - 1) range[2 + threadIdx.x / kWave] = run;
    __syncthreads();
    for (int w = 0; w < (int)threadIdx.x / kWave; ++w) before = max(before, range[2 + w]);
    for (int k = 0; k < per; ++k) mark[threadIdx.x * per + k] = max(v[k], before);
    __syncthreads();
}
constexpr int kTileRange = 2 + 1024 / kWave;  // words of tile_items' `range`, of the largest workgroup

// For rows that are narrower than a wave: key[i] = the item of token i (-1: none), src[i] = its id (-1: contributes nothing); the blocks
// behind those of the tokens zero the rows of items without tokens.
constexpr int kKeyTile = 2048;
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_item_keys(TokenList t, int32_t* key, int32_t* src, int token_blocks, T* out,
                                                      int64_t out_ld, int dim) {
    if ((int)blockIdx.x >= token_blocks) {
        zero_empty_items<T, V>(t, (int64_t)blockIdx.x - token_blocks, out, out_ld, dim);
        return;
    }
    __shared__ int32_t mark[kKeyTile], range[kTileRange];
    const int64_t first = (int64_t)blockIdx.x * kKeyTile;
    const int n = (int)min((int64_t)kKeyTile, t.count - first);
    tile_items<kKeyTile, kBlock>(t, first, n, mark, range);
    for (int i = threadIdx.x; i < n; i += kBlock) {
        key[first + i] = mark[i] < t.items ? mark[i] : -1;
        bool bad;
        src[first + i] = t.id(first + i, &bad);
        count_rejected(t.rejected, bad);
    }
}

enum : uint8_t {
    kHead = 1,    // the piece's first run began before it; its sum is head[piece]
    kThrough = 2  // and goes on behind it
};

struct SumList {
    const int32_t* key;    // ascending; a key outside [0, out_rows) is written nowhere
    const int32_t* src;    // a source outside [0, row_count) contributes nothing
    const float* factor;   // or NULL
    float* part;           // [piece][head, tail][dim]
    uint8_t* flags;        // [piece]
    int32_t* open;         // [piece] key of the piece's last run if that began in it and goes on behind it (its sum is tail[piece]); else -1
    uint8_t* present;      // [out_rows] set for keys that occur, or NULL
    int64_t count;
    int64_t row_count, out_rows;
    int piece;             // entries of a piece of the list
    float scale;

    __device__ inline bool real(int32_t k) const { return k >= 0 && k < out_rows; }
    // What a piece leaves beside its sums; by one lane.
    __device__ inline void leave(int64_t g, uint8_t f, int32_t k) const {
        flags[g] = f;
        open[g] = k;
        if (present && k >= 0) present[k] = 1;
    }
};

// For rows that are narrower than a wave: a group of lanes goes through one piece of the list with a running sum; lanes are across the
// columns.  Eight rows are asked for at a time.  Runs that lie within the piece are written to `out`, the first and the last, where
// they go on beyond it, to `part`.
template <typename T, typename O, int V>
__global__ __launch_bounds__(kBlock) void k_segment_sum(SumList s, const T* rows, int64_t ld, O* out, int64_t out_ld, int dim,
                                                        int lanes_log2) {
    const int64_t g = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lanes_log2;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1);
    const int64_t first = g * s.piece;
    if (first >= s.count || lane * V >= dim) return;
    const int col = piece_column<V>(lane, dim);
    const int64_t end = min(first + s.piece, s.count);
    rows += col;
    out += col;
    float* part = s.part + g * 2 * dim + col;
    int32_t cur = s.key[first];
    bool before = first > 0 && s.key[first - 1] == cur;
    uint8_t flags = 0;
    float acc[V] = {};
    auto flush = [&]() {
        if (before) {
            store_values<V>(part, acc);
            flags |= kHead;
        } else if (s.real(cur)) {
            float f[V];
            for (int k = 0; k < V; ++k) f[k] = acc[k] * s.scale;
            store_values<V>(out + (int64_t)cur * out_ld, f);
            if (s.present && lane == 0) s.present[cur] = 1;
        }
    };
    constexpr int U = 8;
    for (int64_t i = first; i < end; i += U) {
        int32_t key[U];
        Lane<T, V> x[U];
        float w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = min(i + u, end - 1);
            key[u] = s.key[at];
            const int32_t src = s.src[at];
            const bool ok = src >= 0 && src < s.row_count && i + u < end;
            w[u] = s.factor ? s.factor[at] : 1.f;
            w[u] = ok ? w[u] : 0.f;
            x[u].load(rows + (int64_t)(ok ? src : 0) * ld);
            x[u].keep(ok);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (key[u] != cur) {
                flush();
                cur = key[u];
                before = false;
                for (int k = 0; k < V; ++k) acc[k] = 0.f;
            }
            float f[V];
            x[u].get(f);
            for (int k = 0; k < V; ++k) acc[k] += w[u] * f[k];
        }
    }
    const bool goes_on = end < s.count && s.key[end] == cur;
    if (goes_on && before) {
        store_values<V>(part, acc);
        flags |= kHead | kThrough;
    } else if (goes_on) {
        store_values<V>(part + dim, acc);
    } else {
        flush();
    }
    if (lane == 0) s.leave(g, flags, goes_on && !before && s.real(cur) ? cur : -1);
}

// Items without tokens that a wave passes one by one before it looks for the next item over all (k_wave_sum).  128 bfloat16, 40,000 tokens, an empty
// item to each: 28 us, 38 with a search at once; six empty items to each token: 51 one by one, 46 with the search; a million between two texts: 103 ms and 84 us.
constexpr int kEmptyItems = 3;

// For rows of 256 bytes and more: a wave goes through one piece of the list (E columns per lane, blockIdx.y: 64 E columns).  64 entries are
// read at once, one per lane; each is then handed to all lanes through scalar registers, so that a row's address, the end of a run and
// the branch over what contributes nothing cost the vector units nothing: per entry they unpack and add E columns.  Eight or sixteen rows are
// asked for at a time.  131,072 items of 64 tokens, 256 bfloat16: 390 us, bound by the caches (groups of 32 lanes with keys and sources read by every
// lane: 640 us); 20,011 items of 60 tokens, 128 bfloat16: 40 us.  With ITEMS the keys are the items, whose bounds are read from the offsets as they come; the blocks behind those of the list
// zero the rows of items without tokens.  PAST: `out` is not to take the caches from `rows`.
template <typename T, typename O, int E, bool ITEMS, bool PAST>
__global__ __launch_bounds__(kBlock) void k_wave_sum(SumList s, TokenList t, const T* rows, int64_t ld, O* out, int64_t out_ld, int dim,
                                                     int sum_blocks) {
    if (ITEMS && (int)blockIdx.x >= sum_blocks) {
        if (blockIdx.y == 0) zero_empty_items<O, Piece<O>::n>(t, (int64_t)blockIdx.x - sum_blocks, out, out_ld, dim);
        return;
    }
    const int64_t g = (int64_t)blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t first = g * s.piece;
    if (first >= s.count) return;
    const int64_t end = min(first + s.piece, s.count);
    const int lane = lane_id();
    const int c = (int)blockIdx.y * (kWave * E) + lane * E;
    const bool inside = c < dim;
    const int col = min(c, dim - E);
    const uint32_t off = (uint32_t)col * (uint32_t)sizeof(T);  // beside a row's address, which is the same for all lanes
    out += col;
    float* part = s.part + g * 2 * dim + col;
    int64_t item = 0, next = 0;  // ITEMS: the item at hand and where it ends
    int32_t cur;
    bool before;
    if (ITEMS) {
        item = t.item_by_wave(first);
        next = item < t.items ? t.offsets[item + 1] : INT64_MAX;
        cur = item >= 0 && item < t.items ? (int32_t)item : -1;
        before = cur >= 0 && max(t.offsets[item], (int64_t)0) < first;  // what an item has before the list is no token
    } else {
        cur = s.key[first];
        before = first > 0 && s.key[first - 1] == cur;
    }
    uint8_t flags = 0;
    float acc[E] = {};
    auto flush = [&]() {
        if (before) {
            if (inside) store_values<E>(part, acc);
            flags |= kHead;
        } else if (s.real(cur)) {
            float f[E];
            for (int k = 0; k < E; ++k) f[k] = acc[k] * s.scale;
            if (inside) store_values<E, PAST>(out + (int64_t)cur * out_ld, f);
            if (!ITEMS && s.present && c == 0) s.present[cur] = 1;
        }
        before = false;
        for (int k = 0; k < E; ++k) acc[k] = 0.f;
    };
    constexpr int U = Columns<T, E>::words <= 2 ? 16 : 8;
    constexpr unsigned kAll = (1u << U) - 1;
    for (int64_t base = first; base < end; base += kWave) {
        const int64_t at = base + lane;
        const int n = (int)min((int64_t)kWave, end - base);
        int32_t src = -1, key = cur;
        float w = 0.f;
        unsigned long long ends = 0;  // sorted lists: entries that begin another run
        if (ITEMS) {
            bool bad = false;
            if (lane < n) {
                src = t.id(at, &bad);
                if (src >= 0) w = t.weights ? t.weights[at] : 1.f;
            }
            if (blockIdx.y == 0) count_rejected(t.rejected, bad);
        } else {
            if (lane < n) {
                key = s.key[at];
                src = s.src[at];
                if (!s.real(key) || src >= s.row_count) src = -1;
                if (src >= 0) w = s.factor ? s.factor[at] : 1.f;
            }
            int32_t last = __shfl_up(key, 1, kWave);
            if (lane == 0) last = cur;
            ends = __ballot(lane < n && key != last);
        }
        const unsigned long long real = __ballot(src >= 0);
        const uint64_t address = reinterpret_cast<uint64_t>(rows + (int64_t)max(src, 0) * ld);
        uint32_t low = (uint32_t)address, high = (uint32_t)(address >> 32), factor = __float_as_uint(w);
        for (int j = 0; j < n; j += U) {
            Columns<T, E> x[U];
            float f[U];
            auto ask = [&](int u) {
                x[u].load((uint64_t)(uint32_t)__builtin_amdgcn_readlane(high, u) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, u), off);
            };
            if ((real >> j & kAll) == kAll) {
#pragma unroll
                for (int u = 0; u < U; ++u) ask(u);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (real >> (j + u) & 1)
                        ask(u);
                    else
                        x[u].zero();
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) f[u] = __uint_as_float(__builtin_amdgcn_readlane(factor, u));
            // the next U entries to the first lanes
            low = __shfl_down(low, U, kWave);
            high = __shfl_down(high, U, kWave);
            factor = __shfl_down(factor, U, kWave);
            const int64_t pos = base + j;
            if (ITEMS ? next >= end || next >= pos + U : (ends >> j & kAll) == 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    for (int e = 0; e < E; ++e) acc[e] += f[u] * x[u].get(e);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (ITEMS) {
                        if (pos + u == next && next < end) {
                            flush();
                            int passed = 0;
                            do {
                                ++item;
                            } while (item < t.items && t.offsets[item + 1] <= pos + u && ++passed < kEmptyItems);
                            if (passed == kEmptyItems) item = t.item_by_wave(pos + u);
                            next = item < t.items ? t.offsets[item + 1] : INT64_MAX;
                            cur = item < t.items ? (int32_t)item : -1;
                        }
                    } else if (ends >> (j + u) & 1) {
                        flush();
                        cur = __builtin_amdgcn_readlane(key, j + u);
                    }
                    for (int e = 0; e < E; ++e) acc[e] += f[u] * x[u].get(e);
                }
            }
        }
    }
    const bool goes_on = end < s.count && (ITEMS ? next > end : s.key[end] == cur);
    const bool opens = goes_on && !before;
    if (goes_on && before) {
        if (inside) store_values<E>(part, acc);
        flags |= kHead | kThrough;
    } else if (goes_on) {
        if (inside) store_values<E>(part + dim, acc);
    } else {
        flush();
    }
    if (c == 0) s.leave(g, flags, opens && s.real(cur) ? cur : -1);
}

// Runs that several pieces share: the wave of the piece in which such a run begins adds up its parts, in their order within each group of
// lanes, then the groups'.  One wave joins a run, however many pieces it has: 8.4M tokens, 256 float32 columns, 17 us where the most frequent id has 0.8% of
// them (the sum itself takes 660), 106 where it has 6%, 1.5 ms where there is no other.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void k_segment_join(SumList s, int64_t pieces, O* out, int64_t out_ld, int dim, int lanes_log2) {
    const int64_t p = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kWave;
    if (p >= pieces) return;
    const int32_t key = s.open[p];
    if (key < 0) return;
    int64_t last = p + 1;  // the piece in which the run ends
    for (;; last += kWave) {
        const int64_t at = last + lane_id();
        const unsigned long long m = __ballot(at >= pieces || !(s.flags[at] & kThrough));
        if (m) {
            last += __ffsll(m) - 1;
            break;
        }
    }
    const int lanes = 1 << lanes_log2, groups = kWave >> lanes_log2;
    const int g = lane_id() >> lanes_log2, c = ((int)blockIdx.y << lanes_log2) + (lane_id() & (lanes - 1));
    const bool inside = c * V < dim;
    const int col = inside ? piece_column<V>(c, dim) : 0;
    const float* part = s.part + col;
    float acc[V] = {};
    if (g == 0)
        for (int k = 0; k < V; ++k) acc[k] = part[(p * 2 + 1) * dim + k];
#pragma unroll 4
    for (int64_t j = p + 1 + g; j <= last; j += groups)
        for (int k = 0; k < V; ++k) acc[k] += part[j * 2 * dim + k];
    for (int d = lanes; d < kWave; d <<= 1)
        for (int k = 0; k < V; ++k) acc[k] += __shfl_xor(acc[k], d, kWave);
    if (g == 0 && inside) {
        for (int k = 0; k < V; ++k) acc[k] *= s.scale;
        store_values<V>(out + (int64_t)key * out_ld + col, acc);
    }
}

// Rows of zeros, for the gradient of no tokens at all.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void k_zero_rows(O* out, int64_t out_ld, int64_t rows, int dim, int pieces) {
    const float zero[V] = {};
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < rows * pieces; at += (int64_t)gridDim.x * kBlock) {
        const int64_t r = at / pieces;
        store_values<V>(out + r * out_ld + piece_column<V>((int)(at - r * pieces), dim), zero);
    }
}

// Zeros in the rows of ids that do not occur.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void k_zero_absent(const uint8_t* present, O* out, int64_t out_ld, int64_t rows, int dim) {
    const int64_t first = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kWave * kWave, mine = first + lane_id();
    zero_rows_of_wave<O, V>(mine < rows && !present[mine], first, out, out_ld, dim);
}

// ---- stable radix sort of (id, item, weight) by id -------------------------------------------------------------------
//
// Digits of up to ten bits: two passes for tables of up to a million rows.  A pass reads and writes the list once (12 bytes an entry with
// weights) and once more the keys, to count.  8.4M tokens, a million rows: 267 us for both passes, of which 139 and 77 are the scatters (of 200 MB,
// 44 us as a copy): a tile has eight entries of a digit, 32 bytes, side by side in the first pass, and long runs in the second,
// where few digits hold most.  Three passes of seven bits took 310 us; 1,024 threads per tile 153 and 83 us for the scatters.

constexpr int kSortBlock = 512;
// Entries per thread.  A long list in tiles of 8,192 has eight of each digit to a tile on average, which are written side by side; a short one in tiles
// of 2,048 has four times the workgroups.
constexpr int kLongItems = 16, kShortItems = 4;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kDigitBits = 10;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kClear = kSortBlock * 16;               // bytes a workgroup clears

struct SortPass {
    const int32_t* key;  // NULL in the first pass: ids are read from the list
    const int32_t* src;
    const float* factor;
    int32_t* key_out;
    int32_t* src_out;
    float* factor_out;   // NULL without weights
    uint32_t* hist;      // [tile][digit]
    uint32_t* totals;    // [digit]
    int tiles;
    int shift, bits;
    __device__ inline uint32_t digit(int32_t k) const { return ((uint32_t)k >> shift) & ((1u << bits) - 1); }
};

// Ids that contribute nothing sort behind all others.
__device__ inline int32_t sort_key(const TokenList& t, const SortPass& p, int64_t i) {
    if (p.key) return p.key[i];
    const int32_t id = t.id(i);
    return id < 0 ? (int32_t)t.limit : id;
}

// The blocks behind those of the tiles (first pass) clear the notes of which ids occur.
template <int N>
__global__ __launch_bounds__(kSortBlock) void k_sort_count(TokenList t, SortPass p, uint8_t* present) {
    constexpr int kTile = N * kSortBlock;
    if ((int)blockIdx.x >= p.tiles) {
        const int64_t at = ((int64_t)blockIdx.x - p.tiles) * kClear + threadIdx.x * 16;
        if (at < t.limit) *reinterpret_cast<u32x4*>(present + at) = u32x4{0u, 0u, 0u, 0u};  // its end is padded to 256 bytes
        return;
    }
    __shared__ uint32_t count[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortBlock) count[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile;
    int32_t key[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t i = first + k * kSortBlock + threadIdx.x;
        key[k] = -1;
        if (i < t.count) {
            if (p.key) {
                key[k] = p.key[i];
            } else {
                bool bad;
                key[k] = t.id(i, &bad);
                count_rejected(t.rejected, bad);
                if (key[k] < 0) key[k] = (int32_t)t.limit;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (key[k] >= 0) atomicAdd(&count[p.digit(key[k])], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << p.bits; d += kSortBlock) p.hist[(int64_t)blockIdx.x * kDigits + d] = count[d];
}

// One workgroup for 32 digits: where each tile's entries of a digit begin among all of that digit, and how many there are.  32 threads share a digit's tiles.
constexpr int kOffsetDigits = 32, kOffsetParts = 32;
__global__ __launch_bounds__(kOffsetDigits * kOffsetParts) void k_sort_offsets(SortPass p) {
    __shared__ uint32_t sums[kOffsetParts][kOffsetDigits + 1];
    const int d = threadIdx.x % kOffsetDigits, part = threadIdx.x / kOffsetDigits;
    uint32_t* h = p.hist + blockIdx.x * kOffsetDigits + d;
    const int per = (p.tiles + kOffsetParts - 1) / kOffsetParts;
    const int from = min(part * per, p.tiles), to = min(from + per, p.tiles);
    uint32_t sum = 0;
#pragma unroll 8
    for (int t = from; t < to; ++t) sum += h[(int64_t)t * kDigits];
    sums[part][d] = sum;
    __syncthreads();
    uint32_t run = 0;
    for (int k = 0; k < part; ++k) run += sums[k][d];
    if (part == kOffsetParts - 1) p.totals[blockIdx.x * kOffsetDigits + d] = run + sum;
#pragma unroll 8
    for (int t = from; t < to; ++t) {
        const uint32_t v = h[(int64_t)t * kDigits];
        h[(int64_t)t * kDigits] = run;
        run += v;
    }
}

// Each wave ranks its 64 N consecutive entries 64 at a time among those of the same digit (lanes of one digit are found by a ballot
// per bit), the ranks are made the tile's, and keys, sources and factors are put in order in shared memory, one after the other in the same space, and
// written out as runs.
template <int N>
__global__ __launch_bounds__(kSortBlock) void k_sort_scatter(TokenList t, SortPass p) {
    constexpr int kTile = N * kSortBlock;
    __shared__ uint16_t count[kSortWaves][kDigits];
    __shared__ uint32_t to[kDigits];  // place of a digit's entries of this tile in the output, less their place in the tile
    __shared__ uint32_t smem[kSortWaves + 1];
    __shared__ int32_t range[kTileRange];
    __shared__ int32_t order[kTile];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t first = (int64_t)blockIdx.x * kTile;
    const int n = (int)min((int64_t)kTile, t.count - first);
    for (int k = threadIdx.x; k < kSortWaves * kDigits / 2; k += kSortBlock) reinterpret_cast<uint32_t*>(count)[k] = 0;
    const int mine = wave * (kTile / kSortWaves) + lane;  // entry mine + 64 r of the tile
    int32_t key[N], src[N];
    uint32_t rank[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int at = mine + r * kWave;
        key[r] = at < n ? sort_key(t, p, first + at) : 0;
        if (p.key) src[r] = at < n ? p.src[first + at] : 0;
    }
    if (!p.key) {
        if (t.offsets) tile_items<kTile, kSortBlock>(t, first, n, order, range);
#pragma unroll
        for (int r = 0; r < N; ++r) {
            const int at = mine + r * kWave;
            src[r] = t.offsets ? order[at] : (int32_t)(first + at);
            if (src[r] >= t.items) src[r] = -1;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const bool in = mine + r * kWave < n;
        const uint32_t d = p.digit(key[r]);
        unsigned long long same = __ballot(in);
        for (int b = 0; b < p.bits; ++b) {
            const unsigned long long one = __ballot(d >> b & 1);
            same &= (d >> b & 1) ? one : ~one;
        }
        // every lane of a digit reads its count, then the first writes it back: a wave's accesses to shared memory are in order
        const uint32_t base = count[wave][d];
        rank[r] = base + (uint32_t)__popcll(same & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (in && lane == __ffsll(same) - 1) count[wave][d] = (uint16_t)(base + (uint32_t)__popcll(same));
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    {
        // two neighbouring digits per thread
        static_assert(kDigits == 2 * kSortBlock, "two digits per thread");
        const uint32_t d = 2 * threadIdx.x;
        uint32_t sum[2] = {0, 0}, all[2];
        for (int k = 0; k < kSortWaves; ++k)
            for (int e = 0; e < 2; ++e) sum[e] += count[k][d + e];
        for (int e = 0; e < 2; ++e) all[e] = d + e < 1u << p.bits ? p.totals[d + e] : 0u;
        uint32_t ignored;
        uint32_t begin = block_exclusive_scan<uint32_t, kSortBlock>(sum[0] + sum[1], smem, &ignored);
        uint32_t at = block_exclusive_scan<uint32_t, kSortBlock>(all[0] + all[1], smem, &ignored);
        for (int e = 0; e < 2; ++e) {
            to[d + e] = at + (d + e < 1u << p.bits ? p.hist[(int64_t)blockIdx.x * kDigits + d + e] : 0u) - begin;
            for (int k = 0; k < kSortWaves; ++k) {
                const uint32_t v = count[k][d + e];
                count[k][d + e] = (uint16_t)begin;
                begin += v;
            }
            at += all[e];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r) {
        rank[r] += count[wave][p.digit(key[r])];
        if (mine + r * kWave < n) order[rank[r]] = key[r];
    }
    __syncthreads();
    uint32_t place[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int at = (int)threadIdx.x + r * kSortBlock;
        const int32_t k = at < n ? order[at] : 0;
        place[r] = to[p.digit(k)] + (uint32_t)at;
        if (at < n) p.key_out[place[r]] = k;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (mine + r * kWave < n) order[rank[r]] = src[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int at = (int)threadIdx.x + r * kSortBlock;
        if (at < n) p.src_out[place[r]] = order[at];
    }
    if (!p.factor_out) return;
    __syncthreads();
    const float* factor = p.key ? p.factor : t.weights;
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (mine + r * kWave < n) order[rank[r]] = __float_as_int(factor[first + mine + r * kWave]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int at = (int)threadIdx.x + r * kSortBlock;
        if (at < n) p.factor_out[place[r]] = __int_as_float(order[at]);
    }
}

}  // namespace dynlp
