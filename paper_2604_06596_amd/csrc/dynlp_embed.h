// Rows of items from a table of token rows, and the table's gradient.
//
// Both directions are one sum over a list of (key, source, factor) sorted by key:
//     out[key] = scale * sum of factor * rows[source]
// Forward the key is the item of a token and the source its id (the list is in order as it stands); backward the key is the id
// (the list is sorted by a stable radix sort) and the source the item.  Each row of `rows` is read once per token, from the
// caches as far as they hold it, and each row of `out` is written once.
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

// ---- one row per token -----------------------------------------------------------------------------------------------

// out[i] = scale * weight * table[id]: a copy with a factor.  One 16-byte piece per thread; `pieces` of them make a row.
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_embed_rows(TokenList t, const T* table, int64_t ld, T* out, int64_t out_ld, int dim,
                                                       int pieces) {
    const int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    const int64_t i = at / pieces;
    if (i >= t.count) return;
    const int c = (int)(at - i * pieces);
    const int col = piece_column<V>(c, dim);
    bool bad;
    const int32_t id = t.id(i, &bad);
    if (bad && c == 0 && t.rejected) atomicAdd(t.rejected, 1);
    float f[V] = {};
    if (id >= 0) {
        Lane<T, V> x;
        x.load(table + (int64_t)id * ld + col);
        x.get(f);
        const float s = t.weights ? t.scale * t.weights[i] : t.scale;
        for (int k = 0; k < V; ++k) f[k] *= s;
    }
    store_values<V>(out + i * out_ld + col, f);
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

template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_embed_items(TokenList t, const T* table, int64_t ld, T* out, int64_t out_ld, int dim,
                                                        int lanes_log2) {
    const int64_t b = blockIdx.x;
    int64_t begin, end;
    t.bounds(b, &begin, &end);
    for (int64_t i = begin + threadIdx.x; i < end; i += kBlock) {
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
        t.scale, out + b * out_ld);
}

constexpr int kFewTokens = 8192;     // list entries one workgroup can hold: 32 per thread
constexpr int kZeroRows = 8192;      // rows whose presence one workgroup notes at most

// The gradient for few tokens, without a sort: workgroup i looks through all ids; if token i is the first with its id it lists the
// others, in order, and adds their rows up.  The workgroups behind those zero the rows of ids that do not occur.
template <typename T, typename O, int V>
__global__ __launch_bounds__(kBlock) void k_embed_grad_few(TokenList t, const T* grad, int64_t ld, O* out, int64_t out_ld, int dim,
                                                           int lanes_log2, int zero_rows) {
    __shared__ int32_t list[kFewTokens];
    __shared__ uint32_t smem[kBlock / kWave + 1];
    const int n = (int)t.count;
    if ((int64_t)blockIdx.x < t.count) {
        const int me = (int)blockIdx.x;
        bool bad;
        const int32_t id = t.id(me, &bad);
        if (bad && threadIdx.x == 0 && t.rejected) atomicAdd(t.rejected, 1);
        if (id < 0) return;
        const int per = (n + kBlock - 1) / kBlock;
        uint32_t hits = 0;
        bool earlier = false;
        for (int k = 0; k < per; ++k) {
            const int i = (int)threadIdx.x * per + k;
            if (i < n && t.id(i) == id) {
                hits |= 1u << k;
                earlier |= i < me;
            }
        }
        if (__syncthreads_or(earlier)) return;
        uint32_t total;
        uint32_t at = block_exclusive_scan<uint32_t>((uint32_t)__popc(hits), smem, &total);
        for (int k = 0; k < per; ++k)
            if (hits >> k & 1) list[at++] = (int)threadIdx.x * per + k;
        __syncthreads();
        block_sum<T, O, V>(
            grad, ld, dim, lanes_log2, total,
            [&](int64_t i, float* w) -> int64_t {
                const int pos = list[i];
                *w = t.weights ? t.weights[pos] : 1.f;
                return t.item(pos);
            },
            t.scale, out + (int64_t)id * out_ld);
        return;
    }
    uint32_t* present = reinterpret_cast<uint32_t*>(list);
    const int64_t first = ((int64_t)blockIdx.x - t.count) * zero_rows;
    const int rows = (int)min((int64_t)zero_rows, t.limit - first);
    for (int k = threadIdx.x; k < (zero_rows + 31) / 32; k += kBlock) present[k] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kBlock) {
        const int64_t r = (int64_t)t.id(i) - first;
        if (r >= 0 && r < rows) atomicOr(&present[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    const int pieces = (dim + V - 1) / V;
    float zero[V] = {};
    for (int64_t at = threadIdx.x; at < (int64_t)rows * pieces; at += kBlock) {
        const int r = (int)(at / pieces), c = (int)(at - (int64_t)r * pieces);
        if (!(present[r >> 5] >> (r & 31) & 1)) store_values<V>(out + (first + r) * out_ld + piece_column<V>(c, dim), zero);
    }
}

// ---- long lists: sums over pieces of the list, joined ----------------------------------------------------------------

// key[i] = the item of token i (-1: none), src[i] = its id (-1: contributes nothing); the blocks behind those of the tokens zero the rows of items
// without tokens.
constexpr int kKeyTile = 1024;
template <typename T, int V>
__global__ __launch_bounds__(kBlock) void k_item_keys(TokenList t, int32_t* key, int32_t* src, int token_blocks, T* out,
                                                      int64_t out_ld, int dim) {
    if ((int)blockIdx.x < token_blocks) {
        __shared__ int64_t range[2];
        const int64_t first = (int64_t)blockIdx.x * kKeyTile;
        const int64_t last = min(first + kKeyTile, t.count) - 1;
        if (threadIdx.x < 2) range[threadIdx.x] = t.item_from(threadIdx.x ? last : first, -1, t.items);
        __syncthreads();
        const int64_t lo = range[0], hi = max(range[1], lo);
        for (int64_t i = first + threadIdx.x; i <= last; i += kBlock) {
            const int64_t b = t.item_from(i, lo, hi);
            key[i] = b < t.items ? (int32_t)b : -1;
            bool bad;
            src[i] = t.id(i, &bad);
            count_rejected(t.rejected, bad);
        }
        return;
    }
    const int64_t wave = ((int64_t)blockIdx.x - token_blocks) * (kBlock / kWave) + threadIdx.x / kWave;
    const int64_t mine = wave * kWave + lane_id();
    bool empty = false;
    if (mine < t.items) {
        int64_t begin, end;
        t.bounds(mine, &begin, &end);
        empty = begin == end;
    }
    float zero[V] = {};
    const int pieces = (dim + V - 1) / V;
    for (unsigned long long m = __ballot(empty); m; m &= m - 1) {
        T* row = out + (wave * kWave + __ffsll(m) - 1) * out_ld;
        for (int c = lane_id(); c < pieces; c += kWave) store_values<V>(row + piece_column<V>(c, dim), zero);
    }
}

enum : uint8_t {
    kHead = 1,     // the piece's first run began before it; its sum is head[piece]
    kThrough = 2,  // and goes on behind it
    kOpen = 4      // the piece's last run began in it and goes on behind it; its sum is tail[piece]
};

struct SumList {
    const int32_t* key;    // ascending; a key outside [0, out_rows) is written nowhere
    const int32_t* src;    // a source outside [0, row_count) contributes nothing
    const float* factor;   // or NULL
    float* part;           // [piece][head, tail][dim]
    uint8_t* flags;        // [piece]
    int64_t count;
    int64_t row_count, out_rows;
    int piece;             // entries of a piece of the list, a multiple of 8
    float scale;
};

// A group of lanes goes through one piece of the list with a running sum; lanes are across the columns (blockIdx.y: 2^lanes_log2 lane
// columns each).  Eight rows are asked for at a time.  Runs that lie within the piece are written to `out`, the first and the last, where
// they go on beyond it, to `part`.
template <typename T, typename O, int V>
__global__ __launch_bounds__(kBlock) void k_segment_sum(SumList s, const T* rows, int64_t ld, O* out, int64_t out_ld, int dim,
                                                        int lanes_log2) {
    const int64_t g = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lanes_log2;
    const int lane = threadIdx.x & ((1 << lanes_log2) - 1);
    const int c = ((int)blockIdx.y << lanes_log2) + lane;
    const int64_t first = g * s.piece;
    if (first >= s.count || c * V >= dim + V - 1 || (V > 1 && c * V >= dim)) return;
    const int col = piece_column<V>(c, dim);
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
        } else if (cur >= 0 && cur < s.out_rows) {
            float f[V];
            for (int k = 0; k < V; ++k) f[k] = acc[k] * s.scale;
            store_values<V>(out + (int64_t)cur * out_ld, f);
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
        flags |= kOpen;
    } else {
        flush();
    }
    if (c == 0) s.flags[g] = flags;
}

// Runs that several pieces share: the wave of the piece in which such a run begins adds up its parts, in their order within each group of
// lanes, then the groups'.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void k_segment_join(SumList s, int64_t pieces, O* out, int64_t out_ld, int dim, int lanes_log2) {
    const int64_t p = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / kWave;
    if (p >= pieces || !(s.flags[p] & kOpen)) return;
    const int32_t key = s.key[(p + 1) * s.piece - 1];
    if (key < 0 || key >= s.out_rows) return;
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

// Rows of zeros, for the gradient of ids that do not occur.
template <typename O, int V>
__global__ __launch_bounds__(kBlock) void k_zero_rows(O* out, int64_t out_ld, int64_t rows, int dim, int pieces) {
    const float zero[V] = {};
    for (int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x; at < rows * pieces; at += (int64_t)gridDim.x * kBlock) {
        const int64_t r = at / pieces;
        store_values<V>(out + r * out_ld + piece_column<V>((int)(at - r * pieces), dim), zero);
    }
}

// ---- stable radix sort of (id, item, weight) by id -------------------------------------------------------------------

constexpr int kSortTile = 4096;                       // entries per workgroup
constexpr int kSortItems = kSortTile / kBlock;        // per thread
constexpr int kDigits = 256;

struct SortPass {
    const int32_t* key;  // NULL in the first pass: ids are read from the list
    const int32_t* src;
    const float* factor;
    int32_t* key_out;
    int32_t* src_out;
    float* factor_out;   // NULL without weights
    uint32_t* hist;      // [digit][tile]
    uint32_t* totals;    // [digit]
    int tiles;
    int shift, bits;
};

// Ids that contribute nothing sort behind all others.
__device__ inline int32_t sort_key(const TokenList& t, const SortPass& p, int64_t i) {
    if (p.key) return p.key[i];
    const int32_t id = t.id(i);
    return id < 0 ? (int32_t)t.limit : id;
}

__global__ __launch_bounds__(kBlock) void k_sort_count(TokenList t, SortPass p) {
    __shared__ uint32_t count[kDigits];
    count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortTile;
    const uint32_t mask = (1u << p.bits) - 1;
    for (int k = 0; k < kSortItems; ++k) {
        const int64_t i = first + k * kBlock + threadIdx.x;
        if (i < t.count) {
            if (!p.key) {
                bool bad;
                t.id(i, &bad);
                count_rejected(t.rejected, bad);
            }
            atomicAdd(&count[((uint32_t)sort_key(t, p, i) >> p.shift) & mask], 1u);
        }
    }
    __syncthreads();
    if (threadIdx.x <= mask) p.hist[(int64_t)threadIdx.x * p.tiles + blockIdx.x] = count[threadIdx.x];
}

// One workgroup per digit: where each tile's entries of it begin among all of that digit, and how many there are.
__global__ __launch_bounds__(kBlock) void k_sort_offsets(SortPass p) {
    __shared__ uint32_t smem[kBlock / kWave + 1];
    uint32_t* h = p.hist + (int64_t)blockIdx.x * p.tiles;
    uint32_t run = 0;
    for (int at = 0; at < p.tiles; at += kBlock) {
        const int i = at + (int)threadIdx.x;
        const uint32_t v = i < p.tiles ? h[i] : 0u;
        uint32_t total;
        const uint32_t ex = block_exclusive_scan<uint32_t>(v, smem, &total);
        if (i < p.tiles) h[i] = run + ex;
        run += total;
    }
    if (threadIdx.x == 0) p.totals[blockIdx.x] = run;
}

// Each wave ranks its 1,024 consecutive entries 64 at a time among those of the same digit (lanes of one digit are found by a ballot
// per bit), the ranks are made the tile's, the entries are put in order in shared memory and written out as runs.
__global__ __launch_bounds__(kBlock) void k_sort_scatter(TokenList t, SortPass p) {
    constexpr int kWaves = kBlock / kWave;
    __shared__ uint32_t count[kWaves][kDigits];
    __shared__ uint32_t begin[kDigits];  // of each digit within the tile
    __shared__ uint32_t to[kDigits];     // of each digit's entries of this tile in the output
    __shared__ uint32_t smem[kWaves + 1];
    __shared__ int32_t keys[kSortTile], srcs[kSortTile];
    __shared__ float factors[kSortTile];
    __shared__ int64_t range[2];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const uint32_t mask = (1u << p.bits) - 1;
    const int64_t first = (int64_t)blockIdx.x * kSortTile;
    const int n = (int)min((int64_t)kSortTile, t.count - first);
    for (int k = 0; k < kWaves; ++k) count[k][threadIdx.x] = 0;
    if (!p.key && t.offsets && threadIdx.x < 2) range[threadIdx.x] = t.item_from(threadIdx.x ? first + n - 1 : first, -1, t.items);
    __syncthreads();
    int32_t key[kSortItems];
    uint32_t rank[kSortItems];
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
        const int at = wave * (kSortTile / kWaves) + r * kWave + lane;
        const bool in = at < n;
        key[r] = in ? sort_key(t, p, first + at) : 0;
        const uint32_t d = ((uint32_t)key[r] >> p.shift) & mask;
        unsigned long long same = __ballot(in);
        for (int b = 0; b < p.bits; ++b) {
            const unsigned long long one = __ballot(d >> b & 1);
            same &= (d >> b & 1) ? one : ~one;
        }
        const int leader = in ? __ffsll(same) - 1 : lane;
        uint32_t base = 0;
        if (in && lane == leader) base = atomicAdd(&count[wave][d], (uint32_t)__popcll(same));
        base = __shfl(base, leader, kWave);
        rank[r] = base + (uint32_t)__popcll(same & ((1ull << lane) - 1));
    }
    __syncthreads();
    {
        const uint32_t d = threadIdx.x;
        uint32_t sum = 0;
        for (int k = 0; k < kWaves; ++k) {
            const uint32_t v = count[k][d];
            count[k][d] = sum;
            sum += v;
        }
        uint32_t ignored;
        begin[d] = block_exclusive_scan<uint32_t>(sum, smem, &ignored);
        const uint32_t all = block_exclusive_scan<uint32_t>(d <= mask ? p.totals[d] : 0u, smem, &ignored);
        to[d] = all + (d <= mask ? p.hist[(int64_t)d * p.tiles + blockIdx.x] : 0u);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
        const int at = wave * (kSortTile / kWaves) + r * kWave + lane;
        if (at < n) {
            const uint32_t d = ((uint32_t)key[r] >> p.shift) & mask;
            const uint32_t pos = begin[d] + count[wave][d] + rank[r];
            keys[pos] = key[r];
            if (p.key) {
                srcs[pos] = p.src[first + at];
                if (p.factor_out) factors[pos] = p.factor[first + at];
            } else {
                const int64_t i = first + at;
                int64_t b = i;
                if (t.offsets) {
                    b = t.item_from(i, range[0], max(range[0], range[1]));
                    if (b >= t.items) b = -1;
                }
                srcs[pos] = (int32_t)b;
                if (p.factor_out) factors[pos] = t.weights[i];
            }
        }
    }
    __syncthreads();
    for (int at = threadIdx.x; at < n; at += kBlock) {
        const uint32_t d = ((uint32_t)keys[at] >> p.shift) & mask;
        const uint32_t pos = to[d] + (uint32_t)at - begin[d];
        p.key_out[pos] = keys[at];
        p.src_out[pos] = srcs[at];
        if (p.factor_out) p.factor_out[pos] = factors[at];
    }
}

}  // namespace dynlp
