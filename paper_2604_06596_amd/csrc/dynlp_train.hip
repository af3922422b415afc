// libdynlp: host side of the student's operators (include/dynlp_train.h): checks, launch sizes, C ABI.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <numeric>
#include <string>

#include "dynlp_train.h"
#include "dynlp_adamw.h"
#include "dynlp_embed.h"
#include "dynlp_head.h"

namespace dynlp {
std::string& thread_error();  // what dynlp_last_error(NULL) returns; dynlp.hip
}

using namespace dynlp;

namespace {

static_assert(kStateBlock == DYNLP_STATE_BLOCK, "one block length");
static_assert(16 * kMaxTiles == DYNLP_MAX_CLASSES, "class tiles cover the classes");

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

__attribute__((format(printf, 2, 3))) dynlp_status fail(dynlp_status status, const char* format, ...) {
    char text[256];
    va_list args;
    va_start(args, format);
    std::vsnprintf(text, sizeof text, format, args);
    va_end(args);
    try {
        thread_error() = text;
    } catch (...) {  // no memory for the message
    }
    return status;
}

#define REFUSE(...) return fail(DYNLP_ERR_INVALID_ARG, __VA_ARGS__)

dynlp_status launched() {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? DYNLP_OK : fail(DYNLP_ERR_DEVICE, "kernel launch failed: %s", hipGetErrorString(e));
}

constexpr int64_t kMostRows = 0x7ffffffe;
constexpr int32_t kMostDim = 1 << 28;  // 32 bits hold the bytes of a row

int type_size(int32_t type) { return type == DYNLP_FLOAT32 ? 4 : 2; }

dynlp_status check_matrix(const dynlp_matrix* m, const char* name) {
    if (!m) REFUSE("%s is NULL", name);
    if (m->type < DYNLP_FLOAT32 || m->type > DYNLP_FLOAT16) REFUSE("%s: type %d is not a dynlp_type", name, m->type);
    if (m->rows < 0 || m->rows > kMostRows) REFUSE("%s: %lld rows", name, (long long)m->rows);
    if (m->dim < 1 || m->dim > kMostDim) REFUSE("%s: rows of %d elements", name, m->dim);
    if (m->stride < m->dim) REFUSE("%s: stride %lld is less than the %d elements of a row", name, (long long)m->stride, m->dim);
    if (m->stride > (int64_t(1) << 40)) REFUSE("%s: stride %lld", name, (long long)m->stride);
    if (m->rows > 0 && !m->data) REFUSE("%s: data is NULL", name);
    if (reinterpret_cast<uintptr_t>(m->data) % type_size(m->type)) REFUSE("%s: data is not aligned to its elements", name);
    return DYNLP_OK;
}

dynlp_status check_tokens(const dynlp_tokens* t) {
    if (!t) REFUSE("tokens is NULL");
    if (t->count < 0 || t->count > kMostRows) REFUSE("%lld tokens", (long long)t->count);
    if (t->items < 0 || t->items > kMostRows) REFUSE("%lld items", (long long)t->items);
    if (t->count > 0 && !t->ids) REFUSE("ids is NULL");
    if (!t->offsets && t->items != t->count) REFUSE("without offsets every token is an item: %lld items, %lld tokens", (long long)t->items, (long long)t->count);
    return DYNLP_OK;
}

#define CHECK(call)                            \
    do {                                       \
        const dynlp_status s_ = (call);        \
        if (s_ != DYNLP_OK) return s_;         \
    } while (0)

dynlp_status check_workspace(const dynlp_call* call, int64_t bytes) {
    if (!call) REFUSE("call is NULL");
    if (bytes > 0 && (!call->workspace || call->workspace_bytes < bytes))
        REFUSE("workspace of %lld bytes: %lld are needed", (long long)(call->workspace ? call->workspace_bytes : 0), (long long)bytes);
    if (bytes > 0 && reinterpret_cast<uintptr_t>(call->workspace) % 256) REFUSE("workspace is not aligned to 256 bytes");
    return DYNLP_OK;
}

// Whether rows of a and rows of b share memory.  Rows of two matrices may take turns in one array; where their strides differ, matrices whose rows
// would meet if there were enough of them count as overlapping.
bool overlap(const dynlp_matrix& a, const dynlp_matrix& b) {
    using wide = __int128;  // rows times stride
    if (a.rows == 0 || b.rows == 0) return false;
    const wide width_a = (wide)a.dim * type_size(a.type), width_b = (wide)b.dim * type_size(b.type);
    wide step_a = (wide)a.stride * type_size(a.type), step_b = (wide)b.stride * type_size(b.type);
    const wide behind = (wide) reinterpret_cast<uintptr_t>(b.data) - (wide) reinterpret_cast<uintptr_t>(a.data);
    if (behind >= (a.rows - 1) * step_a + width_a || -behind >= (b.rows - 1) * step_b + width_b) return false;
    if (a.rows == 1) step_a = step_b;
    if (b.rows == 1) step_b = step_a;
    if (step_a != step_b) {
        const wide step = std::gcd((int64_t)step_a, (int64_t)step_b), at = (behind % step + step) % step;
        return at < width_a || at + width_b > step;
    }
    // row i of a and row i + k of b meet where -width_b < behind + k step < width_a
    auto down = [&](wide x) { return (x >= 0 ? x : x - step_a + 1) / step_a; };
    const wide least = -down(width_b - 1 + behind), most = down(width_a - 1 - behind);
    return std::max(least, (wide)(1 - a.rows)) <= std::min(most, (wide)(b.rows - 1));
}

// Hands out the parts of a workspace, or only measures them (base NULL).
struct Carve {
    char* base;
    int64_t used = 0;
    template <typename T>
    T* take(int64_t n) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += round_up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

// The type as a value, and pieces of 16 bytes where a row has one: F is called with (T(), integral V).
template <int V>
struct Width {
    static constexpr int v = V;
};
template <typename F>
void by_type(int32_t type, int dim, F f) {
    if (type == DYNLP_FLOAT32) {
        if (dim >= 4) f(float(), Width<4>());
        else f(float(), Width<1>());
    } else if (type == DYNLP_BFLOAT16) {
        if (dim >= 8) f(bf16(), Width<8>());
        else f(bf16(), Width<1>());
    } else {
        if (dim >= 8) f(f16(), Width<8>());
        else f(f16(), Width<1>());
    }
}

// Lanes across the columns of a row: a power of two, a wave at most.
int lanes_log2(int pieces) {
    int l = 0;
    while (l < 6 && (1 << l) < pieces) ++l;
    return l;
}

constexpr int64_t kMostBlocks = 0xffffffff / kBlock;    // workgroups: a launch has fewer than 2^32 threads
constexpr int64_t kHalfCache = int64_t(128) << 20;  // half the 256 MB before the memory

// ---- embedding --------------------------------------------------------------------------------------------------------

constexpr int64_t kFewPerItem = 2048;  // tokens up to which each item has a workgroup

// Whether items have pieces of the list rather than a workgroup each: long lists, and more items than a launch has workgroups.
bool in_pieces(int64_t count, int64_t items) { return count > kFewPerItem || (count > 0 && items > kMostBlocks); }

// Rows of 256 bytes and more have waves of their own (k_wave_sum).
bool wide_rows(int32_t type, int dim) { return (int64_t)dim * type_size(type) >= 256; }

// Entries of a piece of the list.  Pieces enough for 8,192 to 16,384 waves, or groups of lanes for as many as 8,192 waves, where the list has so many entries
// (5 to 8 waves of k_wave_sum fit each of 1,024 SIMDs, by its registers); not so few entries that the two parts a piece may leave weigh much against the
// rows it reads, and not above 512, so that a run over many pieces is joined soon.
int piece_length(int64_t count, int dim, bool wide) {
    const int64_t lanes = std::min<int64_t>(ceil_div(dim, 8), 64);
    if (wide) {
        const int64_t n = ceil_div(count, 16384);
        return n <= 16 ? 16 : n <= 32 ? 32 : (int)std::min<int64_t>(round_up(n, 64), 512);
    }
    return (int)std::min<int64_t>(std::max<int64_t>(round_up(ceil_div(count * lanes, 8192 * 64), 8), 16), 512);
}

struct SumSpace {
    int32_t *key, *src;
    float* factor;
    int32_t *key2, *src2;
    float* factor2;
    uint32_t *hist, *totals;
    float* part;
    uint8_t *flags, *present;
    int32_t* open;
    int piece, items;  // of a piece of the list; of a thread in a sort
    int64_t pieces, tiles;
};

// sorted: rows of the gradient that is asked for, or -1.
int64_t sum_space(char* base, int64_t count, int dim, bool wide, int64_t sorted, SumSpace* s) {
    Carve c{base};
    s->piece = piece_length(count, dim, wide);
    s->pieces = ceil_div(count, s->piece);
    s->items = count < (int64_t(1) << 18) ? kShortItems : kLongItems;
    s->tiles = ceil_div(count, s->items * kSortBlock);
    if (sorted >= 0 || !wide) {
        s->key = c.take<int32_t>(count);
        s->src = c.take<int32_t>(count);
    }
    if (sorted >= 0) {
        s->factor = c.take<float>(count);
        s->key2 = c.take<int32_t>(count);
        s->src2 = c.take<int32_t>(count);
        s->factor2 = c.take<float>(count);
        s->hist = c.take<uint32_t>(kDigits * s->tiles);
        s->totals = c.take<uint32_t>(kDigits);
        s->present = c.take<uint8_t>(sorted);
    }
    s->part = c.take<float>(s->pieces * 2 * dim);
    s->flags = c.take<uint8_t>(s->pieces);
    s->open = c.take<int32_t>(s->pieces);
    return c.used;
}

// Whatever the type: rows of dim elements may be wide or not.
int64_t sum_space_bytes(int64_t count, int dim, int64_t sorted) {
    SumSpace s{};
    const int64_t narrow = wide_rows(DYNLP_BFLOAT16, dim) ? 0 : sum_space(nullptr, count, dim, false, sorted, &s);
    const int64_t wide = wide_rows(DYNLP_FLOAT32, dim) ? sum_space(nullptr, count, dim, true, sorted, &s) : 0;
    return std::max(narrow, wide);
}

TokenList token_list(const dynlp_tokens* t, int64_t table_rows) {
    return TokenList{t->ids, t->offsets, t->weights, t->rejected, t->count, t->items, table_rows, t->scale, t->ids_are_64 != 0};
}

template <typename T, typename O, int V>
void launch_narrow(const SumList& s, const T* rows, int64_t ld, O* out, int64_t out_ld, int dim, hipStream_t stream) {
    const int l = lanes_log2((int)ceil_div(dim, V));
    const int64_t n = ceil_div(s.count, s.piece);
    k_segment_sum<T, O, V><<<(unsigned)ceil_div(n << l, kBlock), kBlock, 0, stream>>>(s, rows, ld, out, out_ld, dim, l);
    k_segment_join<O, V><<<(unsigned)ceil_div(n * kWave, kBlock), kBlock, 0, stream>>>(s, n, out, out_ld, dim, l);
}

// A lane takes as many columns as a row needs for 64 lanes, 4 to 16 bytes of them.
template <typename T, typename O, bool ITEMS, bool PAST>
void launch_wide(const SumList& s, const TokenList& t, const T* rows, int64_t ld, O* out, int64_t out_ld, int dim, hipStream_t stream) {
    const int64_t n = ceil_div(s.count, s.piece), blocks = ceil_div(n, kBlock / kWave);
    const unsigned grid = (unsigned)(blocks + (ITEMS ? ceil_div(t.items, kBlock) : 0));
    constexpr int e = 4 / (int)sizeof(T);
    auto sum = [&](auto width) {
        constexpr int E = decltype(width)::v;
        k_wave_sum<T, O, E, ITEMS, PAST><<<dim3(grid, (unsigned)ceil_div(dim, kWave * E)), kBlock, 0, stream>>>(s, t, rows, ld, out, out_ld, dim, (int)blocks);
    };
    if (dim <= kWave * e) sum(Width<e>());
    else if (dim <= kWave * 2 * e) sum(Width<2 * e>());
    else sum(Width<4 * e>());
    constexpr int V = Piece<O>::n;
    const int pieces = (int)ceil_div(dim, V), l = lanes_log2(pieces);
    k_segment_join<O, V><<<dim3((unsigned)ceil_div(n * kWave, kBlock), (unsigned)ceil_div(pieces, 1 << l)), kBlock, 0, stream>>>(s, n, out, out_ld, dim, l);
}

// Of a list that nothing else looks at.
dynlp_status launch_count_rejected(const TokenList& t, hipStream_t stream) {
    if (!t.rejected || t.count == 0) return DYNLP_OK;
    k_count_rejected<<<(unsigned)std::min<int64_t>(ceil_div(t.count, kBlock), 1024), kBlock, 0, stream>>>(t);
    return launched();
}

template <typename O>
void launch_zeros(O* out, int64_t out_ld, int64_t rows, int dim, hipStream_t stream) {
    constexpr int P = Piece<O>::n;
    if (dim >= P)
        k_zero_rows<O, P><<<(unsigned)std::min<int64_t>(ceil_div(rows * ceil_div(dim, P), kBlock), 8192), kBlock, 0, stream>>>(
            out, out_ld, rows, dim, (int)ceil_div(dim, P));
    else
        k_zero_rows<O, 1><<<(unsigned)std::min<int64_t>(ceil_div(rows * dim, kBlock), 8192), kBlock, 0, stream>>>(out, out_ld, rows, dim, dim);
}

}  // namespace

extern "C" {

int64_t dynlp_embed_workspace(int64_t count, int64_t items, int32_t dim) {
    if (!in_pieces(count, items) || count > kMostRows || dim < 1) return 0;
    return sum_space_bytes(count, dim, -1);
}

dynlp_status dynlp_embed(const dynlp_matrix* table, const dynlp_tokens* tokens, const dynlp_matrix* out, const dynlp_call* call) {
    CHECK(check_matrix(table, "table"));
    CHECK(check_matrix(out, "out"));
    CHECK(check_tokens(tokens));
    if (out->type != table->type) REFUSE("out has type %d, the table %d", out->type, table->type);
    if (out->dim != table->dim) REFUSE("out has rows of %d elements, the table of %d", out->dim, table->dim);
    if (out->rows != tokens->items) REFUSE("out has %lld rows for %lld items", (long long)out->rows, (long long)tokens->items);
    if (tokens->count > 0 && table->rows == 0) REFUSE("%lld tokens and a table without rows", (long long)tokens->count);
    const bool pieces = tokens->offsets && in_pieces(tokens->count, tokens->items);
    CHECK(check_workspace(call, pieces ? dynlp_embed_workspace(tokens->count, tokens->items, table->dim) : 0));
    if (overlap(*table, *out)) REFUSE("out overlaps the table");
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const TokenList t = token_list(tokens, table->rows);
    if (t.items == 0) return launch_count_rejected(t, stream);
    const int dim = table->dim;
    by_type(table->type, dim, [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int V = decltype(width)::v;
        const T* rows = static_cast<const T*>(table->data);
        T* to = static_cast<T*>(out->data);
        const int64_t n = ceil_div(dim, V);
        if (t.count == 0) {
            launch_zeros(to, out->stride, t.items, dim, stream);
        } else if (!t.offsets) {
            k_embed_rows<T, V><<<(unsigned)ceil_div(t.count * n, kBlock * kRowsAhead), kBlock, 0, stream>>>(t, rows, table->stride, to, out->stride, dim, (int)n);
        } else if (!pieces) {
            k_embed_items<T, V><<<(unsigned)t.items, kBlock, 0, stream>>>(t, rows, table->stride, to, out->stride, dim, lanes_log2((int)n));
        } else {
            SumSpace s{};
            const bool wide = wide_rows(table->type, dim);
            sum_space(static_cast<char*>(call->workspace), t.count, dim, wide, -1, &s);
            const SumList list{s.key, s.src, t.weights, s.part, s.flags, s.open, nullptr, t.count, table->rows, t.items, s.piece, t.scale};
            if (wide) {
                launch_wide<T, T, true, false>(list, t, rows, table->stride, to, out->stride, dim, stream);
            } else {
                const int64_t tiles = ceil_div(t.count, kKeyTile);
                k_item_keys<T, V><<<(unsigned)(tiles + ceil_div(t.items, kBlock)), kBlock, 0, stream>>>(t, s.key, s.src, (int)tiles, to, out->stride, dim);
                launch_narrow<T, T, V>(list, rows, table->stride, to, out->stride, dim, stream);
            }
        }
    });
    return launched();
}

int64_t dynlp_embed_grad_workspace(int64_t count, int64_t items, int32_t dim, int64_t table_rows) {
    (void)items;
    if (count <= kFewTokens || count > kMostRows || dim < 1 || table_rows < 0) return 0;
    return sum_space_bytes(count, dim, table_rows);
}

dynlp_status dynlp_embed_grad(const dynlp_matrix* grad, const dynlp_tokens* tokens, const dynlp_matrix* out, const dynlp_call* call) {
    CHECK(check_matrix(grad, "grad"));
    CHECK(check_matrix(out, "out"));
    CHECK(check_tokens(tokens));
    if (out->type != grad->type && out->type != DYNLP_FLOAT32) REFUSE("out has type %d: float32 or grad's (%d) are possible", out->type, grad->type);
    if (out->dim != grad->dim) REFUSE("out has rows of %d elements, grad of %d", out->dim, grad->dim);
    if (grad->rows != tokens->items) REFUSE("grad has %lld rows for %lld items", (long long)grad->rows, (long long)tokens->items);
    const int64_t count = tokens->items == 0 ? 0 : tokens->count;
    CHECK(check_workspace(call, dynlp_embed_grad_workspace(count, tokens->items, grad->dim, out->rows)));
    if (overlap(*grad, *out)) REFUSE("out overlaps grad");
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const TokenList t = token_list(tokens, out->rows);
    if (count == 0 || out->rows == 0) CHECK(launch_count_rejected(t, stream));
    if (out->rows == 0) return DYNLP_OK;
    const int dim = grad->dim;
    auto run = [&](auto type, auto width, auto out_type) {
        using T = decltype(type);
        using O = decltype(out_type);
        constexpr int V = decltype(width)::v;
        const T* rows = static_cast<const T*>(grad->data);
        O* to = static_cast<O*>(out->data);
        if (count == 0) {
            launch_zeros(to, out->stride, out->rows, dim, stream);
        } else if (count <= kFewTokens) {
            // zero rows: workgroups enough for the chip, 64 rows at least for the look through the ids
            const int zero_rows = (int)std::min<int64_t>(std::max<int64_t>(ceil_div(out->rows, 1024), 64), kZeroRows);
            const int zero_blocks = (int)ceil_div(out->rows, zero_rows);
            k_embed_grad_few<T, O, V><<<(unsigned)(zero_blocks + count), kBlock, 0, stream>>>(t, rows, grad->stride, to, out->stride, dim, zero_rows,
                                                                                             zero_blocks);
        } else {
            SumSpace s{};
            const bool wide = wide_rows(grad->type, dim);
            sum_space(static_cast<char*>(call->workspace), count, dim, wide, out->rows, &s);
            int bits = 1;
            while (bits < 31 && (out->rows >> bits) != 0) ++bits;
            const int passes = (bits + kDigitBits - 1) / kDigitBits, per = (bits + passes - 1) / passes;
            SortPass p{};
            for (int k = 0; k < passes; ++k) {
                const bool even = (k & 1) == 0;
                p.key = k == 0 ? nullptr : even ? s.key2 : s.key;
                p.src = even ? s.src2 : s.src;
                p.factor = even ? s.factor2 : s.factor;
                p.key_out = even ? s.key : s.key2;
                p.src_out = even ? s.src : s.src2;
                p.factor_out = !t.weights ? nullptr : even ? s.factor : s.factor2;
                p.hist = s.hist;
                p.totals = s.totals;
                p.tiles = (int)s.tiles;
                p.shift = k * per;
                p.bits = std::min(per, bits - k * per);
                auto pass = [&](auto items) {
                    constexpr int N = decltype(items)::v;
                    k_sort_count<N><<<(unsigned)(s.tiles + (k == 0 ? ceil_div(out->rows, kClear) : 0)), kSortBlock, 0, stream>>>(t, p, s.present);
                    k_sort_offsets<<<(unsigned)ceil_div(1 << p.bits, kOffsetDigits), kOffsetDigits * kOffsetParts, 0, stream>>>(p);
                    k_sort_scatter<N><<<(unsigned)s.tiles, kSortBlock, 0, stream>>>(t, p);
                };
                if (s.items == kShortItems) pass(Width<kShortItems>());
                else pass(Width<kLongItems>());
            }
            const SumList list{p.key_out, p.src_out, p.factor_out, s.part, s.flags, s.open, s.present, count, t.items, out->rows, s.piece, t.scale};
            // a gradient larger than half the cache is written past it, which then keeps the rows that are read (a million rows of 256 float32: 992 us,
            // 1,050 us through the caches)
            if (wide && out->rows * dim * (int64_t)sizeof(O) > kHalfCache)
                launch_wide<T, O, false, true>(list, t, rows, grad->stride, to, out->stride, dim, stream);
            else if (wide)
                launch_wide<T, O, false, false>(list, t, rows, grad->stride, to, out->stride, dim, stream);
            else
                launch_narrow<T, O, V>(list, rows, grad->stride, to, out->stride, dim, stream);
            constexpr int Z = V == 1 ? 1 : Piece<O>::n;
            k_zero_absent<O, Z><<<(unsigned)ceil_div(out->rows, kBlock), kBlock, 0, stream>>>(s.present, to, out->stride, out->rows, dim);
        }
    };
    by_type(grad->type, dim, [&](auto type, auto width) {
        using T = decltype(type);
        if (out->type == DYNLP_FLOAT32)
            run(type, width, float());
        else
            run(type, width, T());
    });
    return launched();
}

}  // extern "C"

// ---- head -------------------------------------------------------------------------------------------------------------

namespace {

dynlp_status check_head(const dynlp_matrix* h, const dynlp_matrix* weight) {
    CHECK(check_matrix(h, "h"));
    CHECK(check_matrix(weight, "weight"));
    if (weight->type != h->type) REFUSE("weight has type %d, h %d", weight->type, h->type);
    if (weight->dim != h->dim) REFUSE("weight has rows of %d elements, h of %d", weight->dim, h->dim);
    if (weight->rows < 1 || weight->rows > DYNLP_MAX_CLASSES) REFUSE("%lld classes: 1 .. %d are possible", (long long)weight->rows, DYNLP_MAX_CLASSES);
    return DYNLP_OK;
}

Head head_of(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias) {
    return Head{h->data, weight->data, bias, h->stride, weight->stride, h->rows, h->dim, (int)weight->rows};
}

template <int N>
struct Tiles {
    static constexpr int v = N;
};
// F is called with (T(), number of class tiles).
template <typename F>
void by_head(int32_t type, int64_t classes, F f) {
    auto tiles = [&](auto t) {
        switch ((classes + 15) / 16) {
            case 1: f(t, Tiles<1>()); break;
            case 2: f(t, Tiles<2>()); break;
            case 3: f(t, Tiles<3>()); break;
            default: f(t, Tiles<4>());
        }
    };
    if (type == DYNLP_FLOAT32) tiles(float());
    else if (type == DYNLP_BFLOAT16) tiles(bf16());
    else tiles(f16());
}

constexpr int64_t kSharedMemory = 160 * 1024;  // of a CU
constexpr int kMostSharedDim = 1 << 14;        // rows of W that may fit it at all
constexpr int64_t kMostFusedStride = 1 << 22;  // elements: 32 bits hold the bytes of a tile of 128 rows

// Whether one pass over h does all: dweight's columns have a wave each, and W fits a workgroup's shared memory beside dz.
bool fits_fused(int dim, int classes, int32_t type) {
    if (dim > kFusedMost) return false;
    bool fits = false;
    by_head(type, classes, [&](auto t, auto tiles) { fits = fused_bytes<decltype(t), decltype(tiles)::v>(dim) <= kSharedMemory; });
    return fits;
}

struct LossSpace {
    float* dz;
    uint8_t* kept;
    float* part;
    int splits;
    bool fused;
    int64_t per_wave;
};

int64_t loss_space(char* base, int64_t rows, int dim, int classes, int32_t type, bool fused, LossSpace* s) {
    Carve c{base};
    s->fused = fused && fits_fused(dim, classes, type);
    if (s->fused) {
        // at most two workgroups for each CU, all with as many tiles but for the last
        const int64_t tiles = std::max<int64_t>(ceil_div(rows, fused_rows((classes + 15) / 16)), 1);
        s->splits = (int)ceil_div(tiles, ceil_div(tiles, 512));
    } else {
        const int64_t across = ceil_div(dim, 16 * (16 / type_size(type)));
        // workgroups of dweight: twice the CUs over all columns, each wave with 64 rows at least
        s->splits = (int)std::min<int64_t>(std::max<int64_t>(512 / across, 1), std::max<int64_t>(ceil_div(rows, 64 * (kBlock / kWave)), 1));
        s->per_wave = round_up(ceil_div(rows, (int64_t)s->splits * (kBlock / kWave)), 32);
        s->dz = c.take<float>(rows * round_up(classes, 16));
        s->kept = c.take<uint8_t>(rows);
    }
    s->part = c.take<float>((int64_t)s->splits * classes * (dim + 1));
    return c.used;
}

// Shared memory beyond 64 KB is to be asked for, once per kernel and device; `done` has a bit per device (those from the 64th on are asked each time).
template <typename F>
void allow_shared(F kernel, std::atomic<uint64_t>& done) {
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return;  // the launch will say so
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedMemory) == hipSuccess)
        done.fetch_or(bit, std::memory_order_relaxed);
    else
        (void)hipGetLastError();  // the launch will say so
}

}  // namespace

extern "C" {

dynlp_status dynlp_head_labels(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, float* soft, int32_t* hard,
                               const dynlp_call* call) {
    CHECK(check_head(h, weight));
    CHECK(check_workspace(call, 0));
    if (h->rows == 0 || (!soft && !hard)) return DYNLP_OK;
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const Head a = head_of(h, weight, bias);
    by_head(h->type, weight->rows, [&](auto type, auto tiles) {
        using T = decltype(type);
        constexpr int CT = decltype(tiles)::v;
        const int64_t bytes = a.dim <= kMostSharedDim ? shared_bytes<T, CT>(a.dim) : kSharedMemory + 1, blocks = ceil_div(a.rows, kLabelRows);
        // a copy of W pays once a workgroup has several tiles of rows
        const int64_t stay = 256 * std::min<int64_t>(kSharedMemory / bytes, 4);
        if (bytes <= kSharedMemory && blocks >= 2 * stay) {
            static std::atomic<uint64_t> allowed{0};
            allow_shared(k_head_labels<T, CT, true>, allowed);
            k_head_labels<T, CT, true><<<(unsigned)stay, kBlock, (size_t)bytes, stream>>>(a, soft, hard);
        } else {
            k_head_labels<T, CT, false><<<(unsigned)blocks, kBlock, 0, stream>>>(a, soft, hard);
        }
    });
    return launched();
}

int64_t dynlp_head_loss_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t type) {
    if (rows < 0 || rows > kMostRows || dim < 1 || classes < 1 || classes > DYNLP_MAX_CLASSES) return 0;
    LossSpace s;
    return std::max(loss_space(nullptr, rows, dim, classes, type, true, &s), loss_space(nullptr, rows, dim, classes, type, false, &s));
}

dynlp_status dynlp_head_loss(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_targets* targets,
                             float* loss, const dynlp_matrix* dh, float* dweight, float* dbias, const dynlp_call* call) {
    CHECK(check_head(h, weight));
    if (!targets) REFUSE("targets is NULL");
    if (h->rows > 0 && !targets->soft == !targets->hard) REFUSE("targets are either soft rows or hard labels");
    if (dh && dh->data) {
        CHECK(check_matrix(dh, "dh"));
        if (dh->type != h->type || dh->dim != h->dim || dh->rows != h->rows) REFUSE("dh has another shape or type than h");
        // a row's logits are made before its dh is stored, but dweight reads h again
        const bool in_place = dh->data == h->data && (dh->stride == h->stride || h->rows == 1);
        if (overlap(*h, *dh) && (dweight || !in_place)) REFUSE("dh overlaps h%s", in_place ? ", which dweight needs" : "");
        if (overlap(*weight, *dh)) REFUSE("dh overlaps weight");
    }
    const int64_t bytes = dweight || dbias ? dynlp_head_loss_workspace(h->rows, h->dim, (int32_t)weight->rows, h->type) : 0;
    CHECK(check_workspace(call, bytes));
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const Head a = head_of(h, weight, bias);
    LossSpace s{};
    if (bytes) loss_space(static_cast<char*>(call->workspace), a.rows, a.dim, a.classes, h->type, a.ld_h < kMostFusedStride, &s);
    by_head(h->type, weight->rows, [&](auto type, auto tiles) {
        using T = decltype(type);
        constexpr int CT = decltype(tiles)::v;
        const Loss g{targets->soft, targets->hard, targets->row_weight, targets->rejected, targets->grad_scale, loss,
                     dh ? dh->data : nullptr, dh ? dh->stride : 0, s.dz, s.kept};
        if (a.rows > 0 && s.fused) {
            auto fused = [&](auto per_wave) {
                constexpr int GPW = decltype(per_wave)::v;
                static std::atomic<uint64_t> allowed{0};
                allow_shared(k_head_fused<T, CT, GPW>, allowed);
                k_head_fused<T, CT, GPW><<<(unsigned)s.splits, kWave * fused_waves(CT), (size_t)fused_bytes<T, CT>(a.dim), stream>>>(a, g, s.part);
            };
            if constexpr (fused_waves(CT) < 8) {
                if (a.dim > kFusedColumns * fused_waves(CT)) fused(Tiles<2>());
                else fused(Tiles<1>());
            } else {
                fused(Tiles<1>());
            }
        } else if (a.rows > 0) {
            for (int64_t row = 0; row < a.rows; row += kMostBlocks * kHeadRows)
                k_head_loss<T, CT><<<(unsigned)std::min(ceil_div(a.rows - row, kHeadRows), kMostBlocks), kBlock, 0, stream>>>(a, g, row);
        }
        if (!bytes) return;
        if (a.rows > 0 && !s.fused) {
            const Outer o{a.h, s.dz, s.kept, s.part, a.ld_h, a.rows, s.per_wave, a.dim, a.classes};
            k_head_outer<T, CT><<<dim3((unsigned)s.splits, (unsigned)ceil_div(a.dim, 16 * Piece<T>::n)), kBlock, 0, stream>>>(o);
        }
        k_head_join<<<(unsigned)std::min(ceil_div((int64_t)a.classes * (a.dim + 1), 16), kMostBlocks), kBlock, 0, stream>>>(
            s.part, a.rows > 0 ? s.splits : 0, a.classes, a.dim, dweight, dbias);
    });
    return launched();
}

// ---- AdamW ------------------------------------------------------------------------------------------------------------

dynlp_status dynlp_adamw_step(int32_t count, const dynlp_adamw_tensor* tensors, const dynlp_adamw_options* o, const dynlp_call* call) {
    if (count < 0 || (count > 0 && !tensors)) REFUSE("%d tensors%s", count, count > 0 ? ", tensors is NULL" : "");
    if (!o) REFUSE("options is NULL");
    CHECK(check_workspace(call, 0));
    if (!(o->lr >= 0.0) || !std::isfinite(o->lr)) REFUSE("lr = %g", o->lr);
    if (!(o->beta1 >= 0.0 && o->beta1 < 1.0)) REFUSE("beta1 = %g is not in [0, 1)", o->beta1);
    if (!(o->beta2 >= 0.0 && o->beta2 < 1.0)) REFUSE("beta2 = %g is not in [0, 1)", o->beta2);
    if (!(o->eps > 0.0) || !std::isfinite(o->eps)) REFUSE("eps = %g", o->eps);
    if (o->step < 1) REFUSE("step = %lld: the first is 1", (long long)o->step);
    if (o->state_bits != 32 && o->state_bits != 8) REFUSE("states of %d bits: 32 or 8 are possible", o->state_bits);
    AdamwBatch b{};
    b.grad_scale = o->grad_scale;
    b.beta1 = (float)o->beta1;
    b.beta2 = (float)o->beta2;
    b.rest1 = (float)(1.0 - o->beta1);
    b.rest2 = (float)(1.0 - o->beta2);
    b.step_size = (float)(o->lr / (1.0 - std::pow(o->beta1, (double)o->step)));
    b.root = (float)(1.0 / std::sqrt(1.0 - std::pow(o->beta2, (double)o->step)));
    b.eps = (float)o->eps;
    if (!(b.eps > 0.f) || !std::isfinite(b.eps)) REFUSE("eps = %g is %g in 32 bits", o->eps, b.eps);
    if (!std::isfinite(b.step_size)) REFUSE("lr = %g makes a step of %g in 32 bits", o->lr, b.step_size);
    const bool bits8 = o->state_bits == 8;
    auto aligned = [](const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; };
    for (int32_t k = 0; k < count; ++k) {
        const dynlp_adamw_tensor& t = tensors[k];
        if (t.n < 0 || t.n > (int64_t(1) << 40)) REFUSE("tensor %d: %lld elements", k, (long long)t.n);
        if (t.param_type < DYNLP_FLOAT32 || t.param_type > DYNLP_FLOAT16 || t.grad_type < DYNLP_FLOAT32 || t.grad_type > DYNLP_FLOAT16 ||
            (t.copy && (t.copy_type < DYNLP_FLOAT32 || t.copy_type > DYNLP_FLOAT16)))
            REFUSE("tensor %d: a type is not a dynlp_type", k);
        if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.f) REFUSE("tensor %d: weight_decay = %g", k, t.weight_decay);
        if (!std::isfinite((float)(o->lr * (double)t.weight_decay))) REFUSE("tensor %d: weight_decay = %g with lr = %g", k, t.weight_decay, o->lr);
        if (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (bits8 && (!t.m_scale || !t.v_scale)))) REFUSE("tensor %d: an array is NULL", k);
        if (!aligned(t.param, type_size(t.param_type)) || !aligned(t.grad, type_size(t.grad_type)) || (t.copy && !aligned(t.copy, type_size(t.copy_type))) ||
            (bits8 ? !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) : !aligned(t.m, 4) || !aligned(t.v, 4)))
            REFUSE("tensor %d: an array is not aligned to its elements", k);
    }
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const uint32_t key = dither_mix(dither_mix(o->seed) ^ (uint32_t)o->step);
    // Arrays larger than half the cache before the memory are read and written past the caches, which keep what a training step reads next (24M elements,
    // 32 bits: 119 us, 132 us through the caches; 256M, 8 bits: 876 and 894 us; three sets of 256 MB in turn: 85 and 92).  Up to the cache's size a set that
    // is stepped with little in between stays in it: alone, 256 MB, 83 us past and 69 through.  A student's whole step, arrays of 180 MB: 198 and 189 us with
    // 8,192 items of 64 columns, 455 and 469 with 65,536 of 256; of 250 MB: 220 and 227, 486 and 512
    int64_t bytes = 0, blocks = 0;
    for (int32_t k = 0; k < count; ++k)
        bytes += tensors[k].n * (type_size(tensors[k].param_type) + type_size(tensors[k].grad_type) + (bits8 ? 2 : 8) + (tensors[k].copy ? type_size(tensors[k].copy_type) : 0));
    const bool past = bytes > kHalfCache;
    auto launch = [&]() {
        if (b.count > 0) {
            if (bits8 && past) k_adamw<true, true><<<(unsigned)blocks, kBlock, 0, stream>>>(b);
            else if (bits8) k_adamw<true, false><<<(unsigned)blocks, kBlock, 0, stream>>>(b);
            else if (past) k_adamw<false, true><<<(unsigned)blocks, kBlock, 0, stream>>>(b);
            else k_adamw<false, false><<<(unsigned)blocks, kBlock, 0, stream>>>(b);
        }
        b.count = 0;
        blocks = 0;
    };
    for (int32_t k = 0; k < count; ++k) {
        const dynlp_adamw_tensor& t = tensors[k];
        if (t.n == 0) continue;
        const int64_t mine = ceil_div(t.n, kStateBlock * (kBlock / kWave));
        // a tensor that fills a launch goes on in the next, where its first workgroup (2^30 at most) lies before the launch's
        for (int64_t done = 0; done < mine;) {
            if (b.count == kAdamwTensors || blocks == kMostBlocks) launch();
            b.t[b.count++] = AdamwTensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.n, (float)(1.0 - o->lr * (double)t.weight_decay),
                                         dither_mix(key ^ (uint32_t)k), t.param_type | t.grad_type << 4 | t.copy_type << 8, (int32_t)(blocks - done)};
            const int64_t now = std::min(mine - done, kMostBlocks - blocks);
            blocks += now;
            done += now;
        }
    }
    launch();
    return launched();
}

}  // extern "C"
