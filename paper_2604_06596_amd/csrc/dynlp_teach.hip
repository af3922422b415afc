// libdynlp: host side of scores and of learning from a teacher's first classes (include/dynlp_train.h): checks, launch sizes, C ABI.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "dynlp_ask.h"
#include "dynlp_host.h"

using namespace dynlp;

namespace {

constexpr int64_t kMostBlocks = 0xffffffff / kBlock;  // workgroups: a launch has fewer than 2^32 threads
constexpr int64_t kMostStride = 1 << 22;              // elements: 32 bits hold the bytes of a tile's rows
constexpr int64_t kLogitsBytes = int64_t(1) << 30;    // of logits in memory at a time (8,192 x 32,768: 776 us, with 256 MB 935)
constexpr int64_t kTermsBytes = int64_t(4) << 30;     // of dz in memory at a time
constexpr int64_t kMostTeachRows = 1 << 24;           // at a time: a launch has fewer than 2^32 threads
constexpr int64_t kTilesBytes = DYNLP_MAX_WIDE_CLASSES / 256 * 4;  // of shared memory: k_teach_lists counts the entries of each tile, beside arrays of its own
static_assert(kTilesBytes <= 64 * 1024 && DYNLP_MAX_TOP <= 8 * 16, "k_teach_lists");

// ---- products ---------------------------------------------------------------------------------------------------------

struct Tiling {
    int tm, tn, wm, wn;
};
constexpr int kRoom = 512;  // workgroups that the chip has room for: two on each CU, by their shared memory
// The tile with which the product (m: the fast index of the result) is done soonest.  Weighed: what a product takes in tiles of a size, relative to the largest: 8,192 x
// 32,768 x 1,024 with logits and their sums 1, 1.48, 1.40, 1.12, 1.45 and 3.3 in the order of the table, 8,192 x 8,192 x 1,024 without them (157 us with the largest) 1, 1.57, 1.39,
// 1.15, 1.39 and 3.6.  Rounds of kRoom tiles; where sums may be split in parts of 8 steps (steps > 0), the tiles share the chip evenly.
Tiling tiling(int64_t m, int64_t n, int64_t steps) {
    struct Weighed {
        Tiling t;
        double weight;
    };
    static const Weighed all[] = {{{256, 128, 2, 2}, 1.0}, {{128, 64, 2, 2}, 1.5}, {{256, 64, 4, 1}, 1.4}, {{128, 128, 2, 2}, 1.1}, {{64, 256, 1, 4}, 1.4}, {{256, 16, 4, 1}, 3.5}};
    const Weighed* best = nullptr;
    double least = 0.0;
    for (const Weighed& w : all) {
        const bool few = n <= 64;  // rows: bound by reading the other operand
        if (w.t.tm * w.t.tn == 128 * 64 && !few) continue;
        if (w.t.tm < 256 && m > (few ? 1 << 20 : 1024)) continue;  // k_teach_lists counts the tiles of classes in 64 KB
        const int64_t tiles = ceil_div(m, w.t.tm) * ceil_div(n, w.t.tn);
        const double rounds = steps > 0 ? (double)tiles / (double)std::min<int64_t>(kRoom, tiles * std::max<int64_t>(steps / 8, 1)) : (double)ceil_div(tiles, kRoom);
        const double cost = rounds * w.t.tm * w.t.tn * w.weight;
        if (!best || cost < least) best = &w, least = cost;
    }
    return best->t;
}
// Of logits: classes by rows.
Tiling logits_tiling(int64_t classes, int64_t rows) { return tiling(classes, rows, 0); }
template <bool TA, bool TB, bool WOVEN, typename F>
void by_tiling(const Tiling& t, F f) {
    if (t.tn == 16) f(Shape<256, 16, 4, 1, TA, TB, WOVEN>());
    else if (t.tn == 64 && t.tm == 128) f(Shape<128, 64, 2, 2, TA, TB, WOVEN>());
    else if (t.tn == 64) f(Shape<256, 64, 4, 1, TA, TB, WOVEN>());
    else if (t.tm == 64) f(Shape<64, 256, 1, 4, TA, TB, WOVEN>());
    else if (t.tm == 128) f(Shape<128, 128, 2, 2, TA, TB, WOVEN>());
    else f(Shape<256, 128, 2, 2, TA, TB, WOVEN>());
}

// g.whole, g.splits and g.per_split may be set by split_tiles().
template <typename T, bool TA, bool TB, bool WOVEN, typename E>
void launch_product(Wide g, const Tiling& t, int64_t m, int64_t n, const E& e, hipStream_t stream) {
    if (g.tiles_m == 0) {
        g.tiles_m = (int)ceil_div(m, t.tm);
        g.tiles_n = (int)ceil_div(n, t.tn);
        g.whole = g.tiles_m * g.tiles_n;
    }
    by_tiling<TA, TB, WOVEN>(t, [&](auto shape) {
        using S = decltype(shape);
        static std::atomic<uint64_t> allowed{0};
        allow_shared(k_wide<T, S, E>, allowed);
        const int others = g.tiles_m * g.tiles_n - g.whole;
        k_wide<T, S, E><<<(unsigned)(g.whole + others * g.splits), kBlock, kStages * S::stage, stream>>>(g, e);
    });
}

// The chip has room for two workgroups on each CU: the tiles that do not fill it once more have their sums split, so that all of it has work to the end, but in
// parts of 8 steps at least.  Returns the elements of their parts.
Tiling gradient_tiling(const Wide& g, int64_t m, int64_t n) { return tiling(m, n, (int64_t)g.pairs * g.steps); }
int64_t split_tiles(Wide* g, const Tiling& t, int64_t m, int64_t n) {
    g->tiles_m = (int)ceil_div(m, t.tm);
    g->tiles_n = (int)ceil_div(n, t.tn);
    const int64_t tiles = (int64_t)g->tiles_m * g->tiles_n, steps = (int64_t)g->pairs * g->steps;
    const int64_t others = tiles % kRoom, splits = others ? std::min(kRoom / others, steps / 8) : 1;
    g->whole = (int)tiles;
    g->splits = 1;
    if (splits < 2) return 0;
    g->whole = (int)(tiles - others);
    g->per_split = (int)ceil_div(steps, splits);
    g->splits = (int)ceil_div(steps, g->per_split);
    return others * g->splits * t.tm * t.tn;
}

// Pairs of terms, the smallest products first.
void set_pairs(Wide* g, int terms_a, int terms_b) {
    g->pairs = 0;
    g->pair = 0;
    for (int sum = 2; sum >= 0; --sum)
        for (int a = 0; a < terms_a; ++a) {
            const int b = sum - a;
            if (b >= 0 && b < terms_b) g->pair |= (uint32_t)(a | b << 2) << (4 * g->pairs++);
        }
}

// ---- operands ---------------------------------------------------------------------------------------------------------

// A matrix as 16-bit terms whose rows are whole steps and begin at multiples of 16 bytes: as it lies, or laid out anew.
struct Laid {
    const void* p;
    int64_t ld, term;  // elements; bytes
    int terms;
};
int terms_in(int32_t type) { return type == DYNLP_FLOAT32 ? 3 : 1; }
int64_t laid_ld(int64_t dim) { return round_up(dim, kStep); }
bool lies_well(const dynlp_matrix& m) {
    return m.type != DYNLP_FLOAT32 && reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && m.dim % kStep == 0 &&
           (m.rows == 1 || (m.stride % 8 == 0 && m.stride < kMostStride));
}
Laid lay_out(const dynlp_matrix& m, uint16_t* to, hipStream_t stream) {
    if (!to) return {m.data, m.rows == 1 ? m.dim : m.stride, 0, 1};
    const int64_t ld = laid_ld(m.dim), term = m.rows * ld, blocks = std::min<int64_t>(ceil_div(m.rows * (ld / 8), kBlock), 8192);
    if (m.type == DYNLP_FLOAT32)
        k_lay_out<float><<<(unsigned)blocks, kBlock, 0, stream>>>(static_cast<const float*>(m.data), m.stride, m.rows, m.dim, to, ld, term);
    else  // bits alone matter
        k_lay_out<bf16><<<(unsigned)blocks, kBlock, 0, stream>>>(static_cast<const bf16*>(m.data), m.stride, m.rows, m.dim, to, ld, term);
    return {to, ld, 2 * term, terms_in(m.type)};
}
uint16_t* take_laid(Carve& c, int64_t rows, int64_t dim, int32_t type) { return c.take<uint16_t>(rows * laid_ld(dim) * terms_in(type)); }

dynlp_matrix rows_of(const dynlp_matrix& m, int64_t first, int64_t rows) {
    dynlp_matrix r = m;
    r.data = static_cast<char*>(m.data) + first * m.stride * type_size(m.type);
    r.rows = rows;
    return r;
}

Wide logits_product(const Laid& weight, int64_t classes, const Laid& h, int64_t rows, int dim) {
    Wide g{};
    g.a = weight.p, g.ld_a = weight.ld, g.term_a = weight.term, g.m = (int)classes;
    g.b = h.p, g.ld_b = h.ld, g.term_b = h.term, g.n = (int)rows;
    g.k = dim;
    g.steps = (int)(laid_ld(dim) / kStep);
    set_pairs(&g, weight.terms, h.terms);
    return g;
}

// F is called with a value of the type that the products of a matrix's terms are made in.
template <typename F>
void by_terms(int32_t type, F f) {
    if (type == DYNLP_FLOAT16) f(f16());
    else f(bf16());
}

template <typename F>
void by_type(int32_t type, F f) {
    if (type == DYNLP_FLOAT32) f(float());
    else if (type == DYNLP_BFLOAT16) f(bf16());
    else f(f16());
}

dynlp_status check_wide_head(const dynlp_matrix* h, const dynlp_matrix* weight) {
    CHECK(check_matrix(h, "h"));
    CHECK(check_matrix(weight, "weight"));
    if (weight->type != h->type) REFUSE("weight has type %d, h %d", weight->type, h->type);
    if (weight->dim != h->dim) REFUSE("weight has rows of %d elements, h of %d", weight->dim, h->dim);
    if (weight->rows < 1 || weight->rows > DYNLP_MAX_WIDE_CLASSES) REFUSE("%lld classes: 1 .. %d are possible", (long long)weight->rows, DYNLP_MAX_WIDE_CLASSES);
    if (h->dim > DYNLP_MAX_WIDE_DIM) REFUSE("rows of %d elements: %d are possible", h->dim, DYNLP_MAX_WIDE_DIM);
    return DYNLP_OK;
}

// ---- scores -----------------------------------------------------------------------------------------------------------

dynlp_status check_scores(const dynlp_scores* s, int64_t rows, int64_t classes) {
    if (!s) REFUSE("scores is NULL");
    if (s->given < 0 || s->given > DYNLP_MAX_GIVEN) REFUSE("%d given classes: 0 .. %d are possible", s->given, DYNLP_MAX_GIVEN);
    if (s->top < 0 || s->top > DYNLP_MAX_TOP) REFUSE("the first %d classes: 0 .. %d are possible", s->top, DYNLP_MAX_TOP);
    if (s->top > classes) REFUSE("the first %d of %lld classes", s->top, (long long)classes);
    if (rows > 0 && s->given > 0 && (!s->classes || !s->log_given)) REFUSE("given classes without %s", s->classes ? "log_given" : "classes");
    return DYNLP_OK;
}

Scores scores_of(const dynlp_scores* s) {
    return Scores{s->classes, s->log_given, s->entropy, s->top_classes, s->log_top, s->rejected, s->given, s->top_classes || s->log_top ? s->top : 0};
}

// The scores of rows from `row` on.
Scores scores_from(const Scores& s, int64_t row) {
    Scores o = s;
    if (o.classes) o.classes += row * o.given;
    if (o.log_given) o.log_given += row * o.given;
    if (o.entropy) o.entropy += row;
    if (o.top_classes) o.top_classes += row * o.top;
    if (o.log_top) o.log_top += row * o.top;
    return o;
}

template <typename T, bool PROB>
void launch_scores(const T* x, int64_t ld, int64_t rows, int dim, const Scores& o, hipStream_t stream) {
    auto scan = [&](auto pieces, auto waves) {
        constexpr int P = decltype(pieces)::value, W = decltype(waves)::value;
        const int64_t blocks = W == 1 ? ceil_div(rows, kBlock / kWave) : rows;
        static std::atomic<uint64_t> allowed{0};
        allow_shared(k_row_scores<T, PROB, P, W>, allowed);
        k_row_scores<T, PROB, P, W><<<(unsigned)std::min<int64_t>(blocks, 1 << 20), W == 1 ? kBlock : W * kWave, row_space<T>(W), stream>>>(x, ld, rows, dim, o);
    };
    using std::integral_constant;
    constexpr int E = Piece<T>::n, most = 32 / E;  // pieces of a lane: 2,048 values of a wave
    const int need = (int)std::min<int64_t>(ceil_div(dim, E * kWave), most);
    // a lane for each row pays once there are rows for a wave on each of the 1,024 SIMDs
    auto lanes = [&](auto first) {
        constexpr int K = decltype(first)::value;
        k_lane_scores<T, PROB, K><<<(unsigned)std::min<int64_t>(ceil_div(rows, kWave), 1 << 20), kWave, kWave * (dim | 1) * 4, stream>>>(x, ld, rows, dim, o);
    };
    const bool many = dim <= 64 && rows >= 1024 * kWave;
    if (many && o.top <= 2) lanes(integral_constant<int, 2>());
    else if (many && o.top <= 4) lanes(integral_constant<int, 4>());
    else if (many && o.top <= 8) lanes(integral_constant<int, 8>());
    else if (dim <= 64) k_short_scores<T, PROB><<<(unsigned)std::min<int64_t>(ceil_div(rows, kBlock / 16), 2048), kBlock, 0, stream>>>(x, ld, rows, dim, o);
    else if (need == 1) scan(integral_constant<int, 1>(), integral_constant<int, 1>());
    else if (need == 2) scan(integral_constant<int, 2>(), integral_constant<int, 1>());
    else if (dim <= 1024 && most > 4) scan(integral_constant<int, 4>(), integral_constant<int, 1>());
    else if (dim <= 2048) scan(integral_constant<int, most>(), integral_constant<int, 1>());
    // a wave's search for a threshold and its last cuts cost as much as some 10,000 values: one wave for a row where that makes two for each of the 1,024 SIMDs.  us with
    // one and with four, the first 32: 1,024 rows of 5,000 bfloat16 21 and 19, of 100,003 120 and 80, float32 114 and 87; 2,048 rows 23 and 32, 140 and 147, 157 and 160; 4,099
    // rows 31 and 54, 187 and 242, 297 and 301; 16,400 rows of 20,011 bfloat16 197 and 350, float32 247 and 287
    else if (rows >= 2048) scan(integral_constant<int, most>(), integral_constant<int, 1>());
    else if (rows > 512) scan(integral_constant<int, most>(), integral_constant<int, 4>());
    else scan(integral_constant<int, most>(), integral_constant<int, 16>());
}

// Elements of a row of logits: rows that begin a power of two apart are written to few of the memory's channels (8,192 x 32,768, 256 MB at a time: 935 us, 845 so).
int64_t logits_ld(int64_t classes) { return round_up(classes, 16) + 32; }

// Rows whose logits are in memory at a time.
int64_t logits_rows(int64_t rows, int64_t classes) {
    const int64_t most = std::max<int64_t>(kLogitsBytes / (logits_ld(classes) * 4) / 256 * 256, 256);
    return std::min(rows, most);
}

// Classes of a group: a wave's part of the product.  Few rows have more waves than rows, and smaller parts.
int group_size(int64_t rows, int64_t classes) {
    if (rows <= 16) return classes <= 16 * 2048 ? 16 : 64;
    const Tiling t = logits_tiling(classes, rows);
    return t.tm / t.wm;
}

struct ScoreSpace {
    uint16_t *h, *weight;
    float* z;
    GroupSums* sums;
    int64_t rows;  // at a time
    int size, groups;
};
int64_t score_space(char* base, int64_t rows, int64_t dim, int64_t classes, int32_t type, bool lay_h, bool lay_weight, ScoreSpace* s) {
    Carve c{base};
    s->rows = logits_rows(rows, classes);
    s->size = group_size(s->rows, classes);
    s->groups = (int)ceil_div(classes, s->size);
    s->z = c.take<float>(s->rows * logits_ld(classes));
    s->sums = c.take<GroupSums>(s->rows * s->groups);
    if (s->rows <= 16) return c.used;  // rows are read as they lie
    s->weight = lay_weight ? take_laid(c, classes, dim, type) : nullptr;
    s->h = lay_h ? take_laid(c, s->rows, dim, type) : nullptr;
    return c.used;
}

void launch_groups(const ScoreSpace& s, int64_t ld, int64_t rows, int classes, const Scores& o, int64_t row0, hipStream_t stream) {
    int merge = 1, log2 = 0;
    while (ceil_div(s.groups, merge) > kTurns * kWave) merge *= 2;
    while (4 << log2 < s.size * merge) ++log2;
    k_group_scores<<<(unsigned)std::min<int64_t>(rows, 1 << 20), kWave, 0, stream>>>(s.z, ld, s.sums, s.groups, merge, log2, rows, classes, o, row0);
}

// F is called with (T(), number of tiles of 16 classes).
template <typename F>
void by_few_classes(int32_t type, int64_t classes, F f) {
    auto tiles = [&](auto t) {
        switch ((classes + 15) / 16) {
            case 1: f(t, std::integral_constant<int, 1>()); break;
            case 2: f(t, std::integral_constant<int, 2>()); break;
            case 3: f(t, std::integral_constant<int, 3>()); break;
            default: f(t, std::integral_constant<int, 4>());
        }
    };
    if (type == DYNLP_FLOAT32) tiles(float());
    else if (type == DYNLP_BFLOAT16) tiles(bf16());
    else tiles(f16());
}

void launch_few_scores(const dynlp_matrix& h, const dynlp_matrix& weight, const float* bias, const Scores& o, hipStream_t stream) {
    const Head a{h.data, weight.data, bias, h.stride, weight.stride, h.rows, h.dim, (int)weight.rows};
    by_few_classes(h.type, weight.rows, [&](auto type, auto tiles) {
        using T = decltype(type);
        constexpr int CT = decltype(tiles)::value;
        const int64_t bytes = a.dim <= 1 << 14 ? shared_bytes<T, CT>(a.dim) : kSharedMemory + 1, blocks = ceil_div(a.rows, kLabelRows);
        // a copy of W pays once a workgroup has several tiles of rows
        const int64_t stay = 256 * std::min<int64_t>(kSharedMemory / bytes, 4);
        if (bytes <= kSharedMemory && blocks >= 2 * stay) {
            static std::atomic<uint64_t> allowed{0};
            allow_shared(k_few_scores<T, CT, true>, allowed);
            k_few_scores<T, CT, true><<<(unsigned)stay, kBlock, (size_t)bytes, stream>>>(a, o);
        } else {
            for (int64_t row = 0; row < a.rows; row += kMostBlocks * kLabelRows) {
                Head part = a;
                part.h = static_cast<const T*>(a.h) + row * a.ld_h;
                part.rows = std::min(a.rows - row, kMostBlocks * kLabelRows);
                Scores to = o;
                if (row > 0) to = scores_from(o, row);
                k_few_scores<T, CT, false><<<(unsigned)ceil_div(part.rows, kLabelRows), kBlock, 0, stream>>>(part, to);
            }
        }
    });
}

}  // namespace

extern "C" {

int64_t dynlp_row_scores_workspace(int64_t rows, int32_t classes, int32_t top) {
    (void)rows, (void)classes, (void)top;
    return 0;
}

dynlp_status dynlp_row_scores(const dynlp_matrix* x, int32_t probabilities, const dynlp_scores* scores, const dynlp_call* call) {
    CHECK(check_matrix(x, "x"));
    CHECK(check_scores(scores, x->rows, x->dim));
    CHECK(check_workspace(call, dynlp_row_scores_workspace(x->rows, x->dim, scores->top)));
    if (x->rows == 0) return DYNLP_OK;
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const Scores o = scores_of(scores);
    auto run = [&](auto type) {
        using T = decltype(type);
        const T* p = static_cast<const T*>(x->data);
        if (probabilities) launch_scores<T, true>(p, x->stride, x->rows, x->dim, o, stream);
        else launch_scores<T, false>(p, x->stride, x->rows, x->dim, o, stream);
    };
    if (x->type == DYNLP_FLOAT32) run(float());
    else if (x->type == DYNLP_BFLOAT16) run(bf16());
    else run(f16());
    return launched();
}

int64_t dynlp_head_scores_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t type) {
    if (rows < 1 || rows > kMostRows || dim < 1 || dim > DYNLP_MAX_WIDE_DIM || classes < 1 || classes > DYNLP_MAX_WIDE_CLASSES) return 0;
    if (classes <= DYNLP_MAX_CLASSES) return 0;
    ScoreSpace s{};
    return score_space(nullptr, rows, dim, classes, type, true, true, &s);
}

dynlp_status dynlp_head_scores(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_scores* scores, const dynlp_call* call) {
    CHECK(check_wide_head(h, weight));
    CHECK(check_scores(scores, h->rows, weight->rows));
    const int classes = (int)weight->rows;
    CHECK(check_workspace(call, dynlp_head_scores_workspace(h->rows, h->dim, classes, h->type)));
    if (h->rows == 0) return DYNLP_OK;
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    const Scores o = scores_of(scores);
    if (classes <= DYNLP_MAX_CLASSES) {
        launch_few_scores(*h, *weight, bias, o, stream);
        return launched();
    }
    ScoreSpace s{};
    score_space(static_cast<char*>(call->workspace), h->rows, h->dim, classes, h->type, !lies_well(*h), !lies_well(*weight), &s);
    const int64_t ld = logits_ld(classes);
    if (s.rows <= 16) {
        const Head a{h->data, weight->data, bias, h->stride, weight->stride, h->rows, h->dim, classes};
        const Logits e{s.z, ld, s.sums, s.groups, bias, (int)h->rows, classes};
        by_type(h->type, [&](auto type) {
            using T = decltype(type);
            const unsigned blocks = (unsigned)ceil_div(s.groups, kBlock / kWave);
            if (s.size == 16) k_thin_logits<T, 1><<<blocks, kBlock, 0, stream>>>(a, e);
            else k_thin_logits<T, 4><<<blocks, kBlock, 0, stream>>>(a, e);
        });
        launch_groups(s, ld, h->rows, classes, o, 0, stream);
        return launched();
    }
    const Laid w = lay_out(*weight, s.weight, stream);
    const Tiling tile = logits_tiling(classes, s.rows);  // of all turns: its groups have a size
    for (int64_t row = 0; row < h->rows; row += s.rows) {
        const int64_t rows = std::min(s.rows, h->rows - row);
        const Laid x = lay_out(rows_of(*h, row, rows), s.h, stream);
        const Wide g = logits_product(w, classes, x, rows, h->dim);
        const Logits e{s.z, ld, s.sums, s.groups, bias, (int)rows, classes};
        by_terms(h->type, [&](auto type) { launch_product<decltype(type), false, false, false>(g, tile, classes, rows, e, stream); });
        launch_groups(s, ld, rows, classes, o, row, stream);
    }
    return launched();
}

}  // extern "C"

// ---- distillation -----------------------------------------------------------------------------------------------------

namespace {

// Terms of dz that dweight is made of: as many as hold 24 bits of it (22 in float16, and nothing below 2^-39 of the largest weight), or one where the gradients are rounded to
// 16 bits anyway.  One term's rounding errors average to what the result's own rounding adds where many values of dz make a gradient; with few rows some values decide, and the
// error was up to 1.56 times that of the rounding alone.  Two terms are used there, and where the products are short beside the launches.
bool is_small(int64_t rows, int64_t dim, int64_t classes) { return rows <= 256 || (double)rows * (double)dim * (double)classes <= 2147483648.0; }
int dz_terms(int32_t type, int32_t grad_type, bool small) {
    if (type != DYNLP_FLOAT32 && grad_type != DYNLP_FLOAT32) return small ? 2 : 1;
    return type == DYNLP_FLOAT16 ? 2 : 3;
}
// Of these, those that dh is made of.
int dh_terms(int32_t type, bool small) { return type == DYNLP_FLOAT32 ? 3 : small ? 2 : 1; }

struct TeachSpace {
    int64_t rows;  // at a time
    int64_t ld;    // of dz
    uint16_t *h, *weight, *own, *dz;
    uint32_t *zeros, *largest, *kept;
    float *undo, *undo_row, *ratio;
    Lists lists;
    float *top, *sum, *picked, *share, *base, *inverse, *factor;
    float *bias_part, *part, *dweight;
    int64_t part_ld;   // of top, sum, picked and share
    int terms, own_terms, parts;
    bool small;
};

// grad_type: of dweight, or -1 where no gradient is asked for.
int64_t teach_space(char* base, int64_t rows, int64_t dim, int64_t classes, int kept, int32_t type, int32_t grad_type, bool lay_h, bool lay_weight, TeachSpace* s) {
    Carve c{base};
    const bool grads = grad_type >= 0;
    s->small = is_small(rows, dim, classes);
    s->terms = dz_terms(type, grad_type, s->small);
    s->own_terms = type == DYNLP_FLOAT16 ? dh_terms(type, s->small) : 0;
    s->ld = laid_ld(classes);
    const int64_t most = std::max<int64_t>(kTermsBytes / (s->ld * 2 * (s->terms + s->own_terms)) / 256 * 256, 256);
    s->rows = std::min({rows, most, kMostTeachRows});
    const Tiling t = logits_tiling(classes, s->rows);
    s->parts = (int)ceil_div(classes, t.tm) * t.wm;
    s->part_ld = round_up(s->rows, 64);
    s->zeros = c.take<uint32_t>(128);
    s->largest = c.take<uint32_t>(1);
    s->undo = c.take<float>(1);
    s->kept = c.take<uint32_t>(ceil_div(s->rows, 32));
    s->lists.kept = kept;
    s->lists.tiles = (int)ceil_div(classes, t.tm);
    s->lists.log2 = t.tm == 256 ? 8 : t.tm == 128 ? 7 : 6;
    s->lists.entry = c.take<uint2>(round_up(s->rows, kListRows) * kept);
    s->lists.start = c.take<uint32_t>(ceil_div(s->rows, kListRows) * (s->lists.tiles + 1));
    s->lists.entropy = c.take<float>(s->rows);
    s->lists.weight = c.take<float>(s->rows);
    s->base = c.take<float>(s->rows);
    s->inverse = c.take<float>(s->rows);
    s->factor = c.take<float>(s->rows);
    s->undo_row = s->own_terms ? c.take<float>(s->rows) : nullptr;
    s->ratio = s->own_terms ? c.take<float>(s->rows) : nullptr;
    s->top = c.take<float>(s->parts * s->part_ld);
    s->sum = c.take<float>(s->parts * s->part_ld);
    s->picked = c.take<float>(s->parts * s->part_ld);
    s->share = c.take<float>(s->parts * s->part_ld);
    s->weight = lay_weight ? take_laid(c, classes, dim, type) : nullptr;
    s->h = lay_h ? take_laid(c, s->rows, dim, type) : nullptr;
    if (grads) {
        s->own = s->own_terms ? c.take<uint16_t>(s->rows * s->ld * s->own_terms) : nullptr;
        s->dz = c.take<uint16_t>(s->rows * s->ld * s->terms);
        const int64_t parts = ceil_div(s->rows, t.tn) * t.wn;
        s->bias_part = c.take<float>((parts + ceil_div(parts, kBiasParts)) * s->ld);
        Wide by_h{}, by_w{};
        set_pairs(&by_h, terms_in(type), dh_terms(type, s->small));
        set_pairs(&by_w, terms_in(type), s->terms);
        by_h.steps = (int)(laid_ld(classes) / kStep);
        by_w.steps = (int)ceil_div(s->rows, kStep);
        const int64_t split = std::max(split_tiles(&by_h, gradient_tiling(by_h, dim, s->rows), dim, s->rows), split_tiles(&by_w, gradient_tiling(by_w, dim, classes), dim, classes));
        s->part = c.take<float>(rows > s->rows ? kRoom * 256 * 128 : split);  // the most there are, where the last rows are fewer than others
        s->dweight = rows > s->rows && grad_type != DYNLP_FLOAT32 ? c.take<float>(classes * dim) : nullptr;
    }
    return c.used;
}

// The product to its output.
template <typename T, bool TA, bool TB, typename O>
void launch_gradient(Wide g, int64_t m, int64_t n, float* part, float alpha, const float* undo, const float* undo_row, const uint32_t* kept, void* out, int64_t ld,
                     bool add, hipStream_t stream) {
    const Tiling t = gradient_tiling(g, m, n);
    const int64_t parts = split_tiles(&g, t, m, n);
    const Output<O> to{static_cast<O*>(out), ld, (int)n, (int)m, alpha, undo, undo_row, kept, add};
    launch_product<T, TA, TB, sizeof(O) == 2>(g, t, m, n, Store<O>{to, part}, stream);
    if (parts > 0) {
        const int64_t pieces = parts / g.splits / 4;
        k_wide_join<O><<<(unsigned)std::min<int64_t>(ceil_div(pieces, kBlock), 16384), kBlock, 0, stream>>>(g, t.tm, t.tn, part, to);
    }
}

dynlp_status check_teacher(const dynlp_teacher* t, int64_t rows) {
    if (!t) REFUSE("teacher is NULL");
    if (t->kept < 1 || t->kept > DYNLP_MAX_TOP) REFUSE("lists of %d classes: 1 .. %d are possible", t->kept, DYNLP_MAX_TOP);
    if (rows > 0 && (!t->classes || !t->logits)) REFUSE("a teacher without %s", t->classes ? "logits" : "classes");
    if (!(t->temperature > 0.f) || !std::isfinite(t->temperature) || !std::isfinite(1.44269504f / t->temperature) || !std::isfinite(t->temperature * t->temperature))
        REFUSE("temperature = %g", t->temperature);
    if (!std::isfinite(t->grad_scale * t->temperature)) REFUSE("grad_scale = %g with temperature = %g", t->grad_scale, t->temperature);
    return DYNLP_OK;
}

}  // namespace

extern "C" {

int64_t dynlp_head_distill_workspace(int64_t rows, int32_t dim, int32_t classes, int32_t kept, int32_t type, int32_t grad_type) {
    if (rows < 1 || rows > kMostRows || dim < 1 || dim > DYNLP_MAX_WIDE_DIM || classes < 1 || classes > DYNLP_MAX_WIDE_CLASSES || kept < 1 || kept > DYNLP_MAX_TOP) return 0;
    if (classes <= DYNLP_MAX_CLASSES) return grad_type < 0 ? 0 : distill_few_classes_workspace(rows, dim, classes, type);
    TeachSpace s{};
    return teach_space(nullptr, rows, dim, classes, kept, type, grad_type, true, true, &s);
}

dynlp_status dynlp_head_distill(const dynlp_matrix* h, const dynlp_matrix* weight, const float* bias, const dynlp_teacher* teacher, float* loss,
                                const dynlp_matrix* dh, const dynlp_matrix* dweight, float* dbias, const dynlp_call* call) {
    CHECK(check_wide_head(h, weight));
    CHECK(check_teacher(teacher, h->rows));
    const bool want_h = dh && dh->data, want_w = dweight && dweight->data;
    if (want_h) {
        CHECK(check_matrix(dh, "dh"));
        if (dh->type != h->type || dh->dim != h->dim || dh->rows != h->rows) REFUSE("dh has another shape or type than h");
        if (overlap(*h, *dh)) REFUSE("dh overlaps h");
        if (overlap(*weight, *dh)) REFUSE("dh overlaps weight");
    }
    if (want_w) {
        CHECK(check_matrix(dweight, "dweight"));
        if (dweight->type != h->type && dweight->type != DYNLP_FLOAT32) REFUSE("dweight has type %d: float32 or h's (%d) are possible", dweight->type, h->type);
        if (dweight->dim != weight->dim || dweight->rows != weight->rows) REFUSE("dweight has another shape than weight");
        if (overlap(*h, *dweight)) REFUSE("dweight overlaps h");
        if (overlap(*weight, *dweight)) REFUSE("dweight overlaps weight");
        if (want_h && overlap(*dh, *dweight)) REFUSE("dweight overlaps dh");
    }
    const int classes = (int)weight->rows, dim = h->dim;
    const bool grads = want_h || want_w || dbias;
    const int32_t grad_type = want_w ? dweight->type : grads ? h->type : -1;
    CHECK(check_workspace(call, dynlp_head_distill_workspace(h->rows, dim, classes, teacher->kept, h->type, grad_type)));
    const hipStream_t stream = static_cast<hipStream_t>(call->stream);
    if (h->rows == 0) {
        if (want_w)
            by_type(dweight->type, [&](auto type) {
                using O = decltype(type);
                k_teach_zeros<O><<<(unsigned)std::min<int64_t>(ceil_div((int64_t)classes * dim, kBlock), 8192), kBlock, 0, stream>>>(
                    static_cast<O*>(dweight->data), dweight->stride, classes, dim);
            });
        if (dbias) k_teach_zeros<float><<<(unsigned)ceil_div(classes, kBlock), kBlock, 0, stream>>>(dbias, classes, 1, classes);
        return launched();
    }
    const Teacher t{teacher->classes, teacher->logits, teacher->row_weight, teacher->rejected, teacher->kept, classes, 1.f / teacher->temperature,
                    teacher->temperature};
    if (classes <= DYNLP_MAX_CLASSES) {
        distill_few_classes(*h, *weight, bias, t, teacher->grad_scale * teacher->temperature, loss, want_h ? dh : nullptr, want_w ? dweight : nullptr, dbias, call);
        return launched();
    }
    TeachSpace s{};
    teach_space(static_cast<char*>(call->workspace), h->rows, dim, classes, teacher->kept, h->type, grad_type, !lies_well(*h), !lies_well(*weight), &s);
    const Laid w = lay_out(*weight, s.weight, stream);
    const float exponent = 1.44269504f / teacher->temperature, alpha = teacher->grad_scale * teacher->temperature;
    const bool scaled = h->type == DYNLP_FLOAT16;
    for (int64_t row = 0; row < h->rows; row += s.rows) {
        const int64_t rows = std::min(s.rows, h->rows - row);
        const bool add = row > 0;
        const Laid x = lay_out(rows_of(*h, row, rows), s.h, stream);
        k_teach_begin<<<1, kBlock, 0, stream>>>(s.zeros, s.largest);
        Lists lists = s.lists;
        lists.largest = scaled ? s.largest : nullptr;
        auto read_lists = [&](auto entries) {
            constexpr int E = decltype(entries)::value;
            static std::atomic<uint64_t> allowed{0};
            allow_shared(k_teach_lists<E>, allowed, kTilesBytes);
            k_teach_lists<E><<<(unsigned)ceil_div(rows, kListRows), kBlock, lists.tiles * 4, stream>>>(t, lists, row, rows);
        };
        if (teacher->kept <= 16) read_lists(std::integral_constant<int, 1>());
        else if (teacher->kept <= 32) read_lists(std::integral_constant<int, 2>());
        else if (teacher->kept <= 64) read_lists(std::integral_constant<int, 4>());
        else read_lists(std::integral_constant<int, 8>());
        CHECK(launched());  // what follows reads at places that the lists give
        const Wide g = logits_product(w, classes, x, rows, dim);
        const Tiling tile = logits_tiling(classes, s.rows);  // of all chunks: its parts have a size
        const int parts = (int)ceil_div(classes, tile.tm) * tile.wm;
        by_terms(h->type, [&](auto type) {
            using T = decltype(type);
            const Stats stats{bias, lists, s.top, s.sum, s.picked, s.share, s.part_ld, exponent, (int)rows, classes};
            launch_product<T, false, false, true>(g, tile, classes, rows, stats, stream);
            const RowJoin join{s.top, s.sum, s.picked, s.share, s.part_ld, lists.entropy, lists.weight, lists.largest, loss ? loss + row : nullptr, s.base, s.inverse,
                               s.factor, s.kept, s.undo_row, s.ratio, s.undo, teacher->temperature, exponent, (int)rows, parts};
            if (parts <= 64) k_teach_rows<8><<<(unsigned)ceil_div(rows, 32), 256, 0, stream>>>(join);
            else k_teach_rows<32><<<(unsigned)ceil_div(rows, 32), 1024, 0, stream>>>(join);
            if (!grads) return;
            const int64_t term = rows * s.ld;
            auto gradient = [&](auto terms, auto own) {
                constexpr int TERMS = decltype(terms)::value, OWN = decltype(own)::value;
                const bool shared = OWN == 0;  // by dh and dweight
                const Gradient<T, TERMS, OWN> e{bias, lists, s.base, s.inverse, s.factor, s.ratio, want_h ? s.own : nullptr, want_w || (want_h && shared) ? s.dz : nullptr, s.ld, term,
                                                s.bias_part, exponent, (int)rows, classes};
                launch_product<T, false, false, true>(g, tile, classes, rows, e, stream);
            };
            using std::integral_constant;
            if constexpr (__is_same(T, f16)) {
                if (s.terms == 1) gradient(integral_constant<int, 1>(), integral_constant<int, 1>());
                else if (s.own_terms == 1) gradient(integral_constant<int, 2>(), integral_constant<int, 1>());
                else gradient(integral_constant<int, 2>(), integral_constant<int, 2>());
            } else {
                if (s.terms == 1) gradient(integral_constant<int, 1>(), integral_constant<int, 0>());
                else if (s.terms == 2) gradient(integral_constant<int, 2>(), integral_constant<int, 0>());
                else gradient(integral_constant<int, 3>(), integral_constant<int, 0>());
            }
            if (dbias) {
                int64_t parts_n = ceil_div(rows, tile.tn) * tile.wn;
                float* from = s.bias_part;
                const unsigned across = (unsigned)ceil_div(s.ld, 64);
                if (parts_n > kBiasParts) {  // many rows: first some of them at a time
                    float* to = from + parts_n * s.ld;
                    k_teach_bias<<<dim3(across, (unsigned)ceil_div(parts_n, kBiasParts)), kBlock, 0, stream>>>(from, s.ld, (int)parts_n, kBiasParts, (int)s.ld, 1.f, nullptr, to, false);
                    from = to;
                    parts_n = ceil_div(parts_n, kBiasParts);
                }
                k_teach_bias<<<dim3(across, 1), kBlock, 0, stream>>>(from, s.ld, (int)parts_n, (int)parts_n, classes, alpha, s.undo, dbias, add);
            }
            if (want_h) {
                Wide p{};
                p.a = w.p, p.ld_a = w.ld, p.term_a = w.term, p.m = (int)laid_ld(dim);
                p.b = s.own ? s.own : s.dz, p.ld_b = s.ld, p.term_b = 2 * term, p.n = (int)rows;
                p.k = classes;
                p.steps = (int)(laid_ld(classes) / kStep);
                set_pairs(&p, w.terms, dh_terms(h->type, s.small));
                void* to = static_cast<char*>(dh->data) + row * dh->stride * type_size(dh->type);
                auto run = [&](auto out) {
                    launch_gradient<T, true, false, decltype(out)>(p, dim, rows, s.part, alpha, s.own ? nullptr : s.undo, s.undo_row, s.kept, to, dh->stride, false, stream);
                };
                if (h->type == DYNLP_FLOAT32) {
                    if constexpr (__is_same(T, bf16)) run(float());
                } else {
                    run(T());
                }
            }
            if (want_w) {
                Wide p{};
                p.a = x.p, p.ld_a = x.ld, p.term_a = x.term, p.m = (int)laid_ld(dim);
                p.b = s.dz, p.ld_b = s.ld, p.term_b = 2 * term, p.n = (int)s.ld;
                p.k = (int)rows;
                p.steps = (int)ceil_div(rows, kStep);
                p.kept = s.kept;
                p.zeros = s.zeros;
                set_pairs(&p, x.terms, s.terms);
                if (dweight->type == DYNLP_FLOAT32) {
                    launch_gradient<T, true, true, float>(p, dim, classes, s.part, alpha, s.undo, nullptr, nullptr, dweight->data, dweight->stride, add, stream);
                } else if (s.dweight) {
                    launch_gradient<T, true, true, float>(p, dim, classes, s.part, alpha, s.undo, nullptr, nullptr, s.dweight, dim, add, stream);
                    if (row + rows == h->rows)
                        k_round<T><<<(unsigned)std::min<int64_t>(ceil_div((int64_t)classes * dim, kBlock), 16384), kBlock, 0, stream>>>(
                            s.dweight, classes, dim, static_cast<T*>(dweight->data), dweight->stride);
                } else {
                    launch_gradient<T, true, true, T>(p, dim, classes, s.part, alpha, s.undo, nullptr, nullptr, dweight->data, dweight->stride, false, stream);
                }
            }
        });
    }
    return launched();
}

}  // extern "C"
