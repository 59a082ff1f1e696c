// Host side of the paged cache: argument validation and launch geometry.  No kernels here.
#include "tr_internal.h"

#include <float.h>
#include <math.h>
#include <string.h>
#include <algorithm>
#include <utility>

namespace {

const int64_t INT_LIMIT = ((int64_t)1 << 31) - 1;
const int32_t MOST_HEADS = 1 << 20;     // with 2^31 tokens of them, counts of bytes stay below 2^62
const int32_t MOST_REQUESTS = 65536;    // of a decode step
const int64_t MOST_KEYS = 1ll << 30;    // that a row of the table has room for
const int64_t MOST_UNITS = 1ll << 30;   // of a batch: the kernel counts them in 32 bits

int page_shift(int32_t page_size)
{
    if (page_size < 8 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return -1;
    return __builtin_ctz((unsigned)page_size);
}
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Checks the pool against the shape and gives the form that the kernels address.
int pool_of(const char* who, const tr_shape* sh, const tr_pages* p, TrPool* out)
{
    if (p->reserved != 0) return tr_fail(TR_ERR_INVALID_ARG, "%s: reserved of tr_pages must be 0", who);
    if (p->dtype != sh->dtype || p->n_kv_heads != sh->n_kv_heads || p->head_dim != sh->head_dim)
        return tr_fail(TR_ERR_SHAPE, "%s: pages of type %d with %d heads of %d channels, the shape has type %d, %d heads, %d channels", who, p->dtype,
                       p->n_kv_heads, p->head_dim, sh->dtype, sh->n_kv_heads, sh->head_dim);
    const int shift = page_shift(p->page_size);
    if (shift < 0) return tr_fail(TR_ERR_INVALID_ARG, "%s: page_size %d is not a power of two from 8 to 1024", who, p->page_size);
    if (p->n_pages < 1 || (int64_t)p->n_pages * p->page_size > INT_LIMIT) return tr_fail(TR_ERR_INVALID_ARG, "%s: n_pages %d", who, p->n_pages);
    if (!p->k || !p->v) return tr_fail(TR_ERR_INVALID_ARG, "%s: k or v of the pages is NULL", who);
    const int64_t e = tr_elem_bytes(sh), widest = (int64_t)64 << 20;
    // a stride of a single page or head is never applied; whether the others keep rows apart matters where rows are written
    if (p->row_stride < sh->head_dim || (p->n_kv_heads > 1 && p->head_stride < sh->head_dim) || (p->n_pages > 1 && p->page_stride < sh->head_dim))
        return tr_fail(TR_ERR_INVALID_ARG, "%s: strides of the pages are smaller than a head", who);
    if (p->head_stride < 0 || p->page_stride < 0) // of a single head or page
        return tr_fail(TR_ERR_INVALID_ARG, "%s: strides of the pages are out of range", who);
    if (p->row_stride > widest / e || p->head_stride > widest / e || p->page_stride > (widest * 64 - 1) / e)
        return tr_fail(TR_ERR_UNSUPPORTED, "%s: rows or heads of the pages are more than 64 MiB apart, or pages 4 GiB", who);
    if (!aligned16(p->k) || !aligned16(p->v) || p->page_stride * e % 16 || p->row_stride * e % 16 || p->head_stride * e % 16)
        return tr_fail(TR_ERR_INVALID_ARG, "%s: pages and their strides must be 16-byte aligned", who);
    out->k = (char*)p->k;
    out->v = (char*)p->v;
    out->page_stride = (uint32_t)(p->page_stride * e);
    out->row_stride = (uint32_t)(p->row_stride * e);
    out->head_stride = (uint32_t)(p->head_stride * e);
    out->n_pages = p->n_pages;
    out->page_shift = shift;
    return TR_OK;
}

struct Span {
    const void* p;
    int64_t bytes;
};
bool overlap(const Span& a, const Span& b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}
Span ints(const int32_t* p, int64_t n) { return {p, p ? 4 * n : 0}; }
// n rows of `row` bytes, a stride apart
Span rows(const void* p, int64_t n, int64_t stride, int64_t row) { return {p, p ? (n - 1) * stride + row : 0}; }
// all rows of a pool, and what lies between them
Span pool_span(const TrPool& pool, const void* base, const tr_pages* p)
{
    return {base, (p->n_pages - 1) * (int64_t)pool.page_stride + (p->page_size - 1) * (int64_t)pool.row_stride +
                      (p->n_kv_heads - 1) * (int64_t)pool.head_stride + p->head_dim * (int64_t)(p->dtype == TR_F32 ? 4 : 2)};
}

// Whether every row of K and V has bytes of its own.  Strides nest: taken by size, each is at least what the ones below it span.
struct Nest {
    int64_t stride[3], count[3], span[4]; // span[i]: of the axes below i
    int axes = 0;
};
// Whether two rows of the axes below `axes` meet when one of them is `apart` bytes further on: of an axis only the two differences of
// indices can make up for that, between which it lies.
bool rows_meet(const Nest& n, int axes, int64_t apart)
{
    if (axes == 0) return apart > -n.span[0] && apart < n.span[0];
    const int64_t s = n.stride[axes - 1], most = n.count[axes - 1] - 1;
    const int64_t down = apart >= 0 ? apart / s : -((-apart + s - 1) / s);
    for (int64_t i : {down, down + 1})
        if (i >= -most && i <= most && rows_meet(n, axes - 1, apart - i * s)) return true;
    return false;
}
bool rows_apart(const tr_pages* p)
{
    const int64_t e = p->dtype == TR_F32 ? 4 : 2;
    std::pair<int64_t, int64_t> axes[] = {{p->head_stride * e, p->n_kv_heads}, {p->row_stride * e, p->page_size}, {p->page_stride * e, p->n_pages}};
    std::sort(axes, axes + 3);
    Nest n;
    n.span[0] = p->head_dim * e;
    for (const auto& [stride, count] : axes) {
        if (count == 1) continue;
        if (stride < n.span[n.axes]) return false;
        n.stride[n.axes] = stride;
        n.count[n.axes] = count;
        n.span[n.axes + 1] = (count - 1) * stride + n.span[n.axes];
        ++n.axes;
    }
    return !rows_meet(n, n.axes, (int64_t)((intptr_t)p->v - (intptr_t)p->k));
}

} // namespace

extern "C" int tr_page_map(const int32_t* cached_lens, const int32_t* new_lens, const int32_t* first_pos, int32_t n_req, int32_t page_size,
                           const int32_t* free_pages, int32_t n_free, int32_t* block_table, int32_t max_blocks, int32_t* kv_lens,
                           int32_t* cu_new, int32_t* slots, int32_t* pos, int32_t n_slots, int32_t* counts, void* stream)
{
    return tr_guard_int([&]() -> int {
    tr_clear_error();
    if (n_req < 0 || n_free < 0 || max_blocks < 0 || n_slots < 0) return tr_fail(TR_ERR_INVALID_ARG, "tr_page_map: a count is negative");
    if (n_req > TR_MAX_MAP_REQ) return tr_fail(TR_ERR_UNSUPPORTED, "tr_page_map: %d requests, at most %d", n_req, TR_MAX_MAP_REQ);
    const int shift = page_shift(page_size);
    if (shift < 0) return tr_fail(TR_ERR_INVALID_ARG, "tr_page_map: page_size %d is not a power of two from 8 to 1024", page_size);
    if (!cu_new || !counts || (n_req > 0 && (!cached_lens || !new_lens || !kv_lens)) || (n_slots > 0 && (!slots || !pos)) ||
        (n_free > 0 && !free_pages) || (n_req > 0 && max_blocks > 0 && !block_table))
        return tr_fail(TR_ERR_INVALID_ARG, "tr_page_map: an array is NULL");
    const Span in[] = {ints(cached_lens, n_req), ints(new_lens, n_req), ints(first_pos, n_req), ints(free_pages, n_free)};
    const Span out[] = {ints(block_table, (int64_t)n_req * max_blocks), ints(kv_lens, n_req), ints(cu_new, (int64_t)n_req + 1),
                        ints(slots, n_slots), ints(pos, n_slots), ints(counts, 2)};
    for (int i = 0; i < 6; ++i) {
        for (const Span& s : in)
            if (overlap(out[i], s)) return tr_fail(TR_ERR_INVALID_ARG, "tr_page_map: an output overlaps an input");
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return tr_fail(TR_ERR_INVALID_ARG, "tr_page_map: two outputs overlap");
    }
    TrPageMapArgs a;
    memset(&a, 0, sizeof a);
    a.cached = cached_lens;
    a.fresh = new_lens;
    a.first_pos = first_pos;
    a.free_pages = free_pages;
    a.table = block_table;
    a.kv_lens = kv_lens;
    a.cu = cu_new;
    a.slots = slots;
    a.pos = pos;
    a.counts = counts;
    a.n_req = n_req;
    a.n_free = n_free;
    a.max_blocks = max_blocks;
    a.n_slots = n_slots;
    a.page_shift = shift;
    return tr_launch_page_map(a, (hipStream_t)stream);
    });
}

extern "C" int tr_rotary_init(int32_t layout, int32_t rotary_dim, double base, int32_t scaling, double factor, double original_len,
                              double slow_turns, double fast_turns, double amplitude, tr_rotary* out)
{
    return tr_guard_int([&]() -> int {
    tr_clear_error();
    if (!out) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: out is NULL");
    if (layout != TR_ROPE_INTERLEAVED && layout != TR_ROPE_HALF) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: layout %d", layout);
    if (rotary_dim < 0 || rotary_dim > 128 || rotary_dim % 16) return tr_fail(TR_ERR_SHAPE, "tr_rotary_init: rotary_dim %d is not a multiple of 16 up to 128", rotary_dim);
    if (!(base > 1.0) || !isfinite(base)) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: base must be finite and > 1");
    if (scaling < TR_SCALE_NONE || scaling > TR_SCALE_PARTS) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: scaling %d", scaling);
    if (scaling != TR_SCALE_NONE && (!(factor >= 1.0) || !isfinite(factor))) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: factor must be finite and >= 1");
    if (!isfinite((float)amplitude)) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: amplitude must be finite");
    if (scaling == TR_SCALE_PARTS && (!(original_len > 0.0) || !isfinite(original_len) || !(slow_turns < fast_turns) || !isfinite(slow_turns) || !isfinite(fast_turns)))
        return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: original_len must be positive and slow_turns below fast_turns");
    tr_rotary r;
    memset(&r, 0, sizeof r);
    r.layout = layout;
    r.rotary_dim = rotary_dim;
    r.amplitude = amplitude;
    const double d = rotary_dim;
    if (scaling == TR_SCALE_BASE && rotary_dim) base *= pow(factor, d / (d - 2.0));
    if (!isfinite(base)) return tr_fail(TR_ERR_INVALID_ARG, "tr_rotary_init: the stretched base is not finite");
    for (int m = 0; m < rotary_dim / 2; ++m) {
        const double theta = pow(base, -2.0 * m / d);
        double f = theta;
        if (scaling == TR_SCALE_LINEAR) f = theta / factor;
        if (scaling == TR_SCALE_PARTS) {
            const double turns = original_len * theta / 6.283185307179586;
            const double c = fmin(fmax((turns - slow_turns) / (fast_turns - slow_turns), 0.0), 1.0);
            f = theta * (c + (1.0 - c) / factor);
        }
        r.freq[m] = f;
    }
    *out = r;
    return TR_OK;
    });
}

extern "C" int tr_paged_append(const tr_shape* shape, const tr_rotary* rotary, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const void* q_norm, const void* k_norm, double eps, const int32_t* pos,
                               const int32_t* slots, int32_t n_tokens, void* q_out, const tr_pages* pages, void* stream)
{
    return tr_guard_int([&]() -> int {
    tr_clear_error();
    const char* const who = "tr_paged_append";
    if (int rc = tr_check_shape(shape)) return rc;
    if (n_tokens < 0) return tr_fail(TR_ERR_INVALID_ARG, "%s: n_tokens < 0", who);
    if (shape->n_q_heads > MOST_HEADS) return tr_fail(TR_ERR_UNSUPPORTED, "%s: %d heads, at most 2^20", who, shape->n_q_heads);
    if ((q != nullptr) != (q_out != nullptr)) return tr_fail(TR_ERR_INVALID_ARG, "%s: q and q_out go together", who);
    const int given = (k != nullptr) + (v != nullptr) + (slots != nullptr) + (pages != nullptr);
    if (n_tokens > 0 && given != 0 && given != 4) return tr_fail(TR_ERR_INVALID_ARG, "%s: k, v, slots and pages go together", who);
    if (!((float)eps >= FLT_MIN) || !isfinite((float)eps)) return tr_fail(TR_ERR_INVALID_ARG, "%s: eps must be finite and a positive normal fp32 value", who);
    TrPagedAppendArgs a;
    memset(&a, 0, sizeof a);
    int layout = shape->rope_layout;
    if (rotary) {
        layout = rotary->layout;
        if (layout != TR_ROPE_INTERLEAVED && layout != TR_ROPE_HALF) return tr_fail(TR_ERR_INVALID_ARG, "%s: layout %d of the rotary", who, layout);
        a.rotary_dim = rotary->rotary_dim;
        if (a.rotary_dim < 0 || a.rotary_dim > shape->head_dim || a.rotary_dim % 16)
            return tr_fail(TR_ERR_SHAPE, "%s: rotary_dim %d is not a multiple of 16 up to head_dim", who, a.rotary_dim);
        if (!isfinite((float)rotary->amplitude)) return tr_fail(TR_ERR_INVALID_ARG, "%s: amplitude must be finite", who);
        a.amplitude = (float)rotary->amplitude;
        for (int m = 0; m < a.rotary_dim / 2; ++m) {
            if (!(rotary->freq[m] >= 0.0 && rotary->freq[m] <= 1.0)) return tr_fail(TR_ERR_INVALID_ARG, "%s: freq[%d] is outside [0, 1]", who, m);
            a.freq[m] = rotary->freq[m];
        }
    } else {
        a.rotary_dim = shape->head_dim;
        a.amplitude = 1.0f;
        tr_fill_theta(shape, a.freq);
    }
    const int64_t e = tr_elem_bytes(shape), q_row = (int64_t)shape->n_q_heads * shape->head_dim, kv_row = (int64_t)shape->n_kv_heads * shape->head_dim;
    if (pages) {
        if (int rc = pool_of(who, shape, pages, &a.pool)) return rc;
        if (!rows_apart(pages)) return tr_fail(TR_ERR_INVALID_ARG, "%s: rows of the pages use the same bytes", who);
    }
    if (n_tokens == 0 || (!q && !k)) return TR_OK;
    if (a.rotary_dim && !pos) return tr_fail(TR_ERR_INVALID_ARG, "%s: pos is NULL", who);
    // tokens may share a row of the input (a stride of 0), they may not overlap in part
    if ((q && (q_stride < 0 || q_stride > INT64_MAX / 8 / n_tokens)) || (k && (k_stride < 0 || k_stride > INT64_MAX / 8 / n_tokens || v_stride < 0 || v_stride > INT64_MAX / 8 / n_tokens)))
        return tr_fail(TR_ERR_INVALID_ARG, "%s: a stride is out of range", who);
    const Span qs = rows(q, n_tokens, q_stride * e, q_row * e), outs = rows(q_out, n_tokens, q_row * e, q_row * e);
    const Span in[] = {rows(k, n_tokens, k_stride * e, kv_row * e), rows(v, n_tokens, v_stride * e, kv_row * e), ints(pos, n_tokens), ints(slots, n_tokens),
                       rows(q_norm, 1, 0, shape->head_dim * e), rows(k_norm, 1, 0, shape->head_dim * e)};
    if (overlap(outs, qs) && !(q == q_out && (n_tokens == 1 || q_stride == q_row)))
        return tr_fail(TR_ERR_INVALID_ARG, "%s: q_out overlaps q without being it (contiguous)", who);
    for (const Span& s : in)
        if (overlap(outs, s)) return tr_fail(TR_ERR_INVALID_ARG, "%s: q_out overlaps an input", who);
    if (pages) {
        for (const Span& pool : {pool_span(a.pool, pages->k, pages), pool_span(a.pool, pages->v, pages)}) {
            for (const Span& s : in)
                if (overlap(pool, s)) return tr_fail(TR_ERR_INVALID_ARG, "%s: the pages overlap an input", who);
            if (overlap(pool, qs) || overlap(pool, outs)) return tr_fail(TR_ERR_INVALID_ARG, "%s: the pages overlap q or q_out", who);
        }
    }
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(q_norm) || !aligned16(k_norm) || (q && q_stride * e % 16) ||
        (k && (k_stride * e % 16 || v_stride * e % 16)))
        return tr_fail(TR_ERR_INVALID_ARG, "%s: tensors and their strides must be 16-byte aligned", who);
    a.q = (const char*)q;
    a.k = (const char*)k;
    a.v = (const char*)v;
    a.q_out = (char*)q_out;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.pos = pos;
    a.slots = slots;
    a.q_stride = q_stride * e;
    a.k_stride = k_stride * e;
    a.v_stride = v_stride * e;
    a.n_tokens = n_tokens;
    a.n_q_heads = q ? shape->n_q_heads : 0;
    a.n_kv_heads = k ? shape->n_kv_heads : 0;
    a.eps = (float)eps;
    // A workgroup takes as many tokens as give its threads eight units each, if there are workgroups enough then.  us for 1 token /
    // this: 24000 rows of 4 KV heads of 128 44.6 / 23.6, 16000 tokens of 16 + 4 heads of 64 47.6 / 23.9, 16001 of 32 + 8 of 128 88.3 / 79.0.
    const int64_t units = (int64_t)(a.n_q_heads + 2 * a.n_kv_heads) * shape->head_dim * e / 16; // of a token
    while ((2 << a.tile_shift) <= TR_PAGED_APPEND_TOKENS && (units << a.tile_shift) * 2 <= 2048 && n_tokens >= 2048ll << a.tile_shift) ++a.tile_shift;
    // Streamed stores make the call itself faster at any size, and what reads its results next slower where the caches still
    // hold them: us of the call and a pass over all it wrote, ordinary / streamed, by MB written: 12 MB 18.6 / 17.9, 25 MB 27.9 / 29.4, 49 MB
    // 45.4 / 46.8, 98 MB 78.4 / 84.1, 197 MB 151.5 / 148.0.
    a.stream = 16 * units * n_tokens >= 150ll << 20;
    return tr_launch_paged_append(a, shape->dtype, shape->head_dim, layout, (hipStream_t)stream);
    });
}

namespace {
// What the pieces of cut items need: sums and statistics of two pieces per worker, and who has pieces of which item.  None of it
// depends on the lengths, which are not known here.
struct DecodePlan {
    int64_t items, bound; // items of the batch; most units that they can have
    int32_t ws_rows;
    size_t ml_at, items_at, bytes;
};
DecodePlan decode_plan(const tr_shape* sh, int64_t n_req, int64_t keys)
{
    DecodePlan p;
    const int group = sh->n_q_heads / sh->n_kv_heads, tile = tr_paged_tile_rows(group);
    p.items = n_req * sh->n_kv_heads * ((group + tile - 1) / tile);
    const int unit = tr_paged_unit_keys(sh->dtype);
    const int64_t units = std::max<int64_t>((keys + unit - 1) / unit, 1);
    p.bound = p.items * units;
    p.ws_rows = std::min(group, tile);
    const bool none = units == 1; // a unit is never cut
    p.ml_at = tr_align256(2ull * TR_PAGED_WORKERS * p.ws_rows * sh->head_dim * 4);
    p.items_at = p.ml_at + tr_align256(2ull * TR_PAGED_WORKERS * p.ws_rows * 8);
    p.bytes = none ? 0 : p.items_at + tr_align256((size_t)std::max<int64_t>(p.items, TR_PAGED_WORKERS) * 8);
    return p;
}
} // namespace

extern "C" size_t tr_paged_decode_attn_workspace_size(const tr_shape* shape, int32_t n_req, int32_t max_blocks, int32_t page_size)
{
    return tr_guard_size([&]() -> size_t {
    tr_clear_error();
    if (tr_check_shape(shape) || n_req < 1 || max_blocks < 1 || page_shift(page_size) < 0) return 0;
    if (n_req > MOST_REQUESTS || (int64_t)n_req * shape->n_q_heads > TR_MAX_BLOCKS_256 || (int64_t)max_blocks * page_size > MOST_KEYS) return 0; // refused
    const DecodePlan plan = decode_plan(shape, n_req, (int64_t)max_blocks * page_size);
    return plan.bound > MOST_UNITS ? 0 : plan.bytes;
    });
}

extern "C" int tr_paged_decode_attn(const tr_shape* shape, const void* q, const tr_pages* pages, const int32_t* block_table, int32_t max_blocks,
                                    const int32_t* kv_lens, int32_t n_req, int32_t window, int32_t n_sink, void* out, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    return tr_guard_int([&]() -> int {
    tr_clear_error();
    const char* const who = "tr_paged_decode_attn";
    if (int rc = tr_check_shape(shape)) return rc;
    if (n_req < 0 || max_blocks < 0 || window < 0 || n_sink < 0) return tr_fail(TR_ERR_INVALID_ARG, "%s: a count is negative", who);
    if (n_req > MOST_REQUESTS) return tr_fail(TR_ERR_UNSUPPORTED, "%s: %d requests, at most %d", who, n_req, MOST_REQUESTS);
    if (!pages) return tr_fail(TR_ERR_INVALID_ARG, "%s: pages is NULL", who);
    TrPagedDecodeArgs a;
    memset(&a, 0, sizeof a);
    if (int rc = pool_of(who, shape, pages, &a.pool)) return rc;
    if ((int64_t)max_blocks * pages->page_size > MOST_KEYS) return tr_fail(TR_ERR_INVALID_ARG, "%s: max_blocks %d", who, max_blocks);
    if ((int64_t)n_req * shape->n_q_heads > TR_MAX_BLOCKS_256) return tr_fail(TR_ERR_UNSUPPORTED, "%s: more than 2^24 (request, head) pairs", who);
    if (n_req == 0) return TR_OK;
    if (!q || !out || !kv_lens || (max_blocks > 0 && !block_table)) return tr_fail(TR_ERR_INVALID_ARG, "%s: an array is NULL", who);
    if (!aligned16(q) || !aligned16(out)) return tr_fail(TR_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned", who);
    const int64_t row = (int64_t)shape->n_q_heads * shape->head_dim * tr_elem_bytes(shape);
    const Span outs = rows(out, n_req, row, row);
    if (overlap(outs, rows(q, n_req, row, row)) && out != q) return tr_fail(TR_ERR_INVALID_ARG, "%s: out overlaps q without being it", who);
    for (const Span& s : {pool_span(a.pool, pages->k, pages), pool_span(a.pool, pages->v, pages), ints(block_table, (int64_t)n_req * max_blocks), ints(kv_lens, n_req)})
        if (overlap(outs, s)) return tr_fail(TR_ERR_INVALID_ARG, "%s: out overlaps the pages, the table or the lengths", who);
    a.q = q;
    a.out = out;
    a.table = block_table;
    a.kv_lens = kv_lens;
    a.n_req = n_req;
    a.max_blocks = max_blocks;
    a.window = window;
    a.n_sink = n_sink;
    a.n_q_heads = shape->n_q_heads;
    a.n_kv_heads = shape->n_kv_heads;
    a.group = shape->n_q_heads / shape->n_kv_heads;
    a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)shape->head_dim));
    const DecodePlan plan = decode_plan(shape, n_req, (int64_t)max_blocks * pages->page_size);
    if (plan.bound > MOST_UNITS) return tr_fail(TR_ERR_UNSUPPORTED, "%s: the table has room for more than 2^30 units of 32 (fp32: 16) keys", who);
    if (plan.bytes) {
        if (!workspace || ((uintptr_t)workspace & 255)) return tr_fail(TR_ERR_WORKSPACE, "%s: workspace missing or not 256-byte aligned", who);
        if (workspace_bytes < plan.bytes) return tr_fail(TR_ERR_WORKSPACE, "%s: workspace holds %zu bytes, %zu needed", who, workspace_bytes, plan.bytes);
        a.ws_o = (float*)workspace;
        a.ws_ml = (float*)((char*)workspace + plan.ml_at);
        a.ws_items = (int32_t*)((char*)workspace + plan.items_at);
    }
    a.ws_rows = plan.ws_rows;
    const int64_t workers = std::min<int64_t>((plan.bound + TR_PAGED_MIN_UNITS - 1) / TR_PAGED_MIN_UNITS, TR_PAGED_WORKERS);
    // The join's workgroups, most of which find nothing to do, are what it costs: it looks at the rows of the result or at those
    // that each wave may have cut, whichever are fewer.  us of the whole call by row / by wave: 200 requests of 50 to 1200 rows, 32 / 8
    // heads (6400 rows or 4096) 102.7 / 101.1, 512 of 256 (16384 or 4096) 96.2 / 93.4, 4096 of 10 to 60, 16 / 4 heads of 64 (65536 or 4096)
    // 92.7 / 78.7.
    if (plan.bytes) a.cut = (int64_t)n_req * shape->n_q_heads <= workers * plan.ws_rows ? TR_PAGED_JOIN_BY_ROW : TR_PAGED_JOIN_BY_WAVE;
    return tr_launch_paged_decode(a, shape->dtype, shape->head_dim, (int)workers, (hipStream_t)stream);
    });
}
