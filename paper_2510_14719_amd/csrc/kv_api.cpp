// Host side of the C ABI declared in include/kv_cache.h: argument validation (no HIP call is made before the arguments are
// known to be good, so the error paths run on a machine without a GPU) and dispatch to the kernel launchers.
#include "kv_cache.h"

#include <cmath>
#include <cstdint>

#include "paged_launch.h"

namespace {

typedef long long i64;

// Memory that an operand touches, [first, last) in bytes.
struct Extent {
    std::uintptr_t first, last;
};
bool overlaps(Extent a, Extent b) { return a.first < b.last && b.first < a.last; }
bool overlaps_any(Extent a, const Extent* b, int n)
{
    for (int i = 0; i < n; ++i)
        if (overlaps(a, b[i])) return true;
    return false;
}
Extent flat(const void* p, i64 bytes) { const auto a = reinterpret_cast<std::uintptr_t>(p); return {a, a + (std::uintptr_t)bytes}; }

struct Dim {
    i64 size, stride;                           // of rows of d elements
};

// Checks rows of d elements with `es` bytes each and gives their extent.  Every stride of a dimension larger than one is at least d (`shared`: 0 is
// allowed too, for what is only read) and a multiple of 16 bytes.  `apart`: the rows must not meet, whatever order the dimensions lie in.
int check_rows(const void* p, const Dim* dims, int n, int d, int es, bool shared, bool apart, Extent& e)
{
    if (!p) return KV_ERR_NULL;
    if (reinterpret_cast<std::uintptr_t>(p) & 15u) return KV_ERR_ALIGN;
    const i64 LIMIT = 1ll << 47;                // bytes; the address space of the device
    i64 span = d;
    for (int i = 0; i < n; ++i) {
        if (dims[i].size == 1) continue;
        const i64 s = dims[i].stride;
        if (s * es % 16) return KV_ERR_ALIGN;
        if (s < d && !(shared && s == 0)) return KV_ERR_STRIDE;
        if (s > LIMIT / es / dims[i].size) return KV_ERR_OVERFLOW;
        span += (dims[i].size - 1) * s;
    }
    if (span > LIMIT / es) return KV_ERR_OVERFLOW;
    if (apart) {                                // each stride steps over all that lies inside it
        bool done[4] = {};
        i64 inside = d;
        for (int k = 0; k < n; ++k) {
            int least = -1;
            for (int i = 0; i < n; ++i)
                if (!done[i] && dims[i].size > 1 && (least < 0 || dims[i].stride < dims[least].stride)) least = i;
            if (least < 0) break;
            if (dims[least].stride < inside) return KV_ERR_STRIDE;
            inside += (dims[least].size - 1) * dims[least].stride;
            done[least] = true;
        }
    }
    e = flat(p, span * es);
    return KV_OK;
}

// Whether rows of d elements, `dims` of them from one address, meet the same rows from an address `diff` elements on.  Dimension by dimension from the longest stride: two rows
// can only meet where their distance is no longer than what lies inside that stride.  (Strides that do not step over what lies inside them: taken to meet.)
bool rows_meet(const Dim* dims, int n, i64 d, i64 diff)
{
    const Dim* by[4];
    int count = 0;
    for (int i = 0; i < n; ++i)
        if (dims[i].size > 1) by[count++] = &dims[i];
    for (int i = 1; i < count; ++i)
        for (int k = i; k > 0 && by[k - 1]->stride < by[k]->stride; --k) { const Dim* const t = by[k]; by[k] = by[k - 1]; by[k - 1] = t; }
    i64 inside[4], reach = d - 1;               // between the first element and the last of what lies inside a stride
    for (int i = count - 1; i >= 0; --i) {
        inside[i] = reach;
        if (by[i]->stride <= reach) return true;
        reach += (by[i]->size - 1) * by[i]->stride;
    }
    i64 left[16] = {diff};                      // distances that are left: at most two for each one before
    int lefts = 1;
    for (int i = 0; i < count; ++i) {
        i64 next[16];
        int nexts = 0;
        for (int k = 0; k < lefts; ++k) {
            const i64 s = by[i]->stride, low = left[k] / s - (left[k] % s < 0);
            for (i64 step = low; step <= low + 1; ++step)
                if (step > -by[i]->size && step < by[i]->size && left[k] - step * s <= inside[i] && step * s - left[k] <= inside[i]) next[nexts++] = left[k] - step * s;
        }
        for (int k = 0; k < nexts; ++k) left[k] = next[k];
        lefts = nexts;
    }
    for (int k = 0; k < lefts; ++k)
        if (left[k] < d && left[k] > -d) return true;
    return false;
}

bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<std::uintptr_t>(p) & (to - 1)) != 0; }
bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2_of(int x) { int n = 0; while (x > 1) { x /= 2; ++n; } return n; }

// The cache, its layers in reach of the call (one, or all), and the extents of k and v.
int check_cache(const kv_pages* c, bool all_layers, bool scales, Extent* e)
{
    if (!c) return KV_ERR_NULL;
    if (!c->k || !c->v) return KV_ERR_NULL;
    if (c->layers < 1 || c->pages < 1 || c->heads < 1 || (c->d != 64 && c->d != 128)) return KV_ERR_SHAPE;
    if (!pow2(c->page_size) || c->page_size < 16 || c->page_size > 4096) return KV_ERR_SHAPE;
    if (c->dtype != KV_FP16 && c->dtype != KV_BF16 && c->dtype != KV_E4M3) return KV_ERR_SHAPE;
    if (scales && (c->k_scale != nullptr) != (c->v_scale != nullptr)) return KV_ERR_NULL;
    if (scales && c->k_scale && c->dtype != KV_E4M3) return KV_ERR_SHAPE;
    if (scales && (misaligned(c->k_scale, 4) || misaligned(c->v_scale, 4))) return KV_ERR_ALIGN;
    const int es = c->dtype == KV_E4M3 ? 1 : 2;
    const Dim dims[4] = {{all_layers ? c->layers : 1, c->layer_stride}, {c->pages, c->page_stride}, {c->heads, c->head_stride}, {c->page_size, c->token_stride}};
    for (int i = 0; i < 2; ++i) {
        const int rc = check_rows(i ? c->v : c->k, dims, 4, c->d, es, false, false, e[i]);
        if (rc != KV_OK) return rc;
    }
    if (c->heads > (1 << 16) || (i64)c->heads * c->page_size * c->d >= (1ll << 31)) return KV_ERR_OVERFLOW;
    // (inside a page the kernels count in 32 bits)
    if (c->token_stride * c->page_size * es >= (1ll << 31)) return KV_ERR_OVERFLOW;
    if (c->k == c->v) return KV_ERR_ALIAS;
    return KV_OK;
}

// A cache that is written: keys and values must not meet.
bool cache_meets(const kv_pages* c, bool all_layers, const Extent* e)
{
    if (!overlaps(e[0], e[1])) return false;
    const int es = c->dtype == KV_E4M3 ? 1 : 2;
    const Dim dims[4] = {{all_layers ? c->layers : 1, c->layer_stride}, {c->pages, c->page_stride}, {c->heads, c->head_stride}, {c->page_size, c->token_stride}};
    return rows_meet(dims, 4, c->d, ((i64)e[1].first - (i64)e[0].first) / es);   // (both are multiples of 16 bytes)
}

// What a call reads beside its rows: the batch's arrays, the scales of the cache, frequencies.
int side_inputs(const kv_pages* c, const kv_batch* b, const double* freq, int rot, Extent* e)
{
    e[0] = flat(b->q_start, 4ll * (b->sequences + 1ll));
    e[1] = flat(b->kv_len, 4ll * b->sequences);
    e[2] = flat(b->table, ((b->sequences - 1ll) * b->table_stride + b->table_width) * 4);
    int n = 3;
    if (c->k_scale) {
        e[n++] = flat(c->k_scale, 4ll * c->heads);
        e[n++] = flat(c->v_scale, 4ll * c->heads);
    }
    if (freq) e[n++] = flat(freq, rot / 2 * 8ll);
    return n;
}

int check_batch(const kv_batch* b, const kv_pages* c)
{
    if (!b) return KV_ERR_NULL;
    if (!b->q_start || !b->kv_len || !b->table) return KV_ERR_NULL;
    if (b->sequences < 1 || b->tokens < 1 || b->table_width < 1 || b->max_q < 1 || b->max_kv < 1) return KV_ERR_SHAPE;
    if ((i64)b->table_width * c->page_size < b->max_kv) return KV_ERR_SHAPE;
    if (b->sequences > 1 && b->table_stride < b->table_width) return KV_ERR_STRIDE;
    if (misaligned(b->q_start, 4) || misaligned(b->kv_len, 4) || misaligned(b->table, 4)) return KV_ERR_ALIGN;
    // (positions and row numbers are 32-bit)
    if (b->max_kv > (1 << 30) || b->tokens > (1 << 30)) return KV_ERR_OVERFLOW;
    return KV_OK;
}

int check_tokens(const kv_rows* r, int tokens, int heads, int d, bool written, Extent& e)
{
    if (!r) return KV_ERR_NULL;
    const Dim dims[2] = {{tokens, r->token_stride}, {heads, r->head_stride}};
    return check_rows(r->p, dims, 2, d, 2, !written, written, e);
}

bool sixteen(int dtype) { return dtype == KV_FP16 || dtype == KV_BF16; }
int max_q_of(const kv_batch* b) { return b->max_q < b->tokens ? b->max_q : b->tokens; }

// Two sets of rows that lie in each other's gaps: slices of the heads of one array of tokens.
bool interleaved(const kv_rows* a, int heads_a, const kv_rows* b, int heads_b, int d)
{
    const i64 ts = a->token_stride * 2, span_a = ((heads_a - 1) * (heads_a > 1 ? a->head_stride : 0) + d) * 2, span_b = ((heads_b - 1) * (heads_b > 1 ? b->head_stride : 0) + d) * 2;
    if (a->token_stride != b->token_stride || span_a > ts || span_b > ts) return false;
    const i64 diff = (i64)reinterpret_cast<std::uintptr_t>(b->p) - (i64)reinterpret_cast<std::uintptr_t>(a->p), at = (diff % ts + ts) % ts;
    return at >= span_a && at + span_b <= ts;
}

bool attn_sizes_ok(const kv_pages* c, int heads)
{
    return heads >= 1 && heads <= (1 << 16) && heads % c->heads == 0;
}
PagedPlan plan_of(const kv_pages* c, const kv_batch* b, int heads)
{
    return paged_plan(b->sequences, b->tokens, max_q_of(b), b->max_kv, heads, c->heads, c->d, c->dtype == KV_E4M3 ? 1 : 2);
}
// Partial results of the small tiles (see PagedArgs): d + 4 floats a slot (O, reference, two sums, padding: a multiple of 16 bytes, as what stands behind them is read
// 16 bytes at a time).  Sequences that go by chunks have none of them, however many tokens they have.
struct FewParts {
    i64 rows, slots;
    int most;                                   // as PagedArgs::part_most
};
FewParts few_parts(const PagedPlan& p, const kv_pages* c, const kv_batch* b, int heads)
{
    if (p.splits <= 1) return {0, 0, 0};
    if (p.few_room > 0) return {0, (i64)p.few_room * c->heads * p.rows, 0};
    const i64 rows = (i64)max_q_of(b) * (heads / c->heads), tiles = (i64)p.row_tiles * p.rows, most = rows < tiles ? rows : tiles;
    const i64 by_token = (i64)b->tokens * heads, by_sequence = (i64)b->sequences * c->heads * most;
    return by_sequence < by_token ? FewParts{by_sequence, by_sequence * p.splits, (int)most} : FewParts{by_token, by_token * p.splits, 0};
}
i64 few_first_bytes(const PagedPlan& p, const kv_batch* b) { return p.splits > 1 && p.few_room > 0 ? ((i64)b->sequences * p.row_tiles + 3) / 4 * 16 : 0; }
i64 workspace_of(const PagedPlan& p, const kv_pages* c, const kv_batch* b, int heads)
{
    return (few_parts(p, c, b, heads).slots + (i64)p.chunk_parts * PAGED_CHUNK_ROWS) * (c->d + 4) * 4 + (p.chunk_parts ? (p.chunk_parts + 1) * 16ll : 0) + (p.splits > 1 ? 16 : 0) + few_first_bytes(p, b);
}
bool grid_ok(const PagedPlan& p, const kv_pages* c, const kv_batch* b, int heads)
{
    const i64 most = 1ll << 23;                 // workgroups of 512 threads: a grid has less than 2^32
    auto fits = [&](i64 tiles, i64 splits) { return tiles < most && tiles * splits < most && tiles * splits * c->heads < most; };
    return fits((i64)p.splits * p.row_tiles, b->sequences) && p.chunk_tiles < most && fits((i64)b->sequences * p.row_tiles, p.rows);
}

void book_arrays(const kv_book* b, Extent* e)
{
    e[0] = flat(b->table, ((i64)(b->rows - 1) * (b->rows > 1 ? b->table_stride : 0) + b->table_width) * 4);
    e[1] = flat(b->ref, 4ll * b->pages);
    e[2] = flat(b->kv_len, 4ll * b->rows);
}
int check_book(const kv_book* b)
{
    if (!b) return KV_ERR_NULL;
    if (!b->ref || !b->table || !b->kv_len) return KV_ERR_NULL;
    if (b->pages < 1 || b->rows < 1 || b->table_width < 1 || !pow2(b->page_size) || b->page_size < 16 || b->page_size > 4096) return KV_ERR_SHAPE;
    if (b->rows > 1 && b->table_stride < b->table_width) return KV_ERR_STRIDE;
    if (misaligned(b->ref, 4) || misaligned(b->table, 4) || misaligned(b->kv_len, 4)) return KV_ERR_ALIGN;
    if (b->pages > (1 << 28) || (i64)b->table_width * b->page_size >= (1ll << 31) || (i64)b->rows * b->table_stride >= (1ll << 46)) return KV_ERR_OVERFLOW;
    Extent e[3];
    book_arrays(b, e);
    if (overlaps(e[0], e[1]) || overlaps(e[0], e[2]) || overlaps(e[1], e[2])) return KV_ERR_ALIAS;
    return KV_OK;
}
// Whether something of so many ints overlaps one of the arrays.
bool ints_overlap(const int* p, i64 n, const Extent* e, int count) { return n > 0 && overlaps_any(flat(p, 4 * n), e, count); }
int check_list(const int* list, int n)
{
    if (n < 0 || n > KV_MAX_LIST) return KV_ERR_SHAPE;
    if (n > 0 && !list) return KV_ERR_NULL;
    return misaligned(list, 4) ? KV_ERR_ALIGN : KV_OK;
}
int check_copy(const kv_pages* c, Extent* e)
{
    const int rc = check_cache(c, true, false, e);
    if (rc != KV_OK) return rc;
    if (cache_meets(c, true, e)) return KV_ERR_ALIAS;
    return (i64)c->layers * 2 * ((i64)c->heads * c->page_size * c->d / 16384 + 1) >= (1ll << 23) ? KV_ERR_OVERFLOW : KV_OK;
}
PageCopy copy_of(const kv_pages* c)
{
    const int es = c->dtype == KV_E4M3 ? 1 : 2;
    const i64 d = c->d, ts = c->page_size > 1 ? c->token_stride : d, hs = c->heads > 1 ? c->head_stride : d * c->page_size;
    const bool solid = (ts == d && hs == d * c->page_size) || (hs == d && ts == d * c->heads) || (c->heads == 1 && ts == d);
    return {(char*)c->k, (char*)c->v, c->layer_stride * es, c->page_stride * es, c->head_stride * es, c->token_stride * es,
            c->layers, c->pages, c->heads, c->page_size, c->d * es, solid};
}
bool same_pages(const kv_pages* c, const kv_book* b) { return c->pages == b->pages && c->page_size == b->page_size; }
int launched(int rc) { return rc == 0 ? KV_OK : KV_ERR_LAUNCH; }

}  // namespace

extern "C" {

int attn_paged_check_args(const kv_pages* cache, const kv_batch* batch, const kv_rows* q, const kv_rows* o, const float* lse, int heads, float scale,
                          int dtype, const void* workspace, long long workspace_bytes)
{
    Extent in[3], eo;
    int rc = check_cache(cache, false, true, in);
    if (rc != KV_OK) return rc;
    if ((rc = check_batch(batch, cache)) != KV_OK) return rc;
    if (!sixteen(dtype) || (cache->dtype != KV_E4M3 && cache->dtype != dtype) || !attn_sizes_ok(cache, heads)) return KV_ERR_SHAPE;
    if (!std::isfinite(scale) || !(scale > 0.0f)) return KV_ERR_SCALE;
    if ((rc = check_tokens(q, batch->tokens, heads, cache->d, false, in[2])) != KV_OK) return rc;
    if ((rc = check_tokens(o, batch->tokens, heads, cache->d, true, eo)) != KV_OK) return rc;
    if (misaligned(lse, 4)) return KV_ERR_ALIGN;
    const PagedPlan p = plan_of(cache, batch, heads);
    if (!grid_ok(p, cache, batch, heads)) return KV_ERR_OVERFLOW;
    const i64 need = workspace_of(p, cache, batch, heads);
    if (need > 0) {
        if (!workspace) return KV_ERR_NULL;
        if (misaligned(workspace, 16)) return KV_ERR_ALIGN;
        if (workspace_bytes < need) return KV_ERR_WORKSPACE;
    }
    if (overlaps_any(eo, in, 2)) return KV_ERR_ALIAS;
    if (overlaps(eo, in[2]) && !interleaved(q, heads, o, heads, cache->d)) return KV_ERR_ALIAS;
    const Extent el = flat(lse, 4ll * batch->tokens * heads), ew = flat(workspace, need);
    if (lse && (overlaps(el, eo) || overlaps_any(el, in, 3))) return KV_ERR_ALIAS;
    if (need > 0 && (overlaps(ew, eo) || overlaps_any(ew, in, 3) || (lse && overlaps(ew, el)))) return KV_ERR_ALIAS;
    Extent side[6];
    const int sides = side_inputs(cache, batch, nullptr, 0, side);
    if (overlaps_any(eo, side, sides) || (lse && overlaps_any(el, side, sides)) || (need > 0 && overlaps_any(ew, side, sides))) return KV_ERR_ALIAS;
    return KV_OK;
}

int attn_paged(const kv_pages* cache, const kv_batch* batch, const kv_rows* q, const kv_rows* o, float* lse, int heads, float scale, int causal,
               int dtype, void* workspace, long long workspace_bytes, void* stream)
{
    const int rc = attn_paged_check_args(cache, batch, q, o, lse, heads, scale, dtype, workspace, workspace_bytes);
    if (rc != KV_OK) return rc;
    const PagedPlan p = plan_of(cache, batch, heads);
    const int es = cache->dtype == KV_E4M3 ? 1 : 2;
    PagedArgs a{};
    a.k = (const char*)cache->k;
    a.v = (const char*)cache->v;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    a.page_bytes = cache->page_stride * es;
    a.head_bytes = cache->head_stride * es;
    a.token_bytes = cache->token_stride * es;
    a.q_start = batch->q_start;
    a.kv_len = batch->kv_len;
    a.table = batch->table;
    a.q = (const char*)q->p;
    a.o = (char*)o->p;
    a.lse = lse;
    a.q_token = q->token_stride * 2;
    a.q_head = q->head_stride * 2;
    a.o_token = o->token_stride * 2;
    a.o_head = o->head_stride * 2;
    const FewParts parts = few_parts(p, cache, batch, heads);
    const i64 few = parts.slots, chunk = (i64)p.chunk_parts * PAGED_CHUNK_ROWS;
    a.part_o = (float*)workspace;
    a.chunk_o = a.part_o + few * cache->d;
    a.part_ml = a.chunk_o + chunk * cache->d;
    a.chunk_ml = a.part_ml + few * 4;
    a.chunk_what = (int*)(a.chunk_ml + chunk * 4);
    a.few_inverse = (float*)(a.chunk_what + (p.chunk_parts ? (p.chunk_parts + 1) * 4 : 0));
    a.part_rows = parts.rows;
    a.part_most = parts.most;
    a.few_first = few_first_bytes(p, batch) > 0 ? (int*)(a.few_inverse + 4) : nullptr;
    a.sequences = batch->sequences;
    a.tokens = batch->tokens;
    a.table_stride = batch->table_stride;
    a.max_q = max_q_of(batch);
    a.max_kv = batch->max_kv;
    a.pages = cache->pages;
    a.page_shift = log2_of(cache->page_size);
    a.heads = heads;
    a.group = heads / cache->heads;
    a.causal = causal != 0;
    a.few_rows = p.few_rows;
    a.rows = p.rows;
    a.row_tiles = p.row_tiles;
    // Pieces of a fixed length are numbered through on the device too where sequences are far shorter than the bound: that costs 4 us in 200, an empty workgroup 2 ns (one token each of 64
    // sequences of 300 ... 16384, 32 heads on 8, d 128, bound as it is / 2 / 8 / 32 times that, us numbered 209 / 209 / 210 / 210, else 205 / 206 / 243 / 441).  All tokens lie in
    // pages, so unless sequences share pages there are no more pieces than this (if they do, the length grows).
    const i64 row_tiles = (i64)batch->sequences * p.row_tiles, room = row_tiles + p.row_tiles * ((i64)cache->pages * cache->page_size / p.split);
    const bool fixed = p.splits > 1 && p.few_room == 0 && room * 6 < row_tiles * p.splits;
    a.few_room = fixed ? (int)room : p.few_room;
    a.few_fixed = fixed;
    a.few_finest = 1.f / (float)p.split;
    const int longest = fixed ? batch->max_kv : p.split_max;
    a.few_coarsest = a.few_room ? 1.f / (float)longest : 0.f;
    a.few_step = a.few_room ? std::log2((float)longest / (float)p.split) / 63.f : 0.f;
    a.split = p.split;
    a.splits = p.splits;
    a.chunk_parts = p.chunk_parts;
    a.scale = scale;
    return launched(attn_paged_launch(a, p, cache->d, dtype, cache->dtype, stream));
}

long long attn_paged_workspace(const kv_pages* cache, const kv_batch* batch, int heads)
{
    if (!cache || !batch || cache->heads < 1 || (cache->d != 64 && cache->d != 128) || batch->sequences < 1 || batch->tokens < 1 || batch->max_q < 1 ||
        batch->max_kv < 1 || batch->max_kv > (1 << 30) || batch->tokens > (1 << 30) || !attn_sizes_ok(cache, heads)) return -1;
    const PagedPlan p = plan_of(cache, batch, heads);
    return grid_ok(p, cache, batch, heads) ? workspace_of(p, cache, batch, heads) : -1;
}

int rope_check_args(const rope_tensor* x, const rope_tensor* y, int batches, int heads, int tokens, int d, const int* pos, long long pos_stride,
                    const double* freq, int rot, int layout, float amplitude, int dtype)
{
    if (!x || !y || !x->p || !y->p || !freq) return KV_ERR_NULL;
    if (batches < 1 || heads < 1 || tokens < 1 || d < 16 || d > 1024 || d % 16 || rot < 16 || rot > d || rot % 16) return KV_ERR_SHAPE;
    if ((layout != KV_HALF && layout != KV_INTERLEAVED) || !sixteen(dtype)) return KV_ERR_SHAPE;
    if (!std::isfinite(amplitude)) return KV_ERR_SCALE;
    if (misaligned(pos, 4) || misaligned(freq, 8)) return KV_ERR_ALIGN;
    if (pos && pos_stride != 0 && pos_stride < tokens) return KV_ERR_STRIDE;
    Extent ex, ey;
    const Dim dx[3] = {{batches, x->batch_stride}, {heads, x->head_stride}, {tokens, x->token_stride}};
    const Dim dy[3] = {{batches, y->batch_stride}, {heads, y->head_stride}, {tokens, y->token_stride}};
    int rc = check_rows(x->p, dx, 3, d, 2, true, false, ex);
    if (rc != KV_OK) return rc;
    if ((rc = check_rows(y->p, dy, 3, d, 2, false, true, ey)) != KV_OK) return rc;
    if (heads > (1 << 16) || ((i64)tokens + 15) / 16 * batches >= (1ll << 24)) return KV_ERR_OVERFLOW;
    const bool in_place = x->p == y->p && (batches == 1 || x->batch_stride == y->batch_stride) && (heads == 1 || x->head_stride == y->head_stride) &&
                          (tokens == 1 || x->token_stride == y->token_stride);
    if (!in_place && overlaps(ex, ey)) return KV_ERR_ALIAS;
    const Extent ep = flat(pos, ((i64)(batches - 1) * pos_stride + tokens) * 4), ef = flat(freq, rot / 2 * 8ll);
    if ((pos && overlaps(ep, ey)) || overlaps(ef, ey)) return KV_ERR_ALIAS;
    return KV_OK;
}

int rope(const rope_tensor* x, const rope_tensor* y, int batches, int heads, int tokens, int d, const int* pos, long long pos_stride,
         const double* freq, int rot, int layout, float amplitude, int inverse, int dtype, void* stream)
{
    const int rc = rope_check_args(x, y, batches, heads, tokens, d, pos, pos_stride, freq, rot, layout, amplitude, dtype);
    if (rc != KV_OK) return rc;
    const RopeArgs a{(const char*)x->p, (char*)y->p, pos, freq, x->batch_stride * 2, x->head_stride * 2, x->token_stride * 2,
                     y->batch_stride * 2, y->head_stride * 2, y->token_stride * 2, pos_stride, batches, heads, tokens, d, rot, layout,
                     amplitude, inverse ? -amplitude : amplitude};
    return launched(rope_launch(a, dtype, stream));
}

int rope_frequencies(double* freq, int rot, double base, int scaling, double factor, double trained, double low, double high)
{
    if (!freq) return KV_ERR_NULL;
    if (rot < 2 || rot > 1024 || rot % 2 || !std::isfinite(base) || !(base > 1)) return KV_ERR_SHAPE;
    if (scaling < ROPE_PLAIN || scaling > ROPE_PARTS) return KV_ERR_SHAPE;
    if (scaling != ROPE_PLAIN && (!std::isfinite(factor) || !(factor >= 1))) return KV_ERR_SHAPE;
    if (scaling == ROPE_BASE && rot <= 2) return KV_ERR_SHAPE;
    if (scaling == ROPE_PARTS && (!std::isfinite(trained) || !(trained > 0) || !(low >= 0) || !(high > low) || !std::isfinite(high))) return KV_ERR_SHAPE;
    if (scaling == ROPE_BASE) base *= std::pow(factor, (double)rot / (rot - 2));
    for (int m = 0; m < rot / 2; ++m) {
        const double f = std::pow(base, -2.0 * m / rot);
        if (scaling == ROPE_LINEAR) freq[m] = f / factor;
        else if (scaling == ROPE_PARTS) {
            const double turns = trained * f / (2 * 3.14159265358979323846);
            const double keep = turns >= high ? 1 : turns <= low ? 0 : (turns - low) / (high - low);
            freq[m] = f * keep + f / factor * (1 - keep);
        } else freq[m] = f;
    }
    return KV_OK;
}

int kv_append_check_args(const kv_pages* cache, const kv_batch* batch, const kv_rows* k, const kv_rows* v, const kv_rows* q, const kv_rows* q_out,
                         int heads, const double* freq, int rot, int layout, float amplitude, int dtype)
{
    Extent out[3], in[3];
    int rc = check_cache(cache, false, true, out);
    if (rc != KV_OK) return rc;
    if ((rc = check_batch(batch, cache)) != KV_OK) return rc;
    const bool has_q = q && q->p, has_out = q_out && q_out->p;
    if (has_q != has_out || (has_q && !freq)) return KV_ERR_NULL;
    if (!sixteen(dtype) || (cache->dtype != KV_E4M3 && cache->dtype != dtype)) return KV_ERR_SHAPE;
    if (freq ? rot < 16 || rot > cache->d || rot % 16 || (layout != KV_HALF && layout != KV_INTERLEAVED) : rot != 0) return KV_ERR_SHAPE;
    if (has_q && heads < 1) return KV_ERR_SHAPE;
    if (freq && !std::isfinite(amplitude)) return KV_ERR_SCALE;
    if (misaligned(freq, 8)) return KV_ERR_ALIGN;
    if ((rc = check_tokens(k, batch->tokens, cache->heads, cache->d, false, in[0])) != KV_OK) return rc;
    if ((rc = check_tokens(v, batch->tokens, cache->heads, cache->d, false, in[1])) != KV_OK) return rc;
    int ins = 2;
    bool in_place = false;
    if (has_q) {
        if ((rc = check_tokens(q, batch->tokens, heads, cache->d, false, in[2])) != KV_OK) return rc;
        if ((rc = check_tokens(q_out, batch->tokens, heads, cache->d, true, out[2])) != KV_OK) return rc;
        ins = 3;
        in_place = q->p == q_out->p && (batch->tokens == 1 || q->token_stride == q_out->token_stride) && (heads == 1 || q->head_stride == q_out->head_stride);
        if (heads > (1 << 16)) return KV_ERR_OVERFLOW;
    }
    if (((i64)batch->tokens + 15) / 16 >= (1ll << 24)) return KV_ERR_OVERFLOW;
    for (int i = 0; i < 2; ++i)
        if (overlaps_any(out[i], in, ins)) return KV_ERR_ALIAS;
    if (has_q) {
        if (overlaps(out[2], in[2]) && !in_place && !interleaved(q, heads, q_out, heads, cache->d)) return KV_ERR_ALIAS;
        const kv_rows* const kv[2] = {k, v};
        for (int i = 0; i < 2; ++i)
            if (overlaps(out[2], in[i]) && !interleaved(q_out, heads, kv[i], cache->heads, cache->d)) return KV_ERR_ALIAS;
    }
    if (has_q && (overlaps(out[2], out[0]) || overlaps(out[2], out[1]))) return KV_ERR_ALIAS;
    Extent side[6];
    const int sides = side_inputs(cache, batch, freq, rot, side);
    for (int i = 0; i < (has_q ? 3 : 2); ++i)
        if (overlaps_any(out[i], side, sides)) return KV_ERR_ALIAS;
    if (cache_meets(cache, false, out)) return KV_ERR_ALIAS;
    return KV_OK;
}

int kv_append(const kv_pages* cache, const kv_batch* batch, const kv_rows* k, const kv_rows* v, const kv_rows* q, const kv_rows* q_out, int heads,
              const double* freq, int rot, int layout, float amplitude, int dtype, void* stream)
{
    const int rc = kv_append_check_args(cache, batch, k, v, q, q_out, heads, freq, rot, layout, amplitude, dtype);
    if (rc != KV_OK) return rc;
    const int es = cache->dtype == KV_E4M3 ? 1 : 2;
    const bool has_q = q && q->p;
    AppendArgs a{};
    a.k_cache = (char*)cache->k;
    a.v_cache = (char*)cache->v;
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    a.page_bytes = cache->page_stride * es;
    a.head_bytes = cache->head_stride * es;
    a.token_bytes = cache->token_stride * es;
    a.q_start = batch->q_start;
    a.kv_len = batch->kv_len;
    a.table = batch->table;
    a.k = (const char*)k->p;
    a.v = (const char*)v->p;
    a.freq = freq;
    a.k_token = k->token_stride * 2;
    a.k_head = k->head_stride * 2;
    a.v_token = v->token_stride * 2;
    a.v_head = v->head_stride * 2;
    if (has_q) {
        a.q = (const char*)q->p;
        a.q_out = (char*)q_out->p;
        a.q_token = q->token_stride * 2;
        a.q_head = q->head_stride * 2;
        a.o_token = q_out->token_stride * 2;
        a.o_head = q_out->head_stride * 2;
        a.heads = heads;
    }
    a.sequences = batch->sequences;
    a.tokens = batch->tokens;
    a.table_stride = batch->table_stride;
    a.max_q = max_q_of(batch);
    a.max_kv = batch->max_kv;
    a.pages = cache->pages;
    a.page_shift = log2_of(cache->page_size);
    a.key_heads = cache->heads;
    a.d = cache->d;
    a.rot = rot;
    a.layout = layout;
    a.amplitude = amplitude;
    return launched(kv_append_launch(a, dtype, cache->dtype, stream));
}

int kv_reserve(const kv_book* book, const int* list, const int* new_len, int n, int* missing, void* stream)
{
    int rc = check_book(book);
    if (rc != KV_OK) return rc;
    if ((rc = check_list(list, n)) != KV_OK || (rc = check_list(new_len, n)) != KV_OK) return rc;
    if (!missing) return KV_ERR_NULL;
    if (misaligned(missing, 4)) return KV_ERR_ALIGN;
    if ((i64)n * book->table_width >= (1ll << 31)) return KV_ERR_OVERFLOW;       // (wants are counted in 32 bits)
    Extent e[5];
    book_arrays(book, e);
    if (ints_overlap(list, n, e, 3) || ints_overlap(new_len, n, e, 3)) return KV_ERR_ALIAS;
    e[3] = flat(list, 4ll * n);
    e[4] = flat(new_len, 4ll * n);
    if (ints_overlap(missing, 1, e, n > 0 ? 5 : 3)) return KV_ERR_ALIAS;
    return launched(kv_reserve_launch(*book, list, new_len, n, missing, stream));
}

int kv_free(const kv_book* book, const int* list, int n, void* stream)
{
    int rc = check_book(book);
    if (rc != KV_OK) return rc;
    if ((rc = check_list(list, n)) != KV_OK) return rc;
    Extent e[3];
    book_arrays(book, e);
    if (ints_overlap(list, n, e, 3)) return KV_ERR_ALIAS;
    return n == 0 ? KV_OK : launched(kv_free_launch(*book, list, n, stream));
}

int kv_fork(const kv_pages* cache, const kv_book* book, const int* src, const int* dst, int n, int* missing, void* stream)
{
    Extent e[7];                                // the book, the cache, the lists
    int rc = check_copy(cache, e + 3);
    if (rc != KV_OK || (rc = check_book(book)) != KV_OK) return rc;
    if ((rc = check_list(src, n)) != KV_OK || (rc = check_list(dst, n)) != KV_OK) return rc;
    if (!missing) return KV_ERR_NULL;
    if (misaligned(missing, 4)) return KV_ERR_ALIGN;
    if (!same_pages(cache, book)) return KV_ERR_SHAPE;
    book_arrays(book, e);
    if (ints_overlap(src, n, e, 5) || ints_overlap(dst, n, e, 5) || overlaps_any(e[3], e, 3) || overlaps_any(e[4], e, 3)) return KV_ERR_ALIAS;
    e[5] = flat(src, 4ll * n);
    e[6] = flat(dst, 4ll * n);
    if (ints_overlap(missing, 1, e, n > 0 ? 7 : 5)) return KV_ERR_ALIAS;
    return launched(kv_fork_launch(copy_of(cache), *book, src, dst, n, missing, stream));
}

long long kv_compact_workspace(int pages) { return pages < 1 || pages > (1 << 28) ? -1 : (2ll * pages + 8) * 4; }

int kv_compact(const kv_pages* cache, const kv_book* book, void* workspace, long long workspace_bytes, void* stream)
{
    Extent e[5];                                // the book, the cache
    int rc = check_copy(cache, e + 3);
    if (rc != KV_OK || (rc = check_book(book)) != KV_OK) return rc;
    if (!workspace) return KV_ERR_NULL;
    if (misaligned(workspace, 16)) return KV_ERR_ALIGN;
    if (!same_pages(cache, book)) return KV_ERR_SHAPE;
    if (workspace_bytes < kv_compact_workspace(book->pages)) return KV_ERR_WORKSPACE;
    book_arrays(book, e);
    if (overlaps_any(flat(workspace, kv_compact_workspace(book->pages)), e, 5) || overlaps_any(e[3], e, 3) || overlaps_any(e[4], e, 3)) return KV_ERR_ALIAS;
    return launched(kv_compact_launch(copy_of(cache), *book, (int*)workspace, stream));
}

int kv_copy_pages(const kv_pages* cache, const int* src, const int* dst, int n, void* stream)
{
    Extent e[2];
    int rc = check_copy(cache, e);
    if (rc != KV_OK) return rc;
    if ((rc = check_list(src, n)) != KV_OK || (rc = check_list(dst, n)) != KV_OK) return rc;
    if (ints_overlap(src, n, e, 2) || ints_overlap(dst, n, e, 2)) return KV_ERR_ALIAS;
    return n == 0 ? KV_OK : launched(kv_copy_pages_launch(copy_of(cache), src, dst, n, stream));
}

const char* kv_strerror(int code)
{
    switch (code) {
        case KV_OK: return "success";
        case KV_ERR_NULL: return "a pointer argument is NULL (or one of a pair is)";
        case KV_ERR_SHAPE: return "unsupported size, type or combination of them";
        case KV_ERR_SCALE: return "scale must be finite and > 0, amplitude finite";
        case KV_ERR_ALIGN: return "a pointer or a stride is not aligned (rows: 16 bytes)";
        case KV_ERR_OVERFLOW: return "problem too large for the kernels' index arithmetic";
        case KV_ERR_LAUNCH: return "HIP refused a kernel launch";
        case KV_ERR_ALIAS: return "an output overlaps an input or another output";
        case KV_ERR_STRIDE: return "a stride is smaller than what lies inside it";
        case KV_ERR_WORKSPACE: return "the workspace is too small";
        default: return "unknown error code";
    }
}

}  // extern "C"
