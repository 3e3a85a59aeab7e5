// The C entry points of the key-value cache: argument checks, workspace layout, launches.
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "g10_cache.cuh"

namespace g10 {
namespace {

constexpr int64_t kCacheLimit = 0x7fffffff - 64;
constexpr float kLog2E = 1.4426950408889634f;

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
// (strides of a dimension of one entry are never used, but are asked for all the same: they are the caller's arithmetic)
bool row_stride(int64_t s) { return s % 8 == 0; }

// (unit: elements of 16 bytes of a row: 8, or 16 codes)
int32_t view_of(const g10_cache *c, bool rows, CacheView &o, int unit = 8)
{
    if (!c) return G10_ERR_ARG;
    if (c->dtype != G10_BF16 && c->dtype != G10_FP16) return G10_ERR_ARG;
    if (c->num_seqs < 0 || c->kv_heads < 1 || c->head_dim < unit || c->head_dim % unit != 0 || c->page_size < 1 || c->max_pages < 0 || c->num_pages < 0)
        return G10_ERR_ARG;
    if (c->num_seqs > 65535 || c->kv_heads > 1024 || c->head_dim > 256 || c->page_size > 65536 || c->num_pages > kCacheLimit ||
        (int64_t)c->max_pages * c->page_size > kCacheLimit)
        return G10_ERR_LIMIT;
    if (c->num_seqs > 0 && (!c->lengths || (c->max_pages > 0 && !c->page_table) || c->table_stride < c->max_pages)) return G10_ERR_ARG;
    if (!c->status) return G10_ERR_ARG;
    if (rows && c->num_pages > 0) {
        if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return G10_ERR_ARG;
        if (c->page_stride % unit != 0 || c->slot_stride % unit != 0 || c->head_stride % unit != 0) return G10_ERR_ARG;
        if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0) return G10_ERR_ARG;
        // (rows are found by numbers of 32 bits, in units of 16 bytes)
        const __int128 last = (__int128)(c->num_pages - 1) * c->page_stride + (__int128)(c->page_size - 1) * c->slot_stride + (__int128)(c->kv_heads - 1) * c->head_stride;
        if (last / unit + 32 >= 0xffffffffll) return G10_ERR_LIMIT;
    }
    o.k = (const char *)c->k; o.v = (const char *)c->v;
    // (copies of no bytes, for slots whose page is none, are asked for from there all the same: an address that exists)
    if (c->num_pages == 0) o.k = o.v = (const char *)((uintptr_t)c->status & ~(uintptr_t)15);
    o.page_stride = c->page_stride / unit; o.slot_stride = c->slot_stride / unit; o.head_stride = c->head_stride / unit;
    int l = 0;
    while ((1 << l) < c->page_size) ++l;
    o.page_shift = 31 + l;
    o.page_mul = (unsigned)(((uint64_t)1 << (31 + l)) / (uint64_t)c->page_size + 1);
    o.table = c->page_table; o.table_stride = c->table_stride; o.num_pages = c->num_pages;
    o.lengths = c->lengths; o.seen = c->seen ? c->seen : c->lengths;
    o.scores = c->scores; o.positions = c->positions; o.status = (ull *)c->status;
    o.num_seqs = c->num_seqs; o.kv_heads = c->kv_heads; o.head_dim = c->head_dim; o.page_size = c->page_size; o.max_pages = c->max_pages;
    o.capacity = (int)((int64_t)c->max_pages * c->page_size);
    return G10_OK;
}

int32_t packed_view_of(const g10_packed *p, bool rows, CacheView &o)
{
    if (!p || (p->code != G10_INT8 && p->code != G10_E4M3)) return G10_ERR_ARG;
    const int32_t rc = view_of(&p->cache, rows, o, 16);
    if (rc != G10_OK) return rc;
    return rows && p->cache.num_pages > 0 && (!p->scales || ((uintptr_t)p->scales & 7u)) ? G10_ERR_ARG : G10_OK;
}

int32_t status_of(cudaError_t e) { return e == cudaSuccess ? G10_OK : G10_ERR_CUDA; }

struct AttendLayout {
    size_t ml, part, logits, sums, notes, total, bytes;
};
AttendLayout attend_layout(const AttendShape &z, bool scores)
{
    AttendLayout l;
    l.ml = 0;
    l.part = align_up(l.ml + sizeof(float2) * (size_t)z.pieces * z.block_rows);
    l.logits = align_up(l.part + sizeof(float) * (size_t)z.pieces * z.block_rows * z.padded_dim);
    l.sums = align_up(l.logits + (scores ? sizeof(float) * (size_t)z.tiles * z.logit_rows * 64 : 0));
    l.notes = align_up(l.sums + (scores ? sizeof(float) * (size_t)z.items * z.block_rows : 0));
    l.total = align_up(l.notes + (scores && z.logit_rows > 0 ? sizeof(TileNote) * (size_t)z.tiles : 0));
    l.bytes = align_up(l.total + sizeof(int64_t));
    return l;
}

int32_t check_heads(const CacheView &c, int32_t new_tokens, int32_t q_heads, int32_t window, int32_t sinks)
{
    if (new_tokens < 1 || q_heads < 1 || q_heads % c.kv_heads != 0 || window < 0 || sinks < 0) return G10_ERR_ARG;
    return (int64_t)new_tokens * (q_heads / c.kv_heads) > 1024 ? G10_ERR_LIMIT : G10_OK;
}

// What append is asked to do; `nothing`: there is no sequence.
int32_t append_args(const g10_cache_tokens *t, AppendArgs &a, bool &nothing)
{
    nothing = false;
    if (!t || t->new_tokens < 1 || t->q_heads < 0 || t->q_heads > 65536 || t->rotary_dim < 0 || t->rotary_dim % 2 != 0 || t->rotary_dim > a.c.head_dim)
        return G10_ERR_ARG;
    if (t->rotary_dim > 0 && (!t->cos_table || !t->sin_table || t->table_rows < 0)) return G10_ERR_ARG;
    if (!(t->eps >= 0.0f) && (t->q_weight || t->k_weight)) return G10_ERR_ARG;
    nothing = a.c.num_seqs == 0;
    if (nothing) return G10_OK;
    if (!t->k || !t->v || !aligned16(t->k) || !aligned16(t->v) || !row_stride(t->k_seq_stride) || !row_stride(t->k_token_stride) ||
        !row_stride(t->k_head_stride) || !row_stride(t->v_seq_stride) || !row_stride(t->v_token_stride) || !row_stride(t->v_head_stride))
        return G10_ERR_ARG;
    if (t->q_heads > 0 && (!t->q || !t->q_out || !aligned16(t->q) || !aligned16(t->q_out) || !row_stride(t->q_seq_stride) ||
                           !row_stride(t->q_token_stride) || !row_stride(t->q_head_stride)))
        return G10_ERR_ARG;
    if ((t->q_weight && !aligned16(t->q_weight)) || (t->k_weight && !aligned16(t->k_weight))) return G10_ERR_ARG;
    if ((int64_t)a.c.num_seqs * t->new_tokens > kCacheLimit) return G10_ERR_LIMIT;
    a.q = (const char *)t->q; a.k = (const char *)t->k; a.v = (const char *)t->v;
    a.q_seq = t->q_seq_stride; a.q_token = t->q_token_stride; a.q_head = t->q_head_stride;
    a.k_seq = t->k_seq_stride; a.k_token = t->k_token_stride; a.k_head = t->k_head_stride;
    a.v_seq = t->v_seq_stride; a.v_token = t->v_token_stride; a.v_head = t->v_head_stride;
    a.q_out = (char *)t->q_out; a.counts = t->counts;
    a.q_weight = (const char *)t->q_weight; a.k_weight = (const char *)t->k_weight; a.eps = t->eps; a.inv_dim = 1.0f / (float)a.c.head_dim;
    a.cos_table = t->cos_table; a.sin_table = t->sin_table; a.table_rows = t->table_rows;
    a.new_tokens = t->new_tokens; a.q_heads = t->q_heads; a.rotary = t->rotary_dim; a.interleaved = t->interleaved != 0;
    a.scales = nullptr;
    return G10_OK;
}

// What attend is asked to do, but for the workspace.
int32_t attend_args(const g10_cache *cache, const g10_cache_queries *u, AttendArgs &a, bool &nothing)
{
    nothing = false;
    if (!u) return G10_ERR_ARG;
    const int32_t rc = check_heads(a.c, u->new_tokens, u->q_heads, u->window, u->sinks);
    if (rc != G10_OK) return rc;
    if ((u->window > 0 && cache->positions) || (u->add_scores && cache->num_pages > 0 && !cache->scores) || !std::isfinite(u->scale * kLog2E)) return G10_ERR_ARG;
    nothing = a.c.num_seqs == 0;
    if (nothing) return G10_OK;
    if (!u->q || !u->out || !aligned16(u->q) || !aligned16(u->out) || !row_stride(u->q_seq_stride) || !row_stride(u->q_token_stride) ||
        !row_stride(u->q_head_stride))
        return G10_ERR_ARG;
    a.q = (const char *)u->q; a.q_seq = u->q_seq_stride; a.q_token = u->q_token_stride; a.q_head = u->q_head_stride;
    a.counts = u->counts; a.out = (char *)u->out; a.lse = u->lse;
    a.scale_log2 = u->scale * kLog2E;
    a.new_tokens = u->new_tokens; a.q_heads = u->q_heads; a.group = u->q_heads / a.c.kv_heads; a.rows = u->new_tokens * a.group;
    a.window = u->window; a.sinks = u->window > 0 ? u->sinks : 0;
    a.books = u->add_scores != 0;
    return G10_OK;
}
int32_t attend_places(const AttendShape &z, void *ws, size_t ws_bytes, AttendArgs &a)
{
    const AttendLayout l = attend_layout(z, a.books);
    if (!ws || ((uintptr_t)ws & (kAlign - 1)) || ws_bytes < l.bytes) return G10_ERR_WORKSPACE;
    a.row_blocks = z.row_blocks; a.pieces = z.pieces;
    a.ml = (float2 *)((char *)ws + l.ml); a.part = (float *)((char *)ws + l.part);
    a.logits = a.books && z.logit_rows > 0 ? (float *)((char *)ws + l.logits) : nullptr;
    a.sums = (float *)((char *)ws + l.sums); a.notes = (TileNote *)((char *)ws + l.notes); a.total = (int64_t *)((char *)ws + l.total);
#ifdef G10_TEST_HOOKS
    // test build: an arrival that never comes
    const char *const mute = getenv("G10_TEST_CACHE_MUTE");
    a.mute = mute ? atoi(mute) : 0;
#endif
    return G10_OK;
}

// Behind a shared beginning: what the beginning leaves, and room for either part in turn.
struct SharedLayout {
    size_t shared, ml, o, room, bytes;
};
SharedLayout shared_layout(const AttendShape &begin, const AttendShape &rest, int64_t rows, int head_dim)
{
    SharedLayout l;
    l.shared = 0;
    l.ml = align_up(l.shared + sizeof(int32_t));
    l.o = align_up(l.ml + sizeof(float2) * (size_t)rows);
    l.room = align_up(l.o + sizeof(float) * (size_t)rows * head_dim);
    const size_t x = attend_layout(begin, false).bytes, y = attend_layout(rest, false).bytes;
    l.bytes = l.room + (x > y ? x : y);
    return l;
}
// The beginning as one sequence with all sequences' new tokens.
CacheView begin_view(const CacheView &c)
{
    CacheView v = c;
    v.num_seqs = 1;
    return v;
}
int32_t check_shared(const CacheView &c, int32_t new_tokens, int32_t q_heads)
{
    const int32_t rc = check_heads(c, new_tokens, q_heads, 0, 0);
    if (rc != G10_OK) return rc;
    return (int64_t)c.num_seqs * new_tokens * (q_heads / c.kv_heads) > kCacheLimit ? G10_ERR_LIMIT : G10_OK;
}

int32_t evict_args(const g10_cache_plan *p, EvictArgs &a, bool &nothing)
{
    nothing = false;
    if (!p || p->budget < 1) return G10_ERR_ARG;
    if (p->budget > kCacheLimit) return G10_ERR_LIMIT;
    nothing = a.c.num_seqs == 0;
    if (nothing) return G10_OK;
    if (!p->moves || !p->counts || ((uintptr_t)p->moves & 7u)) return G10_ERR_ARG;
    a.budget = p->budget; a.sinks = 0; a.recent = 0; a.moves = p->moves; a.counts = p->counts; a.new_lengths = nullptr;
    return G10_OK;
}

}  // namespace
}  // namespace g10

using namespace g10;

extern "C" {

int32_t g10_cache_append(const g10_cache *cache, const g10_cache_tokens *t, void *stream)
{
    AppendArgs a;
    bool nothing;
    int32_t rc = view_of(cache, true, a.c);
    if (rc == G10_OK) rc = append_args(t, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    return status_of(launch_cache_append(a, cache->dtype, (cudaStream_t)stream));
}

int32_t g10_cache_workspace_bytes(const g10_cache *cache, int32_t new_tokens, int32_t q_heads, int32_t window, int32_t sinks, int32_t add_scores,
                                  size_t *out_bytes)
{
    CacheView c;
    int32_t rc = view_of(cache, false, c);
    if (rc == G10_OK && !out_bytes) rc = G10_ERR_ARG;
    if (rc == G10_OK) rc = check_heads(c, new_tokens, q_heads, window, sinks);
    if (rc != G10_OK) return rc;
    *out_bytes = attend_layout(attend_shape(c, new_tokens * (q_heads / c.kv_heads), new_tokens, window, sinks), add_scores != 0).bytes;
    return G10_OK;
}

int32_t g10_cache_attend(const g10_cache *cache, const g10_cache_queries *u, void *ws, size_t ws_bytes, void *stream)
{
    AttendArgs a;
    bool nothing;
    int32_t rc = view_of(cache, true, a.c);
    if (rc == G10_OK) rc = attend_args(cache, u, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    rc = attend_places(attend_shape(a.c, a.rows, a.new_tokens, a.window, a.sinks), ws, ws_bytes, a);
    return rc != G10_OK ? rc : status_of(launch_cache_attend(a, cache->dtype, (cudaStream_t)stream));
}

int32_t g10_cache_shared_workspace_bytes(const g10_cache *cache, int32_t new_tokens, int32_t q_heads, size_t *out_bytes)
{
    CacheView c;
    int32_t rc = view_of(cache, false, c);
    if (rc == G10_OK && !out_bytes) rc = G10_ERR_ARG;
    if (rc == G10_OK) rc = check_shared(c, new_tokens, q_heads);
    if (rc != G10_OK) return rc;
    const int tokens = c.num_seqs * new_tokens, group = q_heads / c.kv_heads;
    *out_bytes = shared_layout(begin_shape(begin_view(c), tokens * group, tokens), attend_shape(c, new_tokens * group, new_tokens, 0, 0),
                               (int64_t)tokens * q_heads, c.head_dim).bytes;
    return G10_OK;
}

int32_t g10_cache_attend_shared(const g10_cache *cache, const g10_cache_queries *u, const int32_t *shared, void *ws, size_t ws_bytes, void *stream)
{
    RestArgs a;
    bool nothing;
    int32_t rc = view_of(cache, true, a.c);
    if (rc == G10_OK) rc = attend_args(cache, u, a, nothing);
    if (rc != G10_OK) return rc;
    if (!shared || u->window > 0 || u->add_scores) return G10_ERR_ARG;
    if (nothing) return G10_OK;
    if ((rc = check_shared(a.c, u->new_tokens, u->q_heads)) != G10_OK) return rc;
    a.each = a.new_tokens;
    BeginArgs b;
    static_cast<SharedArgs &>(b) = a;
    b.c = begin_view(a.c);
    b.new_tokens = a.c.num_seqs * a.new_tokens; b.rows = b.new_tokens * b.group; b.counts = nullptr;
    const AttendShape y = begin_shape(b.c, b.rows, b.new_tokens), z = attend_shape(a.c, a.rows, a.new_tokens, 0, 0);
    const SharedLayout l = shared_layout(y, z, (int64_t)b.new_tokens * a.q_heads, a.c.head_dim);
    if (!ws || ((uintptr_t)ws & (kAlign - 1)) || ws_bytes < l.bytes) return G10_ERR_WORKSPACE;
    a.shared = b.shared = (int32_t *)((char *)ws + l.shared);
    a.begin_ml = b.begin_ml = (float2 *)((char *)ws + l.ml); a.begin_o = b.begin_o = (float *)((char *)ws + l.o);
    if ((rc = attend_places(y, (char *)ws + l.room, l.bytes - l.room, b)) != G10_OK || (rc = attend_places(z, (char *)ws + l.room, l.bytes - l.room, a)) != G10_OK) return rc;
    return status_of(launch_cache_shared(b, a, shared, cache->dtype, (cudaStream_t)stream));
}

int32_t g10_cache_plan_evictions(const g10_cache *cache, const g10_cache_plan *p, void *stream)
{
    EvictArgs a;
    int32_t rc = view_of(cache, false, a.c);
    if (rc != G10_OK) return rc;
    if (!p || p->budget < 1 || p->sinks < 0 || p->recent < 0 || (int64_t)p->sinks + p->recent > p->budget) return G10_ERR_ARG;
    if (p->budget > kCacheLimit) return G10_ERR_LIMIT;
    if (a.c.num_seqs == 0) return G10_OK;
    if (!p->moves || !p->counts || ((uintptr_t)p->moves & 7u) || (a.c.num_pages > 0 && !a.c.scores)) return G10_ERR_ARG;
    a.budget = p->budget; a.sinks = p->sinks; a.recent = p->recent; a.moves = p->moves; a.counts = p->counts; a.new_lengths = p->new_lengths;
    return status_of(launch_cache_plan(a, (cudaStream_t)stream));
}

int32_t g10_cache_evict(const g10_cache *cache, const g10_cache_plan *p, void *stream)
{
    EvictArgs a;
    bool nothing;
    int32_t rc = view_of(cache, true, a.c);
    if (rc == G10_OK) rc = evict_args(p, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    a.row_units = a.c.head_dim / 8; a.scales = nullptr;
    return status_of(launch_cache_evict(a, (cudaStream_t)stream));
}

// ---- rows of 8-bit codes ----
int32_t g10_packed_append(const g10_packed *packed, const g10_cache_tokens *t, void *stream)
{
    AppendArgs a;
    bool nothing;
    int32_t rc = packed_view_of(packed, true, a.c);
    if (rc == G10_OK) rc = append_args(t, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    a.scales = packed->scales;
    return status_of(launch_packed_append(a, packed->cache.dtype, packed->code, (cudaStream_t)stream));
}

int32_t g10_packed_read(const g10_packed *packed, const g10_packed_rows *r, void *stream)
{
    ReadArgs a;
    int32_t rc = packed_view_of(packed, true, a.c);
    if (rc != G10_OK) return rc;
    if (!r || r->tokens < 0) return G10_ERR_ARG;
    for (const void *p : {(const void *)r->k, (const void *)r->v}) if (!aligned16(p)) return G10_ERR_ARG;
    if ((r->k && (!row_stride(r->k_seq_stride) || !row_stride(r->k_token_stride) || !row_stride(r->k_head_stride))) ||
        (r->v && (!row_stride(r->v_seq_stride) || !row_stride(r->v_token_stride) || !row_stride(r->v_head_stride))))
        return G10_ERR_ARG;
    if (r->tokens > kCacheLimit || (int64_t)a.c.num_seqs * r->tokens > kCacheLimit) return G10_ERR_LIMIT;
    if (a.c.num_seqs == 0 || r->tokens == 0 || (!r->k && !r->v)) return G10_OK;
    a.scales = (const float2 *)packed->scales; a.k = (char *)r->k; a.v = (char *)r->v;
    a.k_seq = r->k_seq_stride; a.k_token = r->k_token_stride; a.k_head = r->k_head_stride;
    a.v_seq = r->v_seq_stride; a.v_token = r->v_token_stride; a.v_head = r->v_head_stride;
    a.starts = r->starts; a.tokens = r->tokens;
    return status_of(launch_packed_read(a, packed->cache.dtype, packed->code, (cudaStream_t)stream));
}

int32_t g10_packed_workspace_bytes(const g10_packed *packed, int32_t new_tokens, int32_t q_heads, int32_t window, int32_t sinks, int32_t add_scores,
                                   size_t *out_bytes)
{
    CacheView c;
    int32_t rc = packed_view_of(packed, false, c);
    if (rc == G10_OK && !out_bytes) rc = G10_ERR_ARG;
    if (rc == G10_OK) rc = check_heads(c, new_tokens, q_heads, window, sinks);
    if (rc != G10_OK) return rc;
    *out_bytes = attend_layout(packed_shape(c, new_tokens * (q_heads / c.kv_heads), new_tokens, window, sinks), add_scores != 0).bytes;
    return G10_OK;
}

int32_t g10_packed_attend(const g10_packed *packed, const g10_cache_queries *u, void *ws, size_t ws_bytes, void *stream)
{
    AttendArgs a;
    bool nothing;
    int32_t rc = packed_view_of(packed, true, a.c);
    if (rc == G10_OK) rc = attend_args(&packed->cache, u, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    rc = attend_places(packed_shape(a.c, a.rows, a.new_tokens, a.window, a.sinks), ws, ws_bytes, a);
    return rc != G10_OK ? rc : status_of(launch_packed_attend(a, (const float2 *)packed->scales, packed->cache.dtype, packed->code, (cudaStream_t)stream));
}

int32_t g10_packed_evict(const g10_packed *packed, const g10_cache_plan *p, void *stream)
{
    EvictArgs a;
    bool nothing;
    int32_t rc = packed_view_of(packed, true, a.c);
    if (rc == G10_OK) rc = evict_args(p, a, nothing);
    if (rc != G10_OK || nothing) return rc;
    a.row_units = a.c.head_dim / 16; a.scales = (float2 *)packed->scales;
    return status_of(launch_cache_evict(a, (cudaStream_t)stream));
}

}  // extern "C"
