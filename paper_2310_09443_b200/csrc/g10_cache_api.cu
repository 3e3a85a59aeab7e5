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

int32_t view_of(const g10_cache *c, bool rows, CacheView &o)
{
    if (!c) return G10_ERR_ARG;
    if (c->dtype != G10_BF16 && c->dtype != G10_FP16) return G10_ERR_ARG;
    if (c->num_seqs < 0 || c->kv_heads < 1 || c->head_dim < 8 || c->head_dim % 8 != 0 || c->page_size < 1 || c->max_pages < 0 || c->num_pages < 0)
        return G10_ERR_ARG;
    if (c->num_seqs > 65535 || c->kv_heads > 1024 || c->head_dim > 256 || c->page_size > 65536 || c->num_pages > kCacheLimit ||
        (int64_t)c->max_pages * c->page_size > kCacheLimit)
        return G10_ERR_LIMIT;
    if (c->num_seqs > 0 && (!c->lengths || (c->max_pages > 0 && !c->page_table) || c->table_stride < c->max_pages)) return G10_ERR_ARG;
    if (!c->status) return G10_ERR_ARG;
    if (rows && c->num_pages > 0) {
        if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return G10_ERR_ARG;
        if (!row_stride(c->page_stride) || !row_stride(c->slot_stride) || !row_stride(c->head_stride)) return G10_ERR_ARG;
        if (c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0) return G10_ERR_ARG;
        // (rows are found by numbers of 32 bits, in units of 16 bytes)
        const __int128 last = (__int128)(c->num_pages - 1) * c->page_stride + (__int128)(c->page_size - 1) * c->slot_stride + (__int128)(c->kv_heads - 1) * c->head_stride;
        if (last / 8 + 32 >= 0xffffffffll) return G10_ERR_LIMIT;
    }
    o.k = (const char *)c->k; o.v = (const char *)c->v;
    // (copies of no bytes, for slots whose page is none, are asked for from there all the same: an address that exists)
    if (c->num_pages == 0) o.k = o.v = (const char *)((uintptr_t)c->status & ~(uintptr_t)15);
    o.page_stride = c->page_stride / 8; o.slot_stride = c->slot_stride / 8; o.head_stride = c->head_stride / 8;
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

}  // namespace
}  // namespace g10

using namespace g10;

extern "C" {

int32_t g10_cache_append(const g10_cache *cache, const g10_cache_tokens *t, void *stream)
{
    AppendArgs a;
    int32_t rc = view_of(cache, true, a.c);
    if (rc != G10_OK) return rc;
    if (!t || t->new_tokens < 1 || t->q_heads < 0 || t->q_heads > 65536 || t->rotary_dim < 0 || t->rotary_dim % 2 != 0 || t->rotary_dim > a.c.head_dim)
        return G10_ERR_ARG;
    if (t->rotary_dim > 0 && (!t->cos_table || !t->sin_table || t->table_rows < 0)) return G10_ERR_ARG;
    if (!(t->eps >= 0.0f) && (t->q_weight || t->k_weight)) return G10_ERR_ARG;
    if (a.c.num_seqs == 0) return G10_OK;
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
    int32_t rc = view_of(cache, true, a.c);
    if (rc != G10_OK) return rc;
    if (!u) return G10_ERR_ARG;
    rc = check_heads(a.c, u->new_tokens, u->q_heads, u->window, u->sinks);
    if (rc != G10_OK) return rc;
    if ((u->window > 0 && cache->positions) || (u->add_scores && cache->num_pages > 0 && !cache->scores) || !std::isfinite(u->scale * kLog2E)) return G10_ERR_ARG;
    if (a.c.num_seqs == 0) return G10_OK;
    if (!u->q || !u->out || !aligned16(u->q) || !aligned16(u->out) || !row_stride(u->q_seq_stride) || !row_stride(u->q_token_stride) ||
        !row_stride(u->q_head_stride))
        return G10_ERR_ARG;
    a.q = (const char *)u->q; a.q_seq = u->q_seq_stride; a.q_token = u->q_token_stride; a.q_head = u->q_head_stride;
    a.counts = u->counts; a.out = (char *)u->out; a.lse = u->lse;
    a.scale_log2 = u->scale * kLog2E;
    a.new_tokens = u->new_tokens; a.q_heads = u->q_heads; a.group = u->q_heads / a.c.kv_heads; a.rows = u->new_tokens * a.group;
    a.window = u->window; a.sinks = u->window > 0 ? u->sinks : 0;
    const AttendShape z = attend_shape(a.c, a.rows, a.new_tokens, a.window, a.sinks);
    const AttendLayout l = attend_layout(z, u->add_scores != 0);
    if (!ws || ((uintptr_t)ws & (kAlign - 1)) || ws_bytes < l.bytes) return G10_ERR_WORKSPACE;
    a.row_blocks = z.row_blocks; a.pieces = z.pieces;
    a.ml = (float2 *)((char *)ws + l.ml); a.part = (float *)((char *)ws + l.part);
    a.books = u->add_scores != 0;
    a.logits = a.books && z.logit_rows > 0 ? (float *)((char *)ws + l.logits) : nullptr;
    a.sums = (float *)((char *)ws + l.sums); a.notes = (TileNote *)((char *)ws + l.notes); a.total = (int64_t *)((char *)ws + l.total);
#ifdef G10_TEST_HOOKS
    // test build: an arrival that never comes
    const char *const mute = getenv("G10_TEST_CACHE_MUTE");
    a.mute = mute ? atoi(mute) : 0;
#endif
    return status_of(launch_cache_attend(a, cache->dtype, (cudaStream_t)stream));
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
    int32_t rc = view_of(cache, true, a.c);
    if (rc != G10_OK) return rc;
    if (!p || p->budget < 1) return G10_ERR_ARG;
    if (p->budget > kCacheLimit) return G10_ERR_LIMIT;
    if (a.c.num_seqs == 0) return G10_OK;
    if (!p->moves || !p->counts || ((uintptr_t)p->moves & 7u)) return G10_ERR_ARG;
    a.budget = p->budget; a.sinks = 0; a.recent = 0; a.moves = p->moves; a.counts = p->counts; a.new_lengths = nullptr;
    return status_of(launch_cache_evict(a, (cudaStream_t)stream));
}

}  // extern "C"
