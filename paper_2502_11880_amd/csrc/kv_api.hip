// C entry points of the paged key-value cache and its attention: argument validation and dispatch.  As in bitnet_api.hip,
// every check runs on the host before anything is enqueued, and no call allocates, copies to the host or synchronises.
#include "bitnet_mi355x.h"
#include "rows.hpp"

namespace {

using bitnet::fail;
using bitnet::hip_status;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxTokens = (int64_t)1 << 24;   // of a call, and of a row of the table
constexpr int64_t kMaxSeqs = (int64_t)1 << 20;
constexpr int64_t kMaxPages = ((int64_t)1 << 30) - 1;
constexpr int64_t kMaxHeads = 1024;

int shift_of(int64_t page_size) {
    for (int s = 4; s <= 8; ++s)
        if (page_size == (int64_t)1 << s) return s;
    return -1;
}
bool cache_dtype_ok(int dtype) { return dtype == BITNET_DTYPE_BF16 || dtype == BITNET_DTYPE_F16; }
bool heads_ok(int64_t kv_heads, int64_t dim) {
    return kv_heads >= 1 && kv_heads <= kMaxHeads && dim >= 4 && dim <= 256 && dim % 4 == 0;
}
bool rows_ok(int64_t n_seqs, int64_t max_pages, int64_t page_size) {
    return n_seqs >= 0 && n_seqs <= kMaxSeqs && max_pages >= 1 && max_pages <= kMaxTokens / page_size;
}

size_t page_bytes(int64_t page_size, int64_t kv_heads, int64_t dim, bool values) {
    return (size_t)(kv_heads * page_size * (values ? dim : (dim + 7) / 8 * 8) * 2);
}

// Sizes and types of a cache, then (where anything is to be done) its pointers.
int check_cache(const bitnet_kv_cache* c, bool pointers) {
    if (!c) return fail(BITNET_E_INVALID, "null cache");
    if (!cache_dtype_ok(c->dtype)) return fail(BITNET_E_INVALID, "cache dtype %d: bf16 (1) or f16 (2) is needed", c->dtype);
    if (shift_of(c->page_size) < 0) return fail(BITNET_E_SHAPE, "page_size %d: 16, 32, 64, 128 or 256 is needed", c->page_size);
    if (!heads_ok(c->n_kv_heads, c->head_dim))
        return fail(BITNET_E_SHAPE, "need 1 <= n_kv_heads <= 1024 and head_dim %% 4 == 0, 4 <= head_dim <= 256; got %d heads of %d",
                    c->n_kv_heads, c->head_dim);
    if (c->n_pages < 1 || c->n_pages > kMaxPages || !rows_ok(c->n_seqs, c->max_pages, c->page_size))
        return fail(BITNET_E_SHAPE, "need 1 <= n_pages < 2^30, n_seqs <= 2^20, 1 <= max_pages, max_pages * page_size <= 2^24; got "
                    "n_pages=%lld n_seqs=%lld max_pages=%lld", (long long)c->n_pages, (long long)c->n_seqs, (long long)c->max_pages);
    if (!pointers) return BITNET_OK;
    if (!c->k || !c->v || !c->table || !c->kv_len) return fail(BITNET_E_INVALID, "null pointer in the cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->table, 4) || !aligned(c->kv_len, 4))
        return fail(BITNET_E_ALIGN, "k and v need 16-byte alignment, table and kv_len 4-byte");
    return BITNET_OK;
}

bitnet::KvCache view_of(const bitnet_kv_cache* c) {
    bitnet::KvCache v{};
    v.k = static_cast<uint16_t*>(c->k);
    v.v = static_cast<uint16_t*>(c->v);
    v.table = c->table;
    v.kv_len = c->kv_len;
    v.k_page = (int64_t)page_bytes(c->page_size, c->n_kv_heads, c->head_dim, false) / 2;
    v.v_page = (int64_t)page_bytes(c->page_size, c->n_kv_heads, c->head_dim, true) / 2;
    v.n_pages = (int)c->n_pages;
    v.max_pages = (int)c->max_pages;
    v.n_seqs = (int)c->n_seqs;
    v.shift = shift_of(c->page_size);
    v.kv_heads = c->n_kv_heads;
    v.dim = c->head_dim;
    v.chunks = (c->head_dim + 7) / 8;
    return v;
}

// What both append calls need of their rows.
int check_append(const bitnet_kv_cache* cache, int src_dtype, const int32_t* q_start, int64_t n_tokens, bool work) {
    if (const int e = check_cache(cache, work)) return e;
    if (src_dtype != BITNET_DTYPE_F32 && src_dtype != cache->dtype)
        return fail(BITNET_E_INVALID, "src_dtype %d: f32 (0) or the cache's (%d) is needed", src_dtype, cache->dtype);
    if (n_tokens < 0 || n_tokens > kMaxTokens) return fail(BITNET_E_SHAPE, "need 0 <= n_tokens <= 2^24; got %lld", (long long)n_tokens);
    if (!q_start && n_tokens != cache->n_seqs)
        return fail(BITNET_E_SHAPE, "without q_start every sequence has one token: n_tokens=%lld, n_seqs=%lld",
                    (long long)n_tokens, (long long)cache->n_seqs);
    return BITNET_OK;
}

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

// What both attention calls need of their queries.
int check_attn(const bitnet_kv_cache* c, int dtype, int64_t heads, int64_t window, int64_t n_sink) {
    if (dtype != BITNET_DTYPE_F32 && dtype != c->dtype)
        return fail(BITNET_E_INVALID, "dtype %d of q and out: f32 (0) or the cache's (%d) is needed", dtype, c->dtype);
    if (heads < 1 || heads > kMaxHeads || heads % c->n_kv_heads != 0)
        return fail(BITNET_E_SHAPE, "need n_heads %% n_kv_heads == 0 and n_heads <= 1024; got %lld over %d", (long long)heads,
                    c->n_kv_heads);
    if (window < 0 || n_sink < 0) return fail(BITNET_E_INVALID, "window and n_sink must not be negative");
    return BITNET_OK;
}

int clip(int64_t n) { return (int)(n < ((int64_t)1 << 30) ? n : (int64_t)1 << 30); }

int check_tables(const bitnet_kv_tables* t, int64_t page_size, int64_t n, bool lengths = true) {
    if (!t) return fail(BITNET_E_INVALID, "null tables");
    if (shift_of(page_size) < 0) return fail(BITNET_E_SHAPE, "page_size %lld: 16, 32, 64, 128 or 256 is needed", (long long)page_size);
    if (t->n_pages < 1 || t->n_pages > kMaxPages || !rows_ok(t->n_seqs, t->max_pages, page_size))
        return fail(BITNET_E_SHAPE, "need 1 <= n_pages < 2^30, n_seqs <= 2^20, 1 <= max_pages, max_pages * page_size <= 2^24; got "
                    "n_pages=%lld n_seqs=%lld max_pages=%lld", (long long)t->n_pages, (long long)t->n_seqs, (long long)t->max_pages);
    if (n < 0 || n > t->n_seqs) return fail(BITNET_E_SHAPE, "need 0 <= n <= n_seqs; got n=%lld", (long long)n);
    if (!t->refs || !aligned(t->refs, 4)) return fail(t->refs ? BITNET_E_ALIGN : BITNET_E_INVALID, "refs missing or not aligned");
    if (t->n_seqs > 0 && (!t->table || (lengths && !t->kv_len))) return fail(BITNET_E_INVALID, "null pointer in the tables");
    if (!aligned(t->table, 4) || !aligned(t->kv_len, 4)) return fail(BITNET_E_ALIGN, "table and kv_len need 4-byte alignment");
    return BITNET_OK;
}

bitnet::KvTables tables_of(const bitnet_kv_tables* t) {
    return {t->table, t->kv_len, t->refs, (int)t->n_seqs, (int)t->max_pages, (int)t->n_pages};
}

int check_list(const int32_t* p, const char* name) {
    if (!p) return fail(BITNET_E_INVALID, "null %s", name);
    if (!aligned(p, 4)) return fail(BITNET_E_ALIGN, "%s needs 4-byte alignment", name);
    return BITNET_OK;
}

int check_pool(const bitnet_kv_pool* p) {
    if (!p || !p->k || !p->v) return fail(BITNET_E_INVALID, "null pool");
    if (!aligned(p->k, 16) || !aligned(p->v, 16)) return fail(BITNET_E_ALIGN, "the pool needs 16-byte alignment");
    const int64_t most = (int64_t)1 << 30;
    if (p->n_layers < 1 || p->n_layers > 65535 || p->n_pages < 1 || p->n_pages > kMaxPages || p->k_page_bytes < 16 ||
        p->v_page_bytes < 16 || p->k_page_bytes % 16 || p->v_page_bytes % 16 || p->k_page_bytes > most || p->v_page_bytes > most)
        return fail(BITNET_E_SHAPE, "need 1 <= n_layers <= 65535, 1 <= n_pages < 2^30, page bytes in multiples of 16 up to 2^30; got "
                    "n_layers=%lld n_pages=%lld bytes=%lld, %lld", (long long)p->n_layers, (long long)p->n_pages,
                    (long long)p->k_page_bytes, (long long)p->v_page_bytes);
    return BITNET_OK;
}

bitnet::KvPool pool_of(const bitnet_kv_pool* p) {
    return {static_cast<uint8_t*>(p->k), static_cast<uint8_t*>(p->v), (int)p->n_layers, (int)p->n_pages, p->k_page_bytes,
            p->v_page_bytes};
}

int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return BITNET_OK;
    if (!ws || have < need) return fail(BITNET_E_WORKSPACE, "workspace holds %zu bytes, %zu needed", ws ? have : (size_t)0, need);
    if (!aligned(ws, 16)) return fail(BITNET_E_ALIGN, "ws needs 16-byte alignment");
    return BITNET_OK;
}

bitnet_status st(int code) { return (bitnet_status)code; }

}  // namespace

extern "C" {

size_t bitnet_kv_page_bytes(int dtype, int64_t page_size, int64_t n_kv_heads, int64_t head_dim, int values) {
    if (!cache_dtype_ok(dtype) || shift_of(page_size) < 0 || !heads_ok(n_kv_heads, head_dim)) return 0;
    return page_bytes(page_size, n_kv_heads, head_dim, values != 0);
}

bitnet_status bitnet_kv_append(const bitnet_kv_cache* cache, const void* k, const void* v, int src_dtype,
                               const int32_t* q_start, int64_t n_tokens, void* stream) {
    const bool work = n_tokens > 0 && cache && cache->n_seqs > 0;
    if (const int e = check_append(cache, src_dtype, q_start, n_tokens, work)) return st(e);
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!k || !v) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(q_start, 4))
        return st(fail(BITNET_E_ALIGN, "k and v need 16-byte alignment, q_start 4-byte"));
    return st(hip_status(bitnet::launch_kv_append(view_of(cache), cache->dtype, k, v, src_dtype == BITNET_DTYPE_F32, q_start,
                                                  (int)n_tokens, (hipStream_t)stream),
                         "bitnet_kv_append launch"));
}

bitnet_status bitnet_kv_append_rope(const bitnet_kv_cache* cache, const bitnet_rotation* rotation, const void* q, int64_t n_heads,
                                    const void* k, const void* v, int src_dtype, const int32_t* q_start, int64_t n_tokens,
                                    void* q_out, void* stream) {
    const bool work = n_tokens > 0 && cache && cache->n_seqs > 0;
    if (const int e = check_append(cache, src_dtype, q_start, n_tokens, work)) return st(e);
    if (const int e = bitnet::check_rotation(rotation, cache->head_dim, work)) return st(e);
    if ((q != nullptr) != (q_out != nullptr)) return st(fail(BITNET_E_INVALID, "q and q_out go together"));
    if (q && (n_heads < 1 || n_heads > kMaxHeads || n_heads % cache->n_kv_heads != 0))
        return st(fail(BITNET_E_SHAPE, "need n_heads %% n_kv_heads == 0 and n_heads <= 1024; got %lld over %d", (long long)n_heads,
                       cache->n_kv_heads));
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!k || !v) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_start, 4))
        return st(fail(BITNET_E_ALIGN, "q, q_out, k and v need 16-byte alignment, q_start 4-byte"));
    if (q) {
        const int64_t row = (int64_t)cache->head_dim * (src_dtype == BITNET_DTYPE_F32 ? 4 : 2) * n_tokens;
        const int64_t q_bytes = row * n_heads, kv_bytes = row * cache->n_kv_heads;
        if ((q != q_out && overlap(q, q_bytes, q_out, q_bytes)) || overlap(q_out, q_bytes, k, kv_bytes) || overlap(q_out, q_bytes, v, kv_bytes))
            return st(fail(BITNET_E_INVALID, "q_out must be q or overlap no input"));
    }
    return st(hip_status(bitnet::launch_kv_append_rope(view_of(cache), cache->dtype, q, q ? (int)n_heads : cache->n_kv_heads, k, v,
                                                       src_dtype == BITNET_DTYPE_F32, q_start, (int)n_tokens,
                                                       bitnet::rope_of(rotation), q_out, (hipStream_t)stream),
                         "bitnet_kv_append_rope launch"));
}

size_t bitnet_attn_decode_workspace_bytes(int64_t n_seqs, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                          int64_t page_size, int64_t max_pages, int64_t window, int64_t n_sink) {
    if (shift_of(page_size) < 0 || !heads_ok(n_kv_heads, head_dim) || !rows_ok(n_seqs, max_pages, page_size) || n_heads < 1 ||
        n_heads > kMaxHeads || n_heads % n_kv_heads || window < 0 || n_sink < 0)
        return 0;
    return bitnet::attn_decode_workspace_bytes((int)n_heads, (int)n_kv_heads, (int)head_dim, (int)page_size, max_pages,
                                               clip(window), clip(n_sink));
}

bitnet_status bitnet_attn_decode(const bitnet_kv_cache* cache, const void* q, int dtype, int64_t n_heads, float scale,
                                 int64_t window, int64_t n_sink, void* out, void* ws, size_t ws_bytes, void* stream) {
    const bool work = cache && cache->n_seqs > 0;
    if (const int e = check_cache(cache, work)) return st(e);
    if (const int e = check_attn(cache, dtype, n_heads, window, n_sink)) return st(e);
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!q || !out) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(q, 16) || !aligned(out, 16)) return st(fail(BITNET_E_ALIGN, "q and out need 16-byte alignment"));
    // a call whose rows stay whole needs none
    const bool splits = bitnet::attn_decode_splits(cache->n_seqs, (int)n_heads, cache->n_kv_heads, cache->page_size,
                                                   cache->max_pages, clip(window), clip(n_sink));
    const size_t need = splits ? bitnet_attn_decode_workspace_bytes(cache->n_seqs, n_heads, cache->n_kv_heads, cache->head_dim,
                                                                    cache->page_size, cache->max_pages, window, n_sink)
                               : 0;
    if (const int e = check_workspace(ws, ws_bytes, need)) return st(e);
    const bitnet::AttnArgs a{q, out, nullptr, (int)cache->n_seqs, (int)n_heads, scale, clip(window), clip(n_sink),
                             dtype == BITNET_DTYPE_F32};
    return st(hip_status(bitnet::launch_attn_decode(view_of(cache), cache->dtype, a, ws, (hipStream_t)stream),
                         "bitnet_attn_decode launch"));
}

size_t bitnet_attn_decode_shared_workspace_bytes(int64_t n_seqs, int64_t n_heads, int64_t n_kv_heads, int64_t head_dim,
                                                 int64_t page_size, int64_t max_pages, int64_t window, int64_t n_sink) {
    if (shift_of(page_size) < 0 || !heads_ok(n_kv_heads, head_dim) || !rows_ok(n_seqs, max_pages, page_size) || n_heads < 1 ||
        n_heads > kMaxHeads || n_heads % n_kv_heads || window < 0 || n_sink < 0)
        return 0;
    return bitnet::attn_shared_workspace_bytes(n_seqs, (int)n_heads, (int)n_kv_heads, (int)head_dim, max_pages * page_size);
}

bitnet_status bitnet_attn_decode_shared(const bitnet_kv_cache* cache, const void* q, int dtype, int64_t n_heads,
                                        const int32_t* group_start, const int32_t* prefix_len, int64_t n_groups, float scale,
                                        int64_t window, int64_t n_sink, void* out, void* ws, size_t ws_bytes, void* stream) {
    const bool work = cache && cache->n_seqs > 0 && n_groups > 0;
    if (const int e = check_cache(cache, work)) return st(e);
    if (const int e = check_attn(cache, dtype, n_heads, window, n_sink)) return st(e);
    if (n_groups < 0 || n_groups > cache->n_seqs)
        return st(fail(BITNET_E_SHAPE, "need 0 <= n_groups <= n_seqs; got %lld groups of %lld", (long long)n_groups, (long long)cache->n_seqs));
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!q || !out || !group_start || !prefix_len) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(group_start, 4) || !aligned(prefix_len, 4))
        return st(fail(BITNET_E_ALIGN, "q and out need 16-byte alignment, group_start and prefix_len 4-byte"));
    const size_t need = bitnet_attn_decode_shared_workspace_bytes(cache->n_seqs, n_heads, cache->n_kv_heads, cache->head_dim,
                                                                  cache->page_size, cache->max_pages, window, n_sink);
    if (const int e = check_workspace(ws, ws_bytes, need)) return st(e);
    const bitnet::AttnArgs a{q, out, group_start, (int)cache->n_seqs, (int)n_heads, scale, clip(window), clip(n_sink),
                             dtype == BITNET_DTYPE_F32};
    return st(hip_status(bitnet::launch_attn_shared(view_of(cache), cache->dtype, a, prefix_len, (int)n_groups, ws, (hipStream_t)stream),
                         "bitnet_attn_decode_shared launch"));
}

size_t bitnet_attn_prefill_workspace_bytes(int cache_dtype, int dtype, int64_t n_seqs, int64_t n_tokens, int64_t n_heads,
                                           int64_t n_kv_heads, int64_t head_dim, int64_t page_size, int64_t max_pages,
                                           int64_t window, int64_t n_sink) {
    if (!cache_dtype_ok(cache_dtype) || (dtype != BITNET_DTYPE_F32 && dtype != cache_dtype) || shift_of(page_size) < 0 ||
        !heads_ok(n_kv_heads, head_dim) || !rows_ok(n_seqs, max_pages, page_size) || n_seqs < 1 || n_heads < 1 ||
        n_heads > kMaxHeads || n_heads % n_kv_heads || n_tokens < 1 || n_tokens > kMaxTokens ||
        n_tokens * n_heads > (int64_t)1 << 30 || n_seqs * n_kv_heads > (int64_t)1 << 22 || window < 0 || n_sink < 0)
        return 0;
    return bitnet::attn_prefill_workspace_bytes(n_seqs, n_tokens, (int)n_heads, (int)n_kv_heads, (int)head_dim, (int)page_size,
                                                max_pages, clip(window), clip(n_sink),
                                                dtype == BITNET_DTYPE_F32 && cache_dtype == BITNET_DTYPE_BF16,
                                                dtype == BITNET_DTYPE_F32);
}

bitnet_status bitnet_attn_prefill(const bitnet_kv_cache* cache, const void* q, int dtype, int64_t n_heads,
                                  const int32_t* q_start, int64_t n_tokens, float scale, int64_t window, int64_t n_sink,
                                  void* out, void* ws, size_t ws_bytes, void* stream) {
    const bool work = n_tokens > 0 && cache && cache->n_seqs > 0;
    if (const int e = check_cache(cache, work)) return st(e);
    if (const int e = check_attn(cache, dtype, n_heads, window, n_sink)) return st(e);
    if (n_tokens < 0 || n_tokens > kMaxTokens || n_tokens * n_heads > (int64_t)1 << 30 ||
        cache->n_seqs * cache->n_kv_heads > (int64_t)1 << 22)   // a grid has fewer than 2^32 threads
        return st(fail(BITNET_E_SHAPE, "need 0 <= n_tokens <= 2^24, n_tokens * n_heads <= 2^30, n_seqs * n_kv_heads <= 2^22; got "
                       "n_tokens=%lld n_heads=%lld n_seqs=%lld", (long long)n_tokens, (long long)n_heads, (long long)cache->n_seqs));
    if (!work) return st(hip_status(hipSuccess, ""));
    if (!q || !out || !q_start) return st(fail(BITNET_E_INVALID, "null pointer argument"));
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(q_start, 4))
        return st(fail(BITNET_E_ALIGN, "q and out need 16-byte alignment, q_start 4-byte"));
    if (!aligned(ws, 16)) return st(fail(BITNET_E_ALIGN, "ws needs 16-byte alignment"));
    const bitnet::AttnArgs a{q, out, q_start, (int)n_tokens, (int)n_heads, scale, clip(window), clip(n_sink),
                             dtype == BITNET_DTYPE_F32};
    return st(hip_status(bitnet::launch_attn_prefill(view_of(cache), cache->dtype, a, ws, ws_bytes, (hipStream_t)stream),
                         "bitnet_attn_prefill launch"));
}

size_t bitnet_kv_workspace_bytes(int64_t n_pages, int64_t n_seqs) {
    if (n_pages < 1 || n_pages > kMaxPages || n_seqs < 0 || n_seqs > kMaxSeqs) return 0;
    return bitnet::kv_workspace_bytes(n_pages, n_seqs);
}

bitnet_status bitnet_kv_copy_pages(const bitnet_kv_pool* pool, const int32_t* src, const int32_t* dst, int64_t n,
                                   void* stream) {
    if (const int e = check_pool(pool)) return st(e);
    if (n < 0 || n > kMaxPages) return st(fail(BITNET_E_SHAPE, "need 0 <= n < 2^30; got %lld", (long long)n));
    if (n == 0) return st(hip_status(hipSuccess, ""));
    if (const int e = check_list(src, "src")) return st(e);
    if (const int e = check_list(dst, "dst")) return st(e);
    return st(hip_status(bitnet::launch_kv_copy(pool_of(pool), src, dst, (int)n, (hipStream_t)stream),
                         "bitnet_kv_copy_pages launch"));
}

bitnet_status bitnet_kv_reserve(const bitnet_kv_tables* tables, const int32_t* seqs, const int32_t* n_new, int64_t n,
                                int64_t page_size, int32_t* n_short, void* ws, size_t ws_bytes, void* stream) {
    if (const int e = check_tables(tables, page_size, n)) return st(e);
    if (n > 0) {
        if (const int e = check_list(seqs, "seqs")) return st(e);
        if (const int e = check_list(n_new, "n_new")) return st(e);
    }
    if (const int e = check_list(n_short, "n_short")) return st(e);
    if (const int e = check_workspace(ws, ws_bytes, bitnet_kv_workspace_bytes(tables->n_pages, tables->n_seqs))) return st(e);
    return st(hip_status(bitnet::launch_kv_reserve(tables_of(tables), seqs, n_new, (int)n, shift_of(page_size), n_short, ws,
                                                   (hipStream_t)stream),
                         "bitnet_kv_reserve launch"));
}

bitnet_status bitnet_kv_fork(const bitnet_kv_pool* pool, const bitnet_kv_tables* tables, const int32_t* parents,
                             const int32_t* children, int64_t n, int64_t page_size, int32_t* n_short, void* ws,
                             size_t ws_bytes, void* stream) {
    if (const int e = check_pool(pool)) return st(e);
    if (const int e = check_tables(tables, page_size, n)) return st(e);
    if (pool->n_pages != tables->n_pages)
        return st(fail(BITNET_E_SHAPE, "the pool has %lld pages, the tables %lld", (long long)pool->n_pages, (long long)tables->n_pages));
    if (n > 0) {
        if (const int e = check_list(parents, "parents")) return st(e);
        if (const int e = check_list(children, "children")) return st(e);
    }
    if (const int e = check_list(n_short, "n_short")) return st(e);
    if (const int e = check_workspace(ws, ws_bytes, bitnet_kv_workspace_bytes(tables->n_pages, tables->n_seqs))) return st(e);
    return st(hip_status(bitnet::launch_kv_fork(pool_of(pool), tables_of(tables), parents, children, (int)n,
                                                shift_of(page_size), n_short, ws, (hipStream_t)stream),
                         "bitnet_kv_fork launch"));
}

bitnet_status bitnet_kv_free(const bitnet_kv_tables* tables, const int32_t* seqs, int64_t n, void* stream) {
    if (const int e = check_tables(tables, 16, n)) return st(e);
    if (n == 0) return st(hip_status(hipSuccess, ""));
    if (const int e = check_list(seqs, "seqs")) return st(e);
    return st(hip_status(bitnet::launch_kv_free(tables_of(tables), seqs, (int)n, (hipStream_t)stream),
                         "bitnet_kv_free launch"));
}

bitnet_status bitnet_kv_trim(const bitnet_kv_tables* tables, const int32_t* seqs, int64_t n, int64_t page_size,
                             int64_t window, int64_t n_sink, void* stream) {
    if (const int e = check_tables(tables, page_size, n)) return st(e);
    if (window < 1 || n_sink < 0) return st(fail(BITNET_E_INVALID, "need window >= 1 and n_sink >= 0"));
    if (n == 0) return st(hip_status(hipSuccess, ""));
    if (const int e = check_list(seqs, "seqs")) return st(e);
    return st(hip_status(bitnet::launch_kv_trim(tables_of(tables), seqs, (int)n, shift_of(page_size), clip(window),
                                                clip(n_sink), (hipStream_t)stream),
                         "bitnet_kv_trim launch"));
}

bitnet_status bitnet_kv_compact(const bitnet_kv_pool* pool, const bitnet_kv_tables* tables, int32_t* n_live, void* ws,
                                size_t ws_bytes, void* stream) {
    if (const int e = check_pool(pool)) return st(e);
    if (const int e = check_tables(tables, 16, 0, false)) return st(e);   // lengths stay
    if (pool->n_pages != tables->n_pages)
        return st(fail(BITNET_E_SHAPE, "the pool has %lld pages, the tables %lld", (long long)pool->n_pages, (long long)tables->n_pages));
    if (const int e = check_list(n_live, "n_live")) return st(e);
    if (const int e = check_workspace(ws, ws_bytes, bitnet_kv_workspace_bytes(tables->n_pages, tables->n_seqs))) return st(e);
    return st(hip_status(bitnet::launch_kv_compact(pool_of(pool), tables_of(tables), n_live, ws, (hipStream_t)stream),
                         "bitnet_kv_compact launch"));
}

}  // extern "C"
