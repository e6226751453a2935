// extern "C" boundary of dense attention and the paged cache: argument validation and dispatch. See stream.h.
#include <cmath>

#include "serve_common.cuh"

using namespace stream;

namespace {

bool known_d(int d) { return d == 16 || d == 32 || d == 64 || d == 128 || d == 256; }
int elem_bytes(int dtype) { return dtype == STREAM_F32 ? 4 : 2; }

// Tokens of a sequence, of a slot and of all prompts: a tile's last row, counted from its first, stays within 32 bits.
constexpr long long kMaxTokens = 0x7fffffffLL - 4095;

stream_status invalid(const char *text) {
    set_error("%s", text);
    return STREAM_ERR_INVALID_ARG;
}
bool natural(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The scale in units of log2. A NaN selects no default, and a finite scale may pass fp32 here: both would make every output NaN.
stream_status make_scale(float scale, int d, float *scale_log2) {
    if (scale <= 0.f) scale = 1.0f / sqrtf((float)d);
    *scale_log2 = scale * 1.4426950408889634f;
    return std::isfinite(*scale_log2) ? STREAM_OK : invalid("scale must be finite, times log2(e) too");
}

// Strides of a [rows, heads, d] tensor: at least a head's row apart, where there is more than one.
bool strides_ok(long long rows, long long s_t, int heads, long long s_h, int d) {
    return (rows <= 1 || s_t >= d) && (heads <= 1 || s_h >= d);
}

stream_status make_prompt(const stream_prompt *p, PromptGeom *g) {
    if (p == nullptr) return invalid("problem is NULL");
    if (p->n_seqs < 1) return invalid("n_seqs must be positive");
    if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) return invalid("n_kv_heads must divide n_q_heads");
    if (p->dtype != STREAM_F32 && p->dtype != STREAM_BF16) { set_error("unknown dtype %d", p->dtype); return STREAM_ERR_INVALID_ARG; }
    if (p->causal != 0 && p->causal != 1) return invalid("causal must be 0 or 1");
    if (p->total_q < 0 || p->total_k < 0) return invalid("total_q and total_k must not be negative");
    if (p->d < 1) return invalid("d must be positive");
    if (!strides_ok(p->total_q, p->q_stride_t, p->n_q_heads, p->q_stride_h, p->d) ||
        !strides_ok(p->total_k, p->kv_stride_t, p->n_kv_heads, p->kv_stride_h, p->d))
        return invalid("token and head strides must be >= d");
    if (!known_d(p->d)) { set_error("d must be 16, 32, 64, 128 or 256 (got %d)", p->d); return STREAM_ERR_UNSUPPORTED; }
    if (p->total_q > kMaxTokens || p->total_k > kMaxTokens || p->n_seqs > (1 << 24) || p->n_q_heads > (1 << 16)) {
        set_error("up to 2^31 - 4096 tokens, 2^24 sequences and 2^16 heads");
        return STREAM_ERR_UNSUPPORTED;
    }
    *g = PromptGeom{};
    g->n_seqs = p->n_seqs; g->H = p->n_q_heads; g->G = p->n_kv_heads; g->hpg = p->n_q_heads / p->n_kv_heads;
    g->d = p->d; g->causal = p->causal; g->total_q = (int)p->total_q; g->total_k = (int)p->total_k;
    // a stride that does not matter gets a value that suits everybody
    g->ks_h = g->G > 1 ? p->kv_stride_h : p->d;
    g->qs_h = g->H > 1 ? p->q_stride_h : p->d;
    g->ks_t = g->total_k > 1 ? p->kv_stride_t : (long long)g->G * p->d;
    g->qs_t = g->total_q > 1 ? p->q_stride_t : (long long)g->H * p->d;
    return STREAM_OK;
}

stream_status make_cache(const stream_cache *c, CacheGeom *g) {
    if (c == nullptr) return invalid("cache is NULL");
    if (c->n_slots < 1 || c->n_pages < 1 || c->page_size < 1 || c->max_pages < 1 || c->n_kv_heads < 1 || c->n_layers < 1 || c->d < 1)
        return invalid("n_slots, n_pages, page_size, max_pages, n_kv_heads, n_layers and d must be positive");
    if (c->dtype != STREAM_F32 && c->dtype != STREAM_BF16) { set_error("unknown dtype %d", c->dtype); return STREAM_ERR_INVALID_ARG; }
    const int d = c->d;
    if ((c->n_layers > 1 && c->stride_l < d) || (c->n_pages > 1 && c->stride_p < d) || (c->page_size > 1 && c->stride_t < d) ||
        (c->n_kv_heads > 1 && c->stride_h < d))
        return invalid("layer, page, token and head strides must be >= d");
    if (!known_d(d)) { set_error("d must be 16, 32, 64, 128 or 256 (got %d)", d); return STREAM_ERR_UNSUPPORTED; }
    if ((long long)c->n_slots * c->max_pages > 0x7fffffffLL || (long long)c->max_pages * c->page_size > kMaxTokens ||
        c->n_pages > (1 << 30) || c->n_slots > (1 << 30) || c->n_kv_heads > (1 << 16) || (long long)c->page_size * c->n_kv_heads * d > 0x3fffffffLL) {
        set_error("too many slots, pages or tokens for 32-bit indexing");
        return STREAM_ERR_UNSUPPORTED;
    }
    *g = CacheGeom{};
    g->n_slots = c->n_slots; g->n_pages = c->n_pages; g->page = c->page_size; g->max_pages = c->max_pages;
    g->G = c->n_kv_heads; g->d = d; g->n_layers = c->n_layers;
    g->s_l = c->n_layers > 1 ? c->stride_l : 0;
    g->s_p = c->n_pages > 1 ? c->stride_p : 0;
    g->s_t = c->page_size > 1 ? c->stride_t : (long long)g->G * d;
    g->s_h = c->n_kv_heads > 1 ? c->stride_h : d;
    return STREAM_OK;
}

stream_status make_ledger(const stream_cache *c, int32_t *page_table, int32_t *seq_len, int32_t *ref_count, const int32_t *info,
                          const void *workspace, size_t bytes, CacheGeom *g) {
    stream_status rc = make_cache(c, g);
    if (rc != STREAM_OK) return rc;
    if (page_table == nullptr || seq_len == nullptr || ref_count == nullptr || info == nullptr)
        return invalid("page_table, seq_len, ref_count and info_out must not be NULL");
    if (!natural(page_table, 4) || !natural(seq_len, 4) || !natural(ref_count, 4) || !natural(info, 16))
        return invalid("the ledger must be 4-byte aligned and info_out 16-byte aligned");
    const size_t need = ledger_workspace_bytes(*g);
    if (workspace == nullptr || bytes < need || ((uintptr_t)workspace & 255) != 0) {
        set_error("workspace must be a 256-byte aligned device buffer of at least %zu bytes", need);
        return STREAM_ERR_WORKSPACE;
    }
    g->table = page_table; g->len = seq_len; g->count = ref_count;
    return STREAM_OK;
}

}  // namespace

extern "C" {

stream_status stream_prompt_attention(const stream_prompt *p, const void *q, const void *k, const void *v, const int32_t *cu_q,
                                      const int32_t *cu_k, float scale, void *out, float *lse_out, void *cuda_stream) {
    PromptGeom g;
    stream_status rc = make_prompt(p, &g);
    if (rc != STREAM_OK) return rc;
    if (cu_q == nullptr || cu_k == nullptr) return invalid("cu_q and cu_k must not be NULL");
    if (g.total_q == 0) return STREAM_OK;  // (nothing to write; the tensors may have no memory)
    if (q == nullptr || out == nullptr || (g.total_k > 0 && (k == nullptr || v == nullptr))) return invalid("q, k, v and out must not be NULL");
    const int e = elem_bytes(p->dtype);
    if (!natural(q, e) || !natural(k, e) || !natural(v, e) || !natural(out, e) || !natural(lse_out, 4) || !natural(cu_q, 4) || !natural(cu_k, 4))
        return invalid("a pointer is not aligned to its elements");
    rc = make_scale(scale, g.d, &g.scale_log2);
    if (rc != STREAM_OK) return rc;
    g.cu_q = cu_q; g.cu_k = cu_k; g.out = out; g.lse = lse_out;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (prompt_tc_supported(g, p->dtype, q, k, v)) return launch_prompt_tc(g, q, k, v, st);
    if (prompt_mma_supported(g, p->dtype, q, k, v)) return launch_prompt_mma(g, q, k, v, st);
    if (prompt_f32_supported(g, p->dtype, q, k, v)) return launch_prompt_f32(g, q, k, v, st);
    return launch_prompt_generic(g, p->dtype, q, k, v, st);
}

size_t stream_cache_workspace_bytes(const stream_cache *c) {
    CacheGeom g;
    if (make_cache(c, &g) != STREAM_OK) return 0;
    return ledger_workspace_bytes(g);
}

stream_status stream_cache_reserve(const stream_cache *c, const int32_t *n_new, int32_t *page_table, int32_t *seq_len,
                                   int32_t *ref_count, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_ledger(c, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes, &g);
    if (rc != STREAM_OK) return rc;
    if (n_new == nullptr || !natural(n_new, 4)) return invalid("n_new must be a 4-byte aligned device array");
    return launch_reserve(g, n_new, info_out, workspace, (cudaStream_t)cuda_stream);
}

stream_status stream_cache_fork(const stream_cache *c, const int32_t *parent, int32_t *page_table, int32_t *seq_len,
                                int32_t *ref_count, int32_t *pairs_out, int32_t *info_out, void *workspace, size_t workspace_bytes,
                                void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_ledger(c, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes, &g);
    if (rc != STREAM_OK) return rc;
    if (parent == nullptr || pairs_out == nullptr || !natural(parent, 4) || !natural(pairs_out, 8))
        return invalid("parent and pairs_out must be device arrays, 4-byte and 8-byte aligned");
    return launch_fork(g, parent, pairs_out, info_out, workspace, (cudaStream_t)cuda_stream);
}

stream_status stream_cache_free(const stream_cache *c, const int32_t *done, int32_t *page_table, int32_t *seq_len,
                                int32_t *ref_count, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_ledger(c, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes, &g);
    if (rc != STREAM_OK) return rc;
    if (done == nullptr || !natural(done, 4)) return invalid("done must be a 4-byte aligned device array");
    return launch_free(g, done, info_out, workspace, (cudaStream_t)cuda_stream);
}

stream_status stream_cache_compact(const stream_cache *c, int32_t *page_table, int32_t *seq_len, int32_t *ref_count,
                                   int32_t *pairs_out, int32_t *info_out, void *workspace, size_t workspace_bytes, void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_ledger(c, page_table, seq_len, ref_count, info_out, workspace, workspace_bytes, &g);
    if (rc != STREAM_OK) return rc;
    if ((pairs_out == nullptr && g.n_pages > 1) || !natural(pairs_out, 8)) return invalid("pairs_out must be an 8-byte aligned device array");
    return launch_compact(g, pairs_out, info_out, workspace, (cudaStream_t)cuda_stream);
}

stream_status stream_cache_copy_pages(const stream_cache *c, void *k_pages, void *v_pages, const int32_t *pairs,
                                      const int32_t *count, int32_t n_pairs, void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_cache(c, &g);
    if (rc != STREAM_OK) return rc;
    if (n_pairs < 0) return invalid("n_pairs must not be negative");
    if (n_pairs == 0) return STREAM_OK;
    const int e = elem_bytes(c->dtype);
    if (k_pages == nullptr || v_pages == nullptr || pairs == nullptr || count == nullptr) return invalid("k_pages, v_pages, pairs and count must not be NULL");
    if (!natural(k_pages, e) || !natural(v_pages, e) || !natural(pairs, 4) || !natural(count, 4)) return invalid("a pointer is not aligned to its elements");
    return launch_copy_pages(g, e, k_pages, v_pages, pairs, count, n_pairs, (cudaStream_t)cuda_stream);
}

stream_status stream_cache_write(const stream_cache *c, int32_t layer, const void *k, const void *v, int64_t total,
                                 int64_t stride_t, int64_t stride_h, const int32_t *cu_new, const int32_t *page_table,
                                 const int32_t *seq_len, const int32_t *done, void *k_pages, void *v_pages, void *cuda_stream) {
    CacheGeom g;
    stream_status rc = make_cache(c, &g);
    if (rc != STREAM_OK) return rc;
    if (layer < 0 || layer >= g.n_layers) return invalid("no such layer");
    if (total < 0 || total > 0x7fffffffLL) return invalid("total must be 0 .. 2^31 - 1");
    if (!strides_ok(total, stride_t, g.G, stride_h, g.d)) return invalid("token and head strides must be >= d");
    if (cu_new == nullptr || page_table == nullptr || seq_len == nullptr) return invalid("cu_new, page_table and seq_len must not be NULL");
    if (total == 0) return STREAM_OK;
    if (k == nullptr || v == nullptr || k_pages == nullptr || v_pages == nullptr) return invalid("k, v, k_pages and v_pages must not be NULL");
    const int e = elem_bytes(c->dtype);
    if (!natural(k, e) || !natural(v, e) || !natural(k_pages, e) || !natural(v_pages, e) || !natural(cu_new, 4) || !natural(page_table, 4) || !natural(seq_len, 4) || !natural(done, 4))
        return invalid("a pointer is not aligned to its elements");
    g.table = const_cast<int32_t *>(page_table);
    g.len = const_cast<int32_t *>(seq_len);
    const long long at = (long long)layer * g.s_l * e;
    return launch_write(g, e, k, v, (int)total, total > 1 ? stride_t : (long long)g.G * g.d, g.G > 1 ? stride_h : g.d, cu_new, done,
                        (char *)k_pages + at, (char *)v_pages + at, (cudaStream_t)cuda_stream);
}

size_t stream_decode_workspace_bytes(const stream_cache *c, int32_t n_q_heads) {
    CacheGeom g;
    if (make_cache(c, &g) != STREAM_OK) return 0;
    if (n_q_heads < 1 || n_q_heads % g.G != 0) { set_error("n_kv_heads must divide n_q_heads"); return 0; }
    return decode_workspace_bytes(g);
}

stream_status stream_decode_attention(const stream_cache *c, int32_t layer, int32_t n_q_heads, const void *q, int64_t q_stride_s,
                                      int64_t q_stride_h, const void *k_pages, const void *v_pages, const int32_t *page_table,
                                      const int32_t *seq_len, float scale, void *out, float *lse_out, void *workspace,
                                      size_t workspace_bytes, void *cuda_stream) {
    DecodeCall a;
    stream_status rc = make_cache(c, &a.c);
    if (rc != STREAM_OK) return rc;
    if (layer < 0 || layer >= a.c.n_layers) return invalid("no such layer");
    if (n_q_heads < 1 || n_q_heads % a.c.G != 0) return invalid("n_kv_heads must divide n_q_heads");
    if (!strides_ok(a.c.n_slots, q_stride_s, n_q_heads, q_stride_h, a.c.d)) return invalid("slot and head strides of q must be >= d");
    if (q == nullptr || k_pages == nullptr || v_pages == nullptr || page_table == nullptr || seq_len == nullptr || out == nullptr)
        return invalid("q, k_pages, v_pages, page_table, seq_len and out must not be NULL");
    const int e = elem_bytes(c->dtype);
    if (!natural(q, e) || !natural(k_pages, e) || !natural(v_pages, e) || !natural(out, e) || !natural(page_table, 4) || !natural(seq_len, 4) || !natural(lse_out, 4))
        return invalid("a pointer is not aligned to its elements");
    if ((long long)a.c.n_slots * n_q_heads > 0x7fffffffLL / 256) { set_error("too many slots and heads for 32-bit indexing"); return STREAM_ERR_UNSUPPORTED; }
    rc = make_scale(scale, a.c.d, &a.scale_log2);
    if (rc != STREAM_OK) return rc;
    const size_t need = decode_workspace_bytes(a.c);
    if (workspace == nullptr || workspace_bytes < need || ((uintptr_t)workspace & 255) != 0) {
        set_error("workspace must be a 256-byte aligned device buffer of at least %zu bytes", need);
        return STREAM_ERR_WORKSPACE;
    }
    a.c.table = const_cast<int32_t *>(page_table);
    a.c.len = const_cast<int32_t *>(seq_len);
    a.H = n_q_heads; a.hpg = n_q_heads / a.c.G;
    a.qs_s = a.c.n_slots > 1 ? q_stride_s : (long long)n_q_heads * a.c.d;
    a.qs_h = n_q_heads > 1 ? q_stride_h : a.c.d;
    const long long at = (long long)layer * a.c.s_l * e;
    a.q = q; a.k = (const char *)k_pages + at; a.v = (const char *)v_pages + at;
    a.out = out; a.lse = lse_out;
    return launch_decode(a, c->dtype, workspace, (cudaStream_t)cuda_stream);
}

}  // extern "C"
