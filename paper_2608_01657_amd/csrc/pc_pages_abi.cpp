// pc_pages_abi.cpp -- the host side of the page operators, of the groups of a
// keyed batch and of the attention over shared prefixes (include/pc.h):
// validation and launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "pc.h"
#include "pc_host.h"
#include "pc_pages.h"

using namespace pcr;

namespace {

bool aligned(const void *p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int32_t check_pool(const pc_pages *p, bool data = true) {
    if (!p) return fail(PC_EINVAL, "pages is NULL");
    if (p->n_pages < 1 || p->n_pages > PC_MAX_POOL_PAGES) return fail(PC_EINVAL, "n_pages %d out of range", p->n_pages);
    if (p->n_seqs < 1 || p->n_seqs > PC_MAX_SEQS) return fail(PC_EINVAL, "n_seqs %d out of range", p->n_seqs);
    if (p->table_width < 1 || p->table_width > 1 << 24)
        return fail(PC_EINVAL, "table_width %d out of range", p->table_width);
    if (p->n_layers < 1 || p->n_layers > 4096) return fail(PC_EINVAL, "n_layers %d out of range", p->n_layers);
    if (p->n_kv_heads < 1 || p->n_kv_heads > 256) return fail(PC_EINVAL, "n_kv_heads %d out of range", p->n_kv_heads);
    if (p->head_dim != 64 && p->head_dim != 128)
        return fail(PC_EUNSUPPORTED, "head_dim %d: only 64 and 128 are implemented", p->head_dim);
    if (p->dtype != PC_BF16 && p->dtype != PC_FP16) return fail(PC_EINVAL, "unknown dtype %d", p->dtype);
    if (p->layout != PC_HEADS_FIRST && p->layout != PC_TOKENS_FIRST)
        return fail(PC_EINVAL, "unknown layout %d", p->layout);
    const int64_t page = (int64_t)kBlk * p->n_kv_heads * p->head_dim;
    if (p->n_pages > 1 && (p->page_stride < page || p->page_stride > 1LL << 40 || p->page_stride % 8))
        return fail(PC_EINVAL, "page_stride %lld: at least a page's %lld elements and a multiple of 8",
                    (long long)p->page_stride, (long long)page);
    if (p->n_layers > 1 && (p->layer_stride < page || p->layer_stride > 1LL << 46 || p->layer_stride % 8))
        return fail(PC_EINVAL, "layer_stride %lld: at least a page's %lld elements and a multiple of 8",
                    (long long)p->layer_stride, (long long)page);
    if (!p->d_table || !p->d_len || !aligned(p->d_table, 4) || !aligned(p->d_len, 4))
        return fail(PC_EINVAL, "d_table or d_len is NULL or misaligned");
    if (!data) return PC_OK;
    if (!p->d_refs || !aligned(p->d_refs, 4)) return fail(PC_EINVAL, "d_refs is NULL or misaligned");
    if (!p->d_k || !p->d_v || !aligned(p->d_k, 16) || !aligned(p->d_v, 16))
        return fail(PC_EINVAL, "d_k or d_v is NULL or not 16-byte aligned");
    return PC_OK;
}

int32_t check_rows(const pc_rows *r, int64_t tokens, int32_t heads, const char *what) {
    if (!r || !r->d_data || !aligned(r->d_data, 16)) return fail(PC_EINVAL, "%s is NULL or not 16-byte aligned", what);
    if ((tokens > 1 && r->token_stride % 8) || (heads > 1 && r->head_stride % 8))
        return fail(PC_EINVAL, "%s: strides must be multiples of 8 elements", what);
    return PC_OK;
}

int32_t check_list(const pc_pages *p, int32_t n, const void *a, const void *b, const int32_t *status) {
    if (n < 0 || n > p->n_seqs) return fail(PC_EINVAL, "a list of %d sequences of a pool of %d", n, p->n_seqs);
    if (n && (!a || !b)) return fail(PC_EINVAL, "a list is NULL");
    if (!status || !aligned(status, 4)) return fail(PC_EINVAL, "d_status is NULL or misaligned");
    return PC_OK;
}

int32_t check_ws(const void *ws, int64_t have, int64_t need) {
    if (!ws || !aligned(ws, 256)) return fail(PC_EINVAL, "d_workspace is NULL or not 256-byte aligned");
    if (have < need)
        return fail(PC_ENOMEM, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
    return PC_OK;
}

int32_t done(hipError_t e, const char *what) { return e == hipSuccess ? ok() : hip_fail(e, what); }

int32_t check_batch(const pc_pages *p, int32_t n_req, int64_t n_tokens, int32_t n_heads) {
    if (n_req < 1) return fail(PC_EINVAL, "n_req %d out of range", n_req);
    if (n_req > PC_MAX_BATCH) return fail(PC_EUNSUPPORTED, "n_req %d: at most %d", n_req, PC_MAX_BATCH);
    if (n_tokens < 0 || n_tokens > 1 << 28) return fail(PC_EINVAL, "n_tokens %lld out of range", (long long)n_tokens);
    if (n_heads < 1 || n_heads > 4096 || n_heads % p->n_kv_heads)
        return fail(PC_EINVAL, "n_heads %d: a multiple of n_kv_heads %d, at most 4096", n_heads, p->n_kv_heads);
    if (attn_ws(n_req, n_tokens, n_heads, p->n_kv_heads, p->head_dim, nullptr, nullptr) < 0)
        return fail(PC_EUNSUPPORTED, "n_tokens %lld x n_heads %d: over 2^31 partial rows", (long long)n_tokens, n_heads);
    return PC_OK;
}

}  // namespace

extern "C" {

int64_t pc_pages_workspace_bytes(const pc_pages *pages, int64_t n) {
    if (int32_t rc = check_pool(pages, false)) return rc;
    if (n < 0 || n > pages->n_seqs) return fail(PC_EINVAL, "a list of %lld sequences of a pool of %d", (long long)n, pages->n_seqs);
    ok();
    return pages_ws(*pages, n, nullptr, nullptr);
}

int32_t pc_pages_fork(const pc_pages *pages, const int32_t *d_parent, const int32_t *d_child, int32_t n,
                      int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (int32_t rc = check_list(pages, n, d_parent, d_child, d_status)) return rc;
    if (n == 0) return ok();
    return done(launch_fork(*pages, d_parent, d_child, n, d_status, static_cast<hipStream_t>(stream)), "pc_pages_fork");
}

int32_t pc_pages_extend(const pc_pages *pages, const int32_t *d_seq, const int32_t *d_add, int32_t n,
                        void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (int32_t rc = check_list(pages, n, d_seq, d_add, d_status)) return rc;
    if (n > PC_MAX_BATCH) return fail(PC_EUNSUPPORTED, "%d sequences: at most %d", n, PC_MAX_BATCH);
    if (int32_t rc = check_ws(d_workspace, workspace_bytes, pages_ws(*pages, n, nullptr, nullptr))) return rc;
    if (n == 0) return ok();
    PagesWs ws;
    pages_ws(*pages, n, static_cast<char *>(d_workspace), &ws);
    return done(launch_extend(*pages, d_seq, d_add, n, ws, d_status, static_cast<hipStream_t>(stream)), "pc_pages_extend");
}

int32_t pc_pages_free(const pc_pages *pages, const int32_t *d_seq, int32_t n, int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (int32_t rc = check_list(pages, n, d_seq, d_seq, d_status)) return rc;
    if (n == 0) return ok();
    return done(launch_free(*pages, d_seq, n, d_status, static_cast<hipStream_t>(stream)), "pc_pages_free");
}

int32_t pc_pages_compact(const pc_pages *pages, int32_t *d_refs_to, int32_t *d_table_to, int32_t *d_n_live,
                         void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (!d_refs_to || !d_table_to || !d_n_live) return fail(PC_EINVAL, "d_refs_to, d_table_to or d_n_live is NULL");
    if (int32_t rc = check_list(pages, 0, nullptr, nullptr, d_status)) return rc;
    if (int32_t rc = check_ws(d_workspace, workspace_bytes, pages_ws(*pages, 0, nullptr, nullptr))) return rc;
    PagesWs ws;
    pages_ws(*pages, 0, static_cast<char *>(d_workspace), &ws);
    return done(launch_compact(*pages, d_refs_to, d_table_to, d_n_live, ws, d_status, static_cast<hipStream_t>(stream)),
                "pc_pages_compact");
}

int32_t pc_pages_write(const pc_pages *pages, int32_t layer, const int32_t *d_seq, const int32_t *d_new_off,
                       int32_t n, int64_t n_tokens, const pc_rows *k_new, const pc_rows *v_new,
                       int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (layer < 0 || layer >= pages->n_layers) return fail(PC_EINVAL, "layer %d of %d", layer, pages->n_layers);
    if (int32_t rc = check_list(pages, n, d_seq, d_new_off, d_status)) return rc;
    if (n_tokens < 0 || n_tokens > 1 << 28) return fail(PC_EINVAL, "n_tokens %lld out of range", (long long)n_tokens);
    if (n == 0 || n_tokens == 0) return ok();
    if (int32_t rc = check_rows(k_new, n_tokens, pages->n_kv_heads, "k_new")) return rc;
    if (int32_t rc = check_rows(v_new, n_tokens, pages->n_kv_heads, "v_new")) return rc;
    return done(launch_write(*pages, layer, d_seq, d_new_off, n, n_tokens, *k_new, *v_new, d_status,
                             static_cast<hipStream_t>(stream)), "pc_pages_write");
}

int32_t pc_prefix_groups(const uint64_t *d_keys, int64_t n_keys, const int64_t *d_key_off, int32_t n_req,
                         int32_t min_blocks, int32_t *d_order, int32_t *d_group_off, int32_t *d_shared,
                         int32_t *d_n_groups, int32_t *d_status, void *stream) {
    if (n_req < 1) return fail(PC_EINVAL, "n_req %d out of range", n_req);
    if (n_req > PC_MAX_BATCH) return fail(PC_EUNSUPPORTED, "n_req %d: at most %d", n_req, PC_MAX_BATCH);
    if (min_blocks < 1) return fail(PC_EINVAL, "min_blocks %d: at least 1", min_blocks);
    if (n_keys < 0 || (n_keys && !d_keys) || !aligned(d_keys, 8)) return fail(PC_EINVAL, "d_keys is NULL or misaligned");
    if (!d_key_off || !d_order || !d_group_off || !d_shared || !d_n_groups || !d_status)
        return fail(PC_EINVAL, "a pointer is NULL");
    return done(launch_groups(d_keys, n_keys, d_key_off, n_req, min_blocks, d_order, d_group_off, d_shared, d_n_groups,
                              d_status, static_cast<hipStream_t>(stream)), "pc_prefix_groups");
}

int64_t pc_attn_workspace_bytes(const pc_pages *pages, int32_t n_req, int64_t n_tokens, int32_t n_heads) {
    if (int32_t rc = check_pool(pages, false)) return rc;
    if (int32_t rc = check_batch(pages, n_req, n_tokens, n_heads)) return rc;
    ok();
    return attn_ws(n_req, n_tokens, n_heads, pages->n_kv_heads, pages->head_dim, nullptr, nullptr);
}

int32_t pc_attn_plan(const pc_pages *pages, const int32_t *d_seq, const int32_t *d_q_off, int32_t n_req,
                     int64_t n_tokens, int32_t n_heads, int32_t causal, const int32_t *d_order,
                     const int32_t *d_group_off, const int32_t *d_shared, const int32_t *d_n_groups,
                     void *d_workspace, int64_t workspace_bytes, int32_t *d_status, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (int32_t rc = check_batch(pages, n_req, n_tokens, n_heads)) return rc;
    if (!d_seq || !d_q_off) return fail(PC_EINVAL, "d_seq or d_q_off is NULL");
    if (!d_status || !aligned(d_status, 4)) return fail(PC_EINVAL, "d_status is NULL or misaligned");
    const int given = !!d_order + !!d_group_off + !!d_shared + !!d_n_groups;
    if (given != 0 && given != 4) return fail(PC_EINVAL, "groups are given by all of their arrays or none");
    if (causal != 0 && causal != 1) return fail(PC_EINVAL, "causal is 0 or 1");
    AttnPlanArgs a{*pages, d_seq, d_q_off, d_order, d_group_off, d_shared, d_n_groups, n_req, n_heads, causal, n_tokens, {}, d_status};
    const int64_t need = attn_ws(n_req, n_tokens, n_heads, pages->n_kv_heads, pages->head_dim,
                                 static_cast<char *>(d_workspace), &a.ws);
    if (int32_t rc = check_ws(d_workspace, workspace_bytes, need)) return rc;
    return done(launch_attn_plan(a, static_cast<hipStream_t>(stream)), "pc_attn_plan");
}

int32_t pc_attn(const pc_pages *pages, int32_t layer, const pc_rows *q, int32_t n_req, int64_t n_tokens,
                int32_t n_heads, float scale, const pc_rows *out, float *d_lse, void *d_workspace,
                int64_t workspace_bytes, void *stream) {
    if (int32_t rc = check_pool(pages)) return rc;
    if (layer < 0 || layer >= pages->n_layers) return fail(PC_EINVAL, "layer %d of %d", layer, pages->n_layers);
    if (int32_t rc = check_batch(pages, n_req, n_tokens, n_heads)) return rc;
    const float scale_log2 = (float)(scale * 1.4426950408889634);
    if (!(scale > 0) || !std::isfinite(scale_log2))
        return fail(PC_EINVAL, "scale must be positive, and scale log2(e) finite");
    if (n_tokens == 0) return ok();
    if (int32_t rc = check_rows(q, n_tokens, n_heads, "q")) return rc;
    if (int32_t rc = check_rows(out, n_tokens, n_heads, "out")) return rc;
    if (!aligned(d_lse, 4)) return fail(PC_EINVAL, "d_lse is misaligned");
    const bool heads_first = pages->layout == PC_HEADS_FIRST;
    AttnArgs a{};
    const int64_t need = attn_ws(n_req, n_tokens, n_heads, pages->n_kv_heads, pages->head_dim,
                                 static_cast<char *>(d_workspace), &a.ws);
    if (int32_t rc = check_ws(d_workspace, workspace_bytes, need)) return rc;
    const int64_t off = layer ? (int64_t)layer * pages->layer_stride : 0;
    a.k = static_cast<const uint16_t *>(pages->d_k) + off;
    a.v = static_cast<const uint16_t *>(pages->d_v) + off;
    a.q = q->d_data;
    a.out = out->d_data;
    a.lse_out = d_lse;
    a.table = pages->d_table;
    a.page_stride = pages->page_stride;
    a.q_token = q->token_stride;
    a.q_head = q->head_stride;
    a.out_token = out->token_stride;
    a.out_head = out->head_stride;
    a.head_stride = heads_first ? kBlk * pages->head_dim : pages->head_dim;
    a.token_stride = heads_first ? pages->head_dim : pages->n_kv_heads * pages->head_dim;
    a.table_width = pages->table_width;
    a.n_pages = pages->n_pages;
    a.n_heads = n_heads;
    a.group = n_heads / pages->n_kv_heads;
    a.scale_log2 = scale_log2;
    a.n_req = n_req;
    a.n_seqs = pages->n_seqs;
    a.head_dim = pages->head_dim;
    a.n_tokens = n_tokens;
    return done(launch_attn(a, pages->dtype, static_cast<hipStream_t>(stream)), "pc_attn");
}

}  // extern "C"
