// Entry points of the paged 4-bit cache (include/gsa.h): argument checks, workspaces, launches.
#include "gsa_cache.cuh"

using namespace gsa;
typedef __nv_bfloat16 bf16;

namespace {

int log2_exact(int v) {
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

// geometry only; fills *v but for the pointers
int check_geometry(const gsa_cache_t* c, CacheView* v) {
    if (!c || c->B < 1 || c->n_pages < 1 || c->max_pages < 1) return GSA_ERR_INVALID_ARG;
    if (!one_of(c->page_tokens, {16, 32, 64, 128}) || !one_of(c->n_kv, {1, 2, 4, 8}) || !one_of(c->d_h, {64, 128}) ||
        !one_of(c->dI, {32, 64}))
        return GSA_ERR_UNSUPPORTED_SHAPE;
    if (c->B > 4096 || c->n_pages > (1 << 20) || (int64_t)c->max_pages * c->page_tokens >= (1 << 24)) return GSA_ERR_UNSUPPORTED_SHAPE;
    const int D = c->n_kv * c->d_h;
    v->n_pages = c->n_pages; v->T = c->page_tokens; v->log_t = log2_exact(c->page_tokens);
    v->max_pages = c->max_pages; v->B = c->B; v->n_kv = c->n_kv; v->d_h = c->d_h; v->dI = c->dI;
    v->rec = (int32_t)align_up((size_t)D + D / 8, 16);
    v->keys_off = v->T * v->rec;
    v->page_bytes = (int64_t)v->T * (v->rec + 2 * c->dI);
    if (v->page_bytes * c->n_pages > 1ll << 36) return GSA_ERR_UNSUPPORTED_SHAPE;          // (the attention counts 16 bytes in 32 bits)
    return GSA_OK;
}

int check_cache(const gsa_cache_t* c, CacheView* v) {
    const int rc = check_geometry(c, v);
    if (rc) return rc;
    if (!c->pool || !c->table || !c->lens || !c->refs || !aligned32(c->pool)) return GSA_ERR_INVALID_ARG;
    v->pool = (unsigned char*)c->pool; v->table = c->table; v->lens = c->lens; v->refs = c->refs;
    return GSA_OK;
}

// a stage on the cache: the parameters have to fit it
int check_stage(const gsa_cache_t* c, const gsa_params_t* p, CacheView* v) {
    int rc = check_cache(c, v);
    if (rc) return rc;
    if ((rc = check_params(p))) return rc;
    if (p->B != c->B || p->n_kv != c->n_kv || p->d_h != c->d_h || p->dI != c->dI) return GSA_ERR_INVALID_ARG;
    if ((int64_t)p->Lk > (int64_t)c->max_pages * c->page_tokens) return GSA_ERR_INVALID_ARG;
    return GSA_OK;
}

size_t list_ws_bytes(const CacheView& v) {
    const size_t lists = cache_page_list_bytes(v), flags = kMaxFlags * 4;
    return kStatusBytes + (lists > flags ? lists : flags);
}

bool ws_ok(const void* ws, size_t have, size_t need) { return ws && aligned16(ws) && have >= need; }

}  // namespace

extern "C" {

int gsa_cache_page_bytes(const gsa_cache_t* c, size_t* bytes) {
    CacheView v{};
    const int rc = check_geometry(c, &v);
    if (rc) return rc;
    if (!bytes) return GSA_ERR_INVALID_ARG;
    *bytes = (size_t)v.page_bytes;
    return GSA_OK;
}

int gsa_cache_workspace_bytes(const gsa_cache_t* c, size_t* bytes) {
    CacheView v{};
    const int rc = check_geometry(c, &v);
    if (rc) return rc;
    if (!bytes) return GSA_ERR_INVALID_ARG;
    *bytes = list_ws_bytes(v);
    return GSA_OK;
}

int gsa_cache_reserve(const gsa_cache_t* c, const int32_t* n_new, int32_t* start, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (!n_new || !start || n_new == start) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_reserve(v, n_new, start, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_append(const gsa_cache_t* c, int32_t L_new, const void* K, const void* V, const void* g2_logits, const void* kI,
                     const int32_t* n_new, const int32_t* start, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (L_new < 1 || L_new > (int64_t)v.max_pages * v.T) return GSA_ERR_INVALID_ARG;
    if (!K || !V || !kI || !aligned32(K) || !aligned32(V) || !aligned16(kI)) return GSA_ERR_INVALID_ARG;
    if ((g2_logits && !aligned32(g2_logits)) || !n_new || !start || n_new == start) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_append(v, L_new, (const bf16*)K, (const bf16*)V, (const bf16*)g2_logits, (const bf16*)kI, n_new, start,
                                       (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_read(const gsa_cache_t* c, int32_t L, void* K, void* V, void* kI, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (L < 1 || L > (int64_t)v.max_pages * v.T || (!K && !V && !kI)) return GSA_ERR_INVALID_ARG;
    if (!aligned32(K) || !aligned32(V) || !aligned16(kI)) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_read(v, L, (bf16*)K, (bf16*)V, (bf16*)kI, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_fork(const gsa_cache_t* c, const int32_t* src_of, int32_t share, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (!src_of) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_fork(v, src_of, share != 0, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_release(const gsa_cache_t* c, const int32_t* drop, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (!drop) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_release(v, drop, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_compact(const gsa_cache_t* c, int32_t* live_pages, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    const int rc = check_cache(c, &v);
    if (rc) return rc;
    if (!live_pages) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_compact(v, live_pages, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_indexer_scores(const gsa_cache_t* c, const gsa_params_t* p, const void* qI, const float* w, const float* bI,
                             float* scores, int64_t row_stride, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    int rc = check_stage(c, p, &v);
    if (rc) return rc;
    if (!qI || !w || !scores || !aligned16(qI) || !aligned16(w) || !aligned16(scores)) return GSA_ERR_INVALID_ARG;
    if (row_stride < p->Lk || row_stride % 4 != 0) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_indexer(v, *p, (const bf16*)qI, w, bI, scores, row_stride, (int32_t*)ws, (cudaStream_t)stream));
}

int gsa_cache_topk(const gsa_cache_t* c, const gsa_params_t* p, const float* scores, int64_t row_stride, int32_t* idx, int32_t* kt,
                   float* var, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    int rc = check_stage(c, p, &v);
    if (rc) return rc;
    if (!scores || !idx || !kt || !aligned16(scores) || !aligned16(idx)) return GSA_ERR_INVALID_ARG;
    if (row_stride < p->Lk || row_stride % 4 != 0) return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, list_ws_bytes(v))) return GSA_ERR_WORKSPACE;
    // (the fallback counter in the head counts up)
    t_dev_status = (int32_t*)ws;
    if ((rc = cuda_rc(launch_clear((cudaStream_t)stream, {ws, (size_t)kStatusBytes})))) return rc;
    const RowRange rr{0, p->B, 0, p->Lq};
    const IdxLayout il{0, 0, p->Lq};
    return cuda_rc(launch_select(*p, rr, scores, row_stride, idx, kt, var, il, (int32_t*)ws + kStatusFallbackWord,
                                 (cudaStream_t)stream, v.lens));
}

int gsa_cache_attn_workspace_bytes(const gsa_params_t* p, size_t* bytes) {
    const int rc = check_params(p);
    if (rc) return rc;
    if (!bytes) return GSA_ERR_INVALID_ARG;
    *bytes = kStatusBytes + cache_attn_scratch_bytes(*p);
    return GSA_OK;
}

int gsa_cache_attn_fwd(const gsa_cache_t* c, const gsa_params_t* p, const void* Q, const void* g1_logits, const int32_t* idx,
                       const int32_t* kt, void* out, void* ws, size_t ws_bytes, void* stream) {
    CacheView v{};
    int rc = check_stage(c, p, &v);
    if (rc) return rc;
    if (!Q || !g1_logits || !idx || !kt || !out || !aligned16(Q) || !aligned16(g1_logits) || !aligned16(idx) || !aligned16(out))
        return GSA_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, kStatusBytes + cache_attn_scratch_bytes(*p))) return GSA_ERR_WORKSPACE;
    return cuda_rc(launch_cache_attn(v, *p, (const bf16*)Q, (const bf16*)g1_logits, idx, kt, (bf16*)out, (int32_t*)ws,
                                     (cudaStream_t)stream));
}

}  // extern "C"
