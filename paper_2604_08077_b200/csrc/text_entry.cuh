// Entry points of the text operators (include/adaspark_attn.h, "Text beside the video"): argument checks and launches.
// Included by adaspark_attn.cu, whose handle and launch helpers they use.
#pragma once
#include "attn_prompt.cuh"
#include "paged_cache.cuh"
#include "paged_decode.cuh"

namespace {

// The handle's device for the length of a call; the caller's is current again afterwards.
struct DeviceScope {
    int before = -1;
    bool changed = false;
    adaspark_status_t enter(adaspark_attn* h, const char* who) {
        cudaError_t e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != h->cfg.device) {
            e = cudaSetDevice(h->cfg.device);
            changed = e == cudaSuccess;
        }
        if (e == cudaSuccess && h->sm_count <= 0) e = cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->cfg.device);
        return e == cudaSuccess ? ADASPARK_OK : fail(h, ADASPARK_ERR_CUDA, "%s: device %d: %s", who, h->cfg.device, cudaGetErrorString(e));
    }
    ~DeviceScope() { if (changed) (void)cudaSetDevice(before); }
};

float text_scale(const adaspark_attn* h) {
    return h->cfg.softmax_scale > 0.f ? h->cfg.softmax_scale : 1.f / std::sqrt((float)h->cfg.head_dim);
}

// bf16 rows [n][heads][D] with strides in elements, 0 standing for the dense ones
struct Rows {
    const __nv_bfloat16* p;
    long long ts, hs;
};
adaspark_status_t check_rows(adaspark_attn* h, const char* who, const char* what, const void* p, int64_t ts, int64_t hs, int heads, Rows& r) {
    const int D = h->cfg.head_dim;
    r.p = (const __nv_bfloat16*)p;
    r.hs = hs ? hs : D;
    r.ts = ts ? ts : (long long)heads * D;
    if (!p) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL %s", who, what);
    if ((uintptr_t)p % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", who, what);
    if (r.hs < D || r.ts < D || r.hs % 8 || r.ts % 8 || r.hs >= (1ll << 38) || r.ts >= (1ll << 38))
        return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: strides of %s (%lld, %lld elements) are not multiples of 8 of at least head_dim", who, what, r.ts, r.hs);
    return ADASPARK_OK;
}

adaspark_status_t check_pages(adaspark_attn* h, const char* who, const adaspark_attn_pages_t* pages, const int32_t* block_table, int32_t table_width, PageGeom& g) {
    if (!pages || !block_table) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pages or block table", who);
    const int D = h->cfg.head_dim, Hkv = h->cfg.n_kv_heads;
    const bool e4m3 = pages->format == ADASPARK_PAGES_E4M3;
    if (pages->format != ADASPARK_PAGES_BF16 && !e4m3) return fail(h, ADASPARK_ERR_UNSUPPORTED, "%s: unknown page format %d", who, pages->format);
    int shift = 4;
    while (shift < 8 && (1 << shift) != pages->page_size) ++shift;
    if ((1 << shift) != pages->page_size) return fail(h, ADASPARK_ERR_UNSUPPORTED, "%s: page_size %d is not one of 16, 32, 64, 128, 256", who, pages->page_size);
    if (pages->n_pages <= 0 || table_width <= 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: %d pages, block table of %d columns", who, pages->n_pages, table_width);
    if (((long long)table_width << shift) > 0x7fffffffll) return fail(h, ADASPARK_ERR_UNSUPPORTED, "%s: %d pages a sequence hold more than 2^31 - 1 tokens", who, table_width);
    const long long dense = (long long)Hkv * D << shift, dense_s = (long long)Hkv << shift;
    const int elem = e4m3 ? 1 : 2;
    g.page_stride = pages->page_stride ? pages->page_stride : dense;
    g.scale_stride = pages->scale_stride ? pages->scale_stride : dense_s;
    if (!pages->k_pages || !pages->v_pages || (e4m3 && (!pages->k_scale || !pages->v_scale)))
        return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pages or scales", who);
    if ((uintptr_t)pages->k_pages % 16 || (uintptr_t)pages->v_pages % 16 || (e4m3 && ((uintptr_t)pages->k_scale % 16 || (uintptr_t)pages->v_scale % 16)))
        return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: pages or scales are not 16-byte aligned", who);
    if (g.page_stride < dense || g.page_stride * elem % 16 || g.page_stride >= (1ll << 38) || (e4m3 && (g.scale_stride < dense_s || g.scale_stride % 16)))
        return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: strides of the pages (%lld elements, scales %lld bytes) are below a page's size or no multiple of 16 bytes", who,
                    g.page_stride, g.scale_stride);
    g.k = (uint8_t*)pages->k_pages;
    g.v = (uint8_t*)pages->v_pages;
    g.ks = e4m3 ? pages->k_scale : nullptr;
    g.vs = e4m3 ? pages->v_scale : nullptr;
    g.table = block_table;
    g.table_width = table_width;
    g.n_pages = pages->n_pages;
    g.page_shift = shift;
    g.Hkv = Hkv;
    return ADASPARK_OK;
}

#define ADASPARK_TRY(expr)                       \
    do {                                         \
        const adaspark_status_t st_ = (expr);    \
        if (st_ != ADASPARK_OK) return st_;      \
    } while (0)

}  // namespace

extern "C" {

int64_t adaspark_attn_text_workspace_bytes(const adaspark_attn_t* h) {
    return h ? (int64_t)align_up(paged_partial_bytes(h->cfg.head_dim, h->cfg.n_q_heads / h->cfg.n_kv_heads)) : 0;
}

adaspark_status_t adaspark_attn_prompt(adaspark_attn_t* h, const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                                       int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, const int32_t* cu_q,
                                       const int32_t* cu_k, int32_t batch, int32_t n_q, int32_t n_k, void* out, float* lse, void* workspace,
                                       size_t workspace_bytes, int32_t* status, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "prompt";
    if (batch < 0 || n_q < 0 || n_k < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: negative size", who);
    h->launches = 0;
    if (batch == 0 || n_q == 0) return ADASPARK_OK;
    Rows rq, rk, rv;
    ADASPARK_TRY(check_rows(h, who, "q", q, q_token_stride, q_head_stride, h->cfg.n_q_heads, rq));
    if (n_k) {
        ADASPARK_TRY(check_rows(h, who, "k", k, k_token_stride, k_head_stride, h->cfg.n_kv_heads, rk));
        ADASPARK_TRY(check_rows(h, who, "v", v, v_token_stride, v_head_stride, h->cfg.n_kv_heads, rv));
    } else {                                       // no keys at all: k and v may be NULL; the tensor maps need some row, which no row sees
        rk = rv = {rq.p, (long long)h->cfg.n_kv_heads * h->cfg.head_dim, h->cfg.head_dim};
    }
    if (!cu_q || !cu_k || !out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pointer", who);
    if ((uintptr_t)out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: out is not 16-byte aligned", who);
    if (!workspace || (uintptr_t)workspace % kAlign) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", who);
    if (workspace_bytes < (size_t)adaspark_attn_text_workspace_bytes(h)) return fail(h, ADASPARK_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu bytes", who, workspace_bytes);
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    PromptGeom g;
    g.cu_q = cu_q;
    g.cu_k = cu_k;
    g.batch = batch;
    g.n_q = n_q;
    g.n_k = n_k;
    g.Hq = h->cfg.n_q_heads;
    g.Hkv = h->cfg.n_kv_heads;
    g.G = g.Hq / g.Hkv;
    g.T = 128 / g.G;
    g.div_w.init(2 * g.T);
    g.div_g.init(g.G);
    g.div_kv.init(g.Hkv);
    g.scale_log2 = text_scale(h) * 1.4426950408889634f;
    g.v = rv.p;
    g.v_ts = rv.ts;
    g.v_hs = rv.hs;
    const int D = h->cfg.head_dim, n_rows = n_k ? n_k : 1;
    CUtensorMap tmQ, tmK, tmV;
    if (!encode_bf16_rows(&tmQ, rq.p, n_q, g.Hq, D, rq.ts, rq.hs, 64, g.G, g.T) || !encode_bf16_rows(&tmK, rk.p, n_rows, g.Hkv, D, rk.ts, rk.hs, 64, 1, 64) ||
        !encode_bf16_rows(&tmV, rv.p, n_rows, g.Hkv, D, rv.ts, rv.hs, D / 2, 1, 128))
        return fail(h, ADASPARK_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
    // a pair of CTAs per tile, at most as many as there are SMs: 2 T tokens a tile, at most one tile of each sequence not full
    const long long most = ((long long)n_q / (2 * g.T) + batch) * g.Hkv;
    const int pairs = (int)(most < h->sm_count / 2 ? most : h->sm_count / 2);
    auto launch = [&](auto kernel, size_t bytes) -> adaspark_status_t {
        if (!set_smem(h, kernel, bytes, "attn_prompt_kernel")) return ADASPARK_ERR_CUDA;
        launch_kernel(true, kernel, dim3(2 * pairs), dim3(kPromptThreads), bytes, (cudaStream_t)cuda_stream, g, tmQ, tmK, tmV, (__nv_bfloat16*)out, lse, status);
        return launch_ok(h, "attn_prompt_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
    };
    return D == 128 ? launch(attn_prompt_kernel<128>, sizeof(PromptSmem<128>) + 1024) : launch(attn_prompt_kernel<64>, sizeof(PromptSmem<64>) + 1024);
}

adaspark_status_t adaspark_attn_paged_write(adaspark_attn_t* h, const adaspark_attn_pages_t* pages, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                                            const void* v, int64_t v_token_stride, int64_t v_head_stride, const int32_t* cu, int32_t batch, int32_t n,
                                            const int32_t* block_table, int32_t table_width, const int32_t* kv_len, int32_t* status, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_write";
    if (batch < 0 || n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: negative size", who);
    h->launches = 0;
    if (batch == 0 || n == 0) return ADASPARK_OK;
    PageGeom g;
    Rows rk, rv;
    ADASPARK_TRY(check_pages(h, who, pages, block_table, table_width, g));
    ADASPARK_TRY(check_rows(h, who, "k", k, k_token_stride, k_head_stride, h->cfg.n_kv_heads, rk));
    ADASPARK_TRY(check_rows(h, who, "v", v, v_token_stride, v_head_stride, h->cfg.n_kv_heads, rv));
    if (!cu || !kv_len) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL cu or kv_len", who);
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    FastDiv rows, heads;
    rows.init(2 * g.Hkv);
    heads.init(g.Hkv);
    auto launch = [&](auto kernel) {
        launch_kernel(true, kernel, dim3((unsigned)((n + kCacheTokens - 1) / kCacheTokens)), dim3(kCacheThreads), 0, (cudaStream_t)cuda_stream, g, rk.p, rk.ts, rk.hs, rv.p, rv.ts, rv.hs,
                      cu, kv_len, batch, n, rows, heads, status);
    };
    const bool e4m3 = pages->format == ADASPARK_PAGES_E4M3;
    if (h->cfg.head_dim == 128) e4m3 ? launch(paged_write_kernel<128, true>) : launch(paged_write_kernel<128, false>);
    else e4m3 ? launch(paged_write_kernel<64, true>) : launch(paged_write_kernel<64, false>);
    return launch_ok(h, "paged_write_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
}

adaspark_status_t adaspark_attn_paged_read(adaspark_attn_t* h, const adaspark_attn_pages_t* pages, const int32_t* cu, int32_t batch, int32_t n,
                                           const int32_t* block_table, int32_t table_width, const int32_t* kv_len, void* k_out, void* v_out, int32_t* status,
                                           void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_read";
    if (batch < 0 || n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: negative size", who);
    h->launches = 0;
    if (batch == 0 || n == 0) return ADASPARK_OK;
    PageGeom g;
    ADASPARK_TRY(check_pages(h, who, pages, block_table, table_width, g));
    if (!cu || !kv_len || !k_out || !v_out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pointer", who);
    if ((uintptr_t)k_out % 16 || (uintptr_t)v_out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: outputs are not 16-byte aligned", who);
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    FastDiv rows, heads;
    rows.init(2 * g.Hkv);
    heads.init(g.Hkv);
    auto launch = [&](auto kernel) {
        launch_kernel(true, kernel, dim3((unsigned)((n + kCacheTokens - 1) / kCacheTokens)), dim3(kCacheThreads), 0, (cudaStream_t)cuda_stream, g, cu, kv_len, batch, n, rows, heads,
                      (__nv_bfloat16*)k_out, (__nv_bfloat16*)v_out, status);
    };
    const bool e4m3 = pages->format == ADASPARK_PAGES_E4M3;
    if (h->cfg.head_dim == 128) e4m3 ? launch(paged_read_kernel<128, true>) : launch(paged_read_kernel<128, false>);
    else e4m3 ? launch(paged_read_kernel<64, true>) : launch(paged_read_kernel<64, false>);
    return launch_ok(h, "paged_read_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
}

adaspark_status_t adaspark_attn_paged_decode(adaspark_attn_t* h, const void* q, int64_t q_token_stride, int64_t q_head_stride, const void* k_new,
                                             int64_t k_token_stride, int64_t k_head_stride, const void* v_new, int64_t v_token_stride, int64_t v_head_stride,
                                             const adaspark_attn_pages_t* pages, const int32_t* block_table, int32_t table_width, const int32_t* kv_len,
                                             int32_t batch, void* out, float* lse, void* workspace, size_t workspace_bytes, int32_t* status, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_decode";
    if (batch < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: negative batch", who);
    h->launches = 0;
    if (batch == 0) return ADASPARK_OK;
    PageGeom g;
    Rows rq, rk = {nullptr, 0, 0}, rv = {nullptr, 0, 0};
    if ((k_new == nullptr) != (v_new == nullptr)) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: k_new and v_new must both be given or both be NULL", who);
    ADASPARK_TRY(check_pages(h, who, pages, block_table, table_width, g));
    ADASPARK_TRY(check_rows(h, who, "q", q, q_token_stride, q_head_stride, h->cfg.n_q_heads, rq));
    if (k_new) {
        ADASPARK_TRY(check_rows(h, who, "k_new", k_new, k_token_stride, k_head_stride, h->cfg.n_kv_heads, rk));
        ADASPARK_TRY(check_rows(h, who, "v_new", v_new, v_token_stride, v_head_stride, h->cfg.n_kv_heads, rv));
    }
    if (!kv_len || !out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL kv_len or out", who);
    if ((uintptr_t)out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: out is not 16-byte aligned", who);
    if (!workspace || (uintptr_t)workspace % kAlign) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", who);
    if (workspace_bytes < (size_t)adaspark_attn_text_workspace_bytes(h)) return fail(h, ADASPARK_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %zu bytes", who, workspace_bytes);
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    const int D = h->cfg.head_dim, Hq = h->cfg.n_q_heads;
    const bool e4m3 = pages->format == ADASPARK_PAGES_E4M3;
    const int tile = paged_tile(e4m3), page_size = pages->page_size;
    PagedCall a;
    a.kv_len = kv_len;
    a.batch = batch;
    a.Hq = Hq;
    a.G = Hq / g.Hkv;
    a.q = rq.p; a.q_ts = rq.ts; a.q_hs = rq.hs;
    a.k_new = rk.p; a.k_ts = rk.ts; a.k_hs = rk.hs;
    a.v_new = rv.p; a.v_ts = rv.ts; a.v_hs = rv.hs;
    a.scale_log2 = text_scale(h) * 1.4426950408889634f;
    a.out = (__nv_bfloat16*)out;
    a.lse = lse;
    a.partial = (float*)workspace;
    a.status = status;
    CUtensorMap tmK, tmV;
    if (!encode_pages(&tmK, g.k, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile) ||
        !encode_pages(&tmV, g.v, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile))
        return fail(h, ADASPARK_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
    // two CTAs per SM, or as many as the tables have tiles
    const long long most = (long long)batch * g.Hkv * (((long long)table_width * page_size + tile - 1) / tile);
    const int n_ctas = (int)(most < kPagedCtas ? most : kPagedCtas);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    auto launch = [&](auto kernel, auto join, size_t bytes) -> adaspark_status_t {
        if (!set_smem(h, kernel, bytes, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        launch_kernel(true, kernel, dim3(n_ctas), dim3(kPagedThreads), bytes, st, g, a, tmK, tmV);
        if (!launch_ok(h, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        launch_kernel(true, join, dim3(Hq, batch), dim3(512), 0, st, g, a, n_ctas);
        return launch_ok(h, "paged_join_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
    };
    if (D == 128)
        return e4m3 ? launch(paged_decode_kernel<128, true>, paged_join_kernel<128, true>, sizeof(PagedSmem<128, true>))
                    : launch(paged_decode_kernel<128, false>, paged_join_kernel<128, false>, sizeof(PagedSmem<128, false>));
    return e4m3 ? launch(paged_decode_kernel<64, true>, paged_join_kernel<64, true>, sizeof(PagedSmem<64, true>))
                : launch(paged_decode_kernel<64, false>, paged_join_kernel<64, false>, sizeof(PagedSmem<64, false>));
}

}  // extern "C"
