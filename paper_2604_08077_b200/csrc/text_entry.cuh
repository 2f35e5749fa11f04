// Entry points of the text operators (include/adaspark_attn.h, "Text beside the video"): argument checks and launches.
// Included by adaspark_attn.cu, whose handle and launch helpers they use.
#pragma once
#include <atomic>
#include <type_traits>

#include "attn_prompt.cuh"
#include "paged_cache.cuh"
#include "paged_decode.cuh"

namespace {

constexpr int kCacheManyTokens = 16384;

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
    __nv_bfloat16* p;
    long long ts, hs;
};
adaspark_status_t check_rows(adaspark_attn* h, const char* who, const char* what, const adaspark_attn_rows_t& rows, int heads, Rows& r) {
    const int D = h->cfg.head_dim;
    const void* p = rows.data;
    r.p = (__nv_bfloat16*)p;
    r.hs = rows.head_stride ? rows.head_stride : D;
    r.ts = rows.token_stride ? rows.token_stride : (long long)heads * D;
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

adaspark_status_t check_workspace(adaspark_attn* h, const char* who, const void* ws, int64_t bytes) {
    if (!ws || (uintptr_t)ws % kAlign) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: workspace NULL or not 256-byte aligned", who);
    const int64_t need = adaspark_attn_text_workspace_bytes(h);
    return bytes >= need ? ADASPARK_OK : fail(h, ADASPARK_ERR_WORKSPACE_TOO_SMALL, "%s: workspace %lld < %lld bytes", who, (long long)bytes, (long long)need);
}

// Room for a kernel's dynamic shared memory, asked for once per kernel and device.
template <auto kKernel>
bool text_smem(adaspark_attn* h, size_t bytes, const char* what) {
    static std::atomic<uint64_t> done{0};
    const uint64_t bit = 1ull << (h->cfg.device & 63);
    if (h->cfg.device < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
    if (!set_smem(h, kKernel, bytes, what)) return false;
    done.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

#define ADASPARK_TRY(expr)                       \
    do {                                         \
        const adaspark_status_t st_ = (expr);    \
        if (st_ != ADASPARK_OK) return st_;      \
    } while (0)

adaspark_status_t paged_rows_impl(adaspark_attn* h, const char* who, const adaspark_attn_paged_rows_t* c, bool write, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    if (!c || c->batch < 0 || c->n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative size", who);
    h->launches = 0;
    if (c->batch == 0 || c->n == 0) return ADASPARK_OK;
    PageGeom g;
    Rows rk, rv;
    ADASPARK_TRY(check_pages(h, who, &c->pages, c->block_table, c->table_width, g));
    ADASPARK_TRY(check_rows(h, who, "k", c->k, h->cfg.n_kv_heads, rk));
    ADASPARK_TRY(check_rows(h, who, "v", c->v, h->cfg.n_kv_heads, rv));
    if (!c->cu || !c->kv_len) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL cu or kv_len", who);
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    const bool e4m3 = c->pages.format == ADASPARK_PAGES_E4M3;
    const int D = h->cfg.head_dim, columns = (2 * g.Hkv * (D / 8) + kCacheThreads - 1) / kCacheThreads;
    // 32 tokens a CTA where that leaves every SM several, 8 where there are few
    const bool many = c->n >= kCacheManyTokens;
    auto launch = [&](auto kernel) {
        const int tokens = many ? 32 : 8;
        launch_kernel(true, kernel, dim3((unsigned)((c->n + tokens - 1) / tokens), columns), dim3(kCacheThreads), 0, (cudaStream_t)cuda_stream, g, rk.p, rk.ts, rk.hs, rv.p,
                      rv.ts, rv.hs, c->cu, c->kv_len, c->batch, c->n, c->status);
    };
    auto with = [&](auto d, auto bytes_held) {
        constexpr int kD = d.value;
        constexpr bool kE4m3 = bytes_held.value;
        if (write) many ? launch(paged_write_kernel<kD, kE4m3, 32>) : launch(paged_write_kernel<kD, kE4m3, 8>);
        else many ? launch(paged_read_kernel<kD, kE4m3, 32>) : launch(paged_read_kernel<kD, kE4m3, 8>);
    };
    const std::integral_constant<int, 128> wide;
    const std::integral_constant<int, 64> narrow;
    if (D == 128) e4m3 ? with(wide, std::true_type()) : with(wide, std::false_type());
    else e4m3 ? with(narrow, std::true_type()) : with(narrow, std::false_type());
    return launch_ok(h, write ? "paged_write_kernel" : "paged_read_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
}

}  // namespace

extern "C" {

int64_t adaspark_attn_text_workspace_bytes(const adaspark_attn_t* h) {
    if (!h) return 0;
    const size_t decode = paged_partial_bytes(h->cfg.head_dim, h->cfg.n_q_heads / h->cfg.n_kv_heads), prompt = prompt_partial_bytes(h->cfg.head_dim);
    return (int64_t)align_up(decode > prompt ? decode : prompt);
}

adaspark_status_t adaspark_attn_prompt(adaspark_attn_t* h, const adaspark_attn_prompt_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "prompt";
    if (!c || c->batch < 0 || c->n_q < 0 || c->n_k < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative size", who);
    const int batch = c->batch, n_q = c->n_q, n_k = c->n_k;
    h->launches = 0;
    if (batch == 0 || n_q == 0) return ADASPARK_OK;
    Rows rq, rk, rv;
    ADASPARK_TRY(check_rows(h, who, "q", c->q, h->cfg.n_q_heads, rq));
    if (n_k) {
        ADASPARK_TRY(check_rows(h, who, "k", c->k, h->cfg.n_kv_heads, rk));
        ADASPARK_TRY(check_rows(h, who, "v", c->v, h->cfg.n_kv_heads, rv));
    } else {                                       // no keys at all: k and v may be NULL; the tensor maps need some row, which no row sees
        rk = rv = {rq.p, (long long)h->cfg.n_kv_heads * h->cfg.head_dim, h->cfg.head_dim};
    }
    if (!c->cu_q || !c->cu_k || !c->out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pointer", who);
    if ((uintptr_t)c->out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: out is not 16-byte aligned", who);
    ADASPARK_TRY(check_workspace(h, who, c->workspace, c->workspace_bytes));
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    PromptGeom g;
    g.cu_q = c->cu_q;
    g.cu_k = c->cu_k;
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
    g.q = rq.p;
    g.q_ts = rq.ts;
    g.q_hs = rq.hs;
    g.k = rk.p;
    g.k_ts = rk.ts;
    g.k_hs = rk.hs;
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
    int pairs = h->sm_count / 2 < kPromptPairs ? h->sm_count / 2 : kPromptPairs;
    const bool cut = prompt_may_cut(most, n_k, c->cu_q == c->cu_k || n_q == n_k, 2 * g.T, g.Hkv);
    float* partial = cut ? (float*)c->workspace : nullptr;
    if (!cut && most < pairs) pairs = (int)most;
    auto launch = [&](auto d) -> adaspark_status_t {
        constexpr auto kernel = attn_prompt_kernel<d.value>;
        const size_t bytes = sizeof(PromptSmem<d.value>) + 1024;
        if (!text_smem<kernel>(h, bytes, "attn_prompt_kernel")) return ADASPARK_ERR_CUDA;
        cudaStream_t st = (cudaStream_t)cuda_stream;
        launch_kernel(true, kernel, dim3(2 * pairs), dim3(kPromptThreads), bytes, st, g, tmQ, tmK, tmV, (__nv_bfloat16*)c->out, c->lse, partial, c->status);
        if (!launch_ok(h, "attn_prompt_kernel")) return ADASPARK_ERR_CUDA;
        if (!cut) return ADASPARK_OK;
        launch_kernel(true, prompt_join_kernel<d.value>, dim3(kPromptParts, 256 / kPromptJoinRows), dim3(kPromptJoinThreads), 0, st, g, pairs, (const float*)partial, (__nv_bfloat16*)c->out, c->lse);
        return launch_ok(h, "prompt_join_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
    };
    return D == 128 ? launch(std::integral_constant<int, 128>()) : launch(std::integral_constant<int, 64>());
}

adaspark_status_t adaspark_attn_paged_write(adaspark_attn_t* h, const adaspark_attn_paged_rows_t* c, void* cuda_stream) {
    return paged_rows_impl(h, "paged_write", c, true, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_read(adaspark_attn_t* h, const adaspark_attn_paged_rows_t* c, void* cuda_stream) {
    return paged_rows_impl(h, "paged_read", c, false, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_decode(adaspark_attn_t* h, const adaspark_attn_paged_decode_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_decode";
    if (!c || c->batch < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative batch", who);
    const int batch = c->batch, table_width = c->table_width;
    h->launches = 0;
    if (batch == 0) return ADASPARK_OK;
    const adaspark_attn_pages_t* pages = &c->pages;
    PageGeom g;
    Rows rq, rk = {nullptr, 0, 0}, rv = {nullptr, 0, 0};
    if ((c->k_new.data == nullptr) != (c->v_new.data == nullptr)) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: k_new and v_new must both be given or both be NULL", who);
    ADASPARK_TRY(check_pages(h, who, pages, c->block_table, table_width, g));
    ADASPARK_TRY(check_rows(h, who, "q", c->q, h->cfg.n_q_heads, rq));
    if (c->k_new.data) {
        ADASPARK_TRY(check_rows(h, who, "k_new", c->k_new, h->cfg.n_kv_heads, rk));
        ADASPARK_TRY(check_rows(h, who, "v_new", c->v_new, h->cfg.n_kv_heads, rv));
    }
    if (!c->kv_len || !c->out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL kv_len or out", who);
    if ((uintptr_t)c->out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: out is not 16-byte aligned", who);
    ADASPARK_TRY(check_workspace(h, who, c->workspace, c->workspace_bytes));
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    const int D = h->cfg.head_dim, Hq = h->cfg.n_q_heads;
    const bool e4m3 = pages->format == ADASPARK_PAGES_E4M3;
    const int tile = paged_tile(e4m3), page_size = pages->page_size;
    PagedCall a;
    a.kv_len = c->kv_len;
    a.batch = batch;
    a.Hq = Hq;
    a.G = Hq / g.Hkv;
    a.q = rq.p; a.q_ts = rq.ts; a.q_hs = rq.hs;
    a.k_new = rk.p; a.k_ts = rk.ts; a.k_hs = rk.hs;
    a.v_new = rv.p; a.v_ts = rv.ts; a.v_hs = rv.hs;
    a.scale_log2 = text_scale(h) * 1.4426950408889634f;
    a.out = (__nv_bfloat16*)c->out;
    a.lse = c->lse;
    a.partial = (float*)c->workspace;
    a.status = c->status;
    CUtensorMap tmK, tmV;
    if (!encode_pages(&tmK, g.k, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile) ||
        !encode_pages(&tmV, g.v, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile))
        return fail(h, ADASPARK_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
    // two CTAs per SM, or as many as the tables have tiles
    const long long most = (long long)batch * g.Hkv * (((long long)table_width * page_size + tile - 1) / tile);
    const int n_ctas = (int)(most < kPagedCtas ? most : kPagedCtas);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    auto launch = [&](auto d, auto bytes_held, auto groups) -> adaspark_status_t {
        constexpr int kD = d.value;
        constexpr bool kE4m3 = bytes_held.value;
        constexpr auto kernel = paged_decode_kernel<kD, kE4m3, groups.value>;
        constexpr size_t bytes = sizeof(PagedSmem<kD, kE4m3>);
        if (!text_smem<kernel>(h, bytes, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        launch_kernel(true, kernel, dim3(n_ctas), dim3(kPagedThreads), bytes, st, g, a, tmK, tmV);
        if (!launch_ok(h, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        if (n_ctas == 1) return ADASPARK_OK;                   // nothing is cut
        if ((long long)batch * g.Hkv <= kPagedFewSequences)
            launch_kernel(true, paged_join_kernel<kD, kE4m3, true>, dim3(batch * g.Hkv, a.G), dim3(kJoinThreads), 0, st, g, a, n_ctas);
        else
            launch_kernel(true, paged_join_kernel<kD, kE4m3, false>, dim3(n_ctas - 1), dim3(kJoinThreads), 0, st, g, a, n_ctas);
        return launch_ok(h, "paged_join_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
    };
    auto with_groups = [&](auto d, auto bytes_held) -> adaspark_status_t {
        return a.G > 8 ? launch(d, bytes_held, std::integral_constant<int, 2>()) : launch(d, bytes_held, std::integral_constant<int, 1>());
    };
    const std::integral_constant<int, 128> wide;
    const std::integral_constant<int, 64> narrow;
    if (D == 128) return e4m3 ? with_groups(wide, std::true_type()) : with_groups(wide, std::false_type());
    return e4m3 ? with_groups(narrow, std::true_type()) : with_groups(narrow, std::false_type());
}

}  // extern "C"
