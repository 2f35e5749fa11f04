// Entry points of the text operators (include/adaspark_attn.h, "Text beside the video"): argument checks and launches.
// Included by adaspark_attn.cu, whose handle and launch helpers they use.
#pragma once
#include <atomic>
#include <type_traits>

#include "attn_prompt.cuh"
#include "paged_cache.cuh"
#include "paged_decode.cuh"
#include "rotary.cuh"

namespace {

constexpr int kCacheManyTokens = 16384;
constexpr int kRotateFew = 300, kRotateMany = 2400, kRotateMost = 32768, kRotateFew64 = 600, kRotateMany64 = 3500;   // tokens

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

// What prompts of packed keys and of pages share.
void prompt_geom(const adaspark_attn* h, const int32_t* cu_q, int batch, int n_q, const Rows& rq, PromptGeom& g) {
    g.cu_q = cu_q;
    g.batch = batch;
    g.n_q = n_q;
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
}
// 2 T tokens a tile, at most one tile of each sequence not full
long long prompt_most_tiles(const PromptGeom& g) { return ((long long)g.n_q / (2 * g.T) + g.batch) * g.Hkv; }

struct PromptOut {
    __nv_bfloat16* out;
    float *lse, *partial;                          // partial null: nothing is cut
    int32_t* status;
};
template <int D, int kKeys>
adaspark_status_t launch_prompt(adaspark_attn* h, const PromptGeom& g, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV, const PromptOut& o,
                                void* cuda_stream) {
    // a pair of CTAs per tile, at most as many as there are SMs
    const long long most = prompt_most_tiles(g);
    int pairs = h->sm_count / 2 < kPromptPairs ? h->sm_count / 2 : kPromptPairs;
    if (!o.partial && most < pairs) pairs = (int)most;
    constexpr auto kernel = attn_prompt_kernel<D, kKeys>;
    const size_t bytes = sizeof(PromptSmem<D, kKeys>) + 1024;
    if (!text_smem<kernel>(h, bytes, "attn_prompt_kernel")) return ADASPARK_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    launch_kernel(true, kernel, dim3(2 * pairs), dim3(prompt_threads(kKeys)), bytes, st, g, tmQ, tmK, tmV, o.out, o.lse, o.partial, o.status);
    if (!launch_ok(h, "attn_prompt_kernel")) return ADASPARK_ERR_CUDA;
    if (!o.partial) return ADASPARK_OK;
    if (kKeys != kKeysPacked && pairs == 1) return ADASPARK_OK;       // one run: nothing is cut
    launch_kernel(true, prompt_join_kernel<D, kKeys != kKeysPacked>, dim3(kKeys == kKeysPacked ? kPromptParts : pairs - 1, 256 / kPromptJoinRows),
                  dim3(kPromptJoinThreads), 0, st, g, pairs, (const float*)o.partial, o.out, o.lse);
    return launch_ok(h, "prompt_join_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
}

// window 0: none
adaspark_status_t paged_decode_impl(adaspark_attn* h, const char* who, const adaspark_attn_paged_decode_t* c, int window, int sinks, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
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
    a.window = window;
    a.sinks = sinks;
    CUtensorMap tmK, tmV;
    if (!encode_pages(&tmK, g.k, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile) ||
        !encode_pages(&tmV, g.v, e4m3, g.n_pages, g.Hkv, page_size, D, g.page_stride, page_size < tile ? page_size : tile))
        return fail(h, ADASPARK_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
    // two CTAs per SM, or as many as the tables have tiles (a window: those that it and the first tokens may lie in)
    long long row_tiles = ((long long)table_width * page_size + tile - 1) / tile;
    if (window > 0) row_tiles = std::min(row_tiles, (long long)window / tile + (long long)sinks / tile + 4);
    const long long most = (long long)batch * g.Hkv * row_tiles;
    const int n_ctas = (int)(most < kPagedCtas ? most : kPagedCtas);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    auto launch = [&](auto d, auto bytes_held, auto groups, auto windowed) -> adaspark_status_t {
        constexpr int kD = d.value;
        constexpr bool kE4m3 = bytes_held.value, kWin = windowed.value;
        constexpr auto kernel = paged_decode_kernel<kD, kE4m3, groups.value, kWin>;
        constexpr size_t bytes = sizeof(PagedSmem<kD, kE4m3>);
        if (!text_smem<kernel>(h, bytes, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        launch_kernel(true, kernel, dim3(n_ctas), dim3(kPagedThreads), bytes, st, g, a, tmK, tmV);
        if (!launch_ok(h, "paged_decode_kernel")) return ADASPARK_ERR_CUDA;
        if (n_ctas == 1) return ADASPARK_OK;                   // nothing is cut
        if ((long long)batch * g.Hkv <= kPagedFewSequences)
            launch_kernel(true, paged_join_kernel<kD, kE4m3, true, kWin>, dim3(batch * g.Hkv, a.G), dim3(kJoinThreads), 0, st, g, a, n_ctas);
        else
            launch_kernel(true, paged_join_kernel<kD, kE4m3, false, kWin>, dim3(n_ctas - 1), dim3(kJoinThreads), 0, st, g, a, n_ctas);
        return launch_ok(h, "paged_join_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
    };
    auto with_window = [&](auto d, auto bytes_held, auto groups) -> adaspark_status_t {
        return window > 0 ? launch(d, bytes_held, groups, std::true_type()) : launch(d, bytes_held, groups, std::false_type());
    };
    auto with_groups = [&](auto d, auto bytes_held) -> adaspark_status_t {
        return a.G > 8 ? with_window(d, bytes_held, std::integral_constant<int, 2>()) : with_window(d, bytes_held, std::integral_constant<int, 1>());
    };
    const std::integral_constant<int, 128> wide;
    const std::integral_constant<int, 64> narrow;
    if (D == 128) return e4m3 ? with_groups(wide, std::true_type()) : with_groups(wide, std::false_type());
    return e4m3 ? with_groups(narrow, std::true_type()) : with_groups(narrow, std::false_type());
}

// What rotate and paged_append share: q (and its out), k, the rotation and the norms.  Rows whose data is NULL are none.
adaspark_status_t check_turned(adaspark_attn* h, const char* who, int n, const adaspark_attn_rows_t& q, const adaspark_attn_rows_t& q_out, const adaspark_attn_rows_t& k,
                               const adaspark_attn_rotary_t* rotary, const void* q_norm, const void* k_norm, float eps, RotateCall& a) {
    const int D = h->cfg.head_dim;
    Rows r;
    if (q.data) {
        ADASPARK_TRY(check_rows(h, who, "q", q, h->cfg.n_q_heads, r));
        a.q = {r.p, r.ts, r.hs};
        ADASPARK_TRY(check_rows(h, who, "q_out", q_out, h->cfg.n_q_heads, r));
        a.q_out = {r.p, r.ts, r.hs};
        a.Hq = h->cfg.n_q_heads;
    }
    if (k.data) {
        ADASPARK_TRY(check_rows(h, who, "k", k, h->cfg.n_kv_heads, r));
        a.k = {r.p, r.ts, r.hs};
        a.Hkv = h->cfg.n_kv_heads;
    }
    if ((uintptr_t)q_norm % 16 || (uintptr_t)k_norm % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: weights of the norms are not 16-byte aligned", who);
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: eps %g", who, eps);
    if (rotary) {
        if (rotary->pairs < 0 || rotary->pairs % 8 || rotary->pairs > D / 2 || rotary->axes < 1)
            return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: %d pairs of a head of %d, %d axes", who, rotary->pairs, D, rotary->axes);
        for (int i = 0; i < rotary->pairs; ++i)
            if (rotary->axis[i] >= rotary->axes) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: pair %d follows axis %d of %d", who, i, rotary->axis[i], rotary->axes);
        a.pairs = rotary->pairs;
        a.adjacent = rotary->adjacent;
        std::memcpy(a.turns, rotary->turns, sizeof(a.turns));
        std::memcpy(a.axis, rotary->axis, sizeof(a.axis));
    }
    a.q_norm = (const __nv_bfloat16*)q_norm;
    a.k_norm = (const __nv_bfloat16*)k_norm;
    a.eps = eps;
    a.n = n;
    return ADASPARK_OK;
}

template <int kPages>
adaspark_status_t launch_rotate(adaspark_attn* h, const RotateCall& a, const PageGeom& p, void* cuda_stream) {
    auto launch = [&](auto kernel, int tokens) {
        launch_kernel(true, kernel, dim3((unsigned)((a.n + tokens - 1) / tokens)), dim3(kRotateThreads), 0, (cudaStream_t)cuda_stream, a, p);
    };
    // As many tokens a CTA as leave every SM a few: what is worked out once for a token or a group is shared by more rows, against CTAs that an SM
    // ends up without.  Measured, us at 1 / 2 / 4 / 8 tokens a CTA, 28 + 4 heads of 128 with norms: 300 tokens 5.3 / 5.5 / 6.6 / 10.3, 1200 9.9 / 9.2 / 9.9 / 11.6,
    // 2400 17.1 / 13.8 / 13.5 / 15.7, 16512 85 / 62 / 49.6 / 55.5; into bf16 pages 65536 384 / 255 / 184 / 193; into 8-bit ones 33000 232 / 156 / 122 / 122,
    // 65536 452 / 302 / 231 / 222.  16 + 4 heads of 64 into bf16 pages and read back, at 2 / 4 / 8 / 16: 400 5.2 / 5.0 / 6.3 / 9.1, 701 6.0 / 5.6 / 6.4 / 9.1,
    // 2400 10.0 / 8.8 / 8.7 / 10.2 (8-bit pages 14.0 / 13.3 / 14.8 / 18.6), 9000 27.8 / 19.4 / 17.6 / 22.1, 33000 85 / 53 / 42 / 43; at 4682 calls one behind the
    // other take 17.9 us with 4 (1.3 waves of CTAs) and 16.5 with 8.  The rule goes by tokens alone; other numbers of heads, with norms, us on the device: 8 + 2 of 128
    // 300 tokens 4.5 / 4.2 / 4.7 / 6.3, 2400 12.9 / 9.4 / 9.1 / 9.6, 33000 140 / 78 / 61 / 53 (bf16 pages 157 / 84 / 62 / 54, 8-bit ones 178 / 107 / 72 / 59); 32 + 8 of 128
    // 300 5.2 / 5.3 / 7.1 / 11.5, 2400 15.4 / 12.9 / 15.3 / 18.4, 33000 168 / 120 / 107 / 114; 8 + 1 of 64, at 2 / 4 / 8, 600 4.5 / 4.0 / 4.7, 3500 9.3 / 6.4 / 7.0, 9000
    // 20.8 / 13.4 / 12.4: up to 14 % lie between the rule's choice and the best one with few heads and many tokens, 18 % with 32 + 8 at 2400
    if (h->cfg.head_dim == 128) {
        if (kPages == 2 && a.n >= kRotateMost) launch(rotate_kernel<128, 2, 8>, 8);
        else a.n >= kRotateMany ? launch(rotate_kernel<128, kPages, 4>, 4) : a.n >= kRotateFew ? launch(rotate_kernel<128, kPages, 2>, 2) : launch(rotate_kernel<128, kPages, 1>, 1);
    } else {
        a.n >= kRotateMany64 ? launch(rotate_kernel<64, kPages, 8>, 8) : a.n >= kRotateFew64 ? launch(rotate_kernel<64, kPages, 4>, 4) : launch(rotate_kernel<64, kPages, 2>, 2);
    }
    return launch_ok(h, "rotate_kernel") ? ADASPARK_OK : ADASPARK_ERR_CUDA;
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
    prompt_geom(h, c->cu_q, batch, n_q, rq, g);
    g.cu_k = c->cu_k;
    g.n_k = n_k;
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
    const bool cut = prompt_may_cut(prompt_most_tiles(g), n_k, c->cu_q == c->cu_k || n_q == n_k, 2 * g.T, g.Hkv);
    const PromptOut o = {(__nv_bfloat16*)c->out, c->lse, cut ? (float*)c->workspace : nullptr, c->status};
    return D == 128 ? launch_prompt<128, kKeysPacked>(h, g, tmQ, tmK, tmV, o, cuda_stream) : launch_prompt<64, kKeysPacked>(h, g, tmQ, tmK, tmV, o, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_write(adaspark_attn_t* h, const adaspark_attn_paged_rows_t* c, void* cuda_stream) {
    return paged_rows_impl(h, "paged_write", c, true, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_read(adaspark_attn_t* h, const adaspark_attn_paged_rows_t* c, void* cuda_stream) {
    return paged_rows_impl(h, "paged_read", c, false, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_decode(adaspark_attn_t* h, const adaspark_attn_paged_decode_t* c, void* cuda_stream) {
    return paged_decode_impl(h, "paged_decode", c, 0, 0, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_decode_window(adaspark_attn_t* h, const adaspark_attn_paged_decode_window_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_decode_window";
    if (!c || c->window < 1 || c->sinks < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call, window below 1 or sinks below 0", who);
    return paged_decode_impl(h, who, &c->step, c->window, c->sinks, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_prompt(adaspark_attn_t* h, const adaspark_attn_paged_prompt_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_prompt";
    if (!c || c->batch < 0 || c->n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative size", who);
    if (c->window < 0 || c->sinks < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: window %d, sinks %d", who, c->window, c->sinks);
    h->launches = 0;
    if (c->batch == 0 || c->n == 0) return ADASPARK_OK;
    PromptGeom g;
    PageGeom& p = g.pages;
    Rows rq;
    ADASPARK_TRY(check_pages(h, who, &c->pages, c->block_table, c->table_width, p));
    ADASPARK_TRY(check_rows(h, who, "q", c->q, h->cfg.n_q_heads, rq));
    if (!c->cu || !c->kv_len || !c->out) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL pointer", who);
    if ((uintptr_t)c->out % 16) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: out is not 16-byte aligned", who);
    if (c->window && ((long long)c->table_width << p.page_shift) > 0x7fffff00ll)      // (a window's steps begin anywhere: the last one ends up to 127 tokens further)
        return fail(h, ADASPARK_ERR_UNSUPPORTED, "%s: %d pages a sequence hold more than 2^31 - 256 tokens", who, c->table_width);
    ADASPARK_TRY(check_workspace(h, who, c->workspace, c->workspace_bytes));
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    prompt_geom(h, c->cu, c->batch, c->n, rq, g);
    g.kv_len = c->kv_len;
    g.window = c->window;
    g.sinks = c->window ? c->sinks : 0;
    // first ones and window, each rounded outwards by a step at most, and the 2 T tokens of a tile
    const long long most = c->window ? (long long)c->sinks / 128 + ((long long)c->window + 2 * g.T) / 128 + 3 : kPromptMostSteps;
    g.most_steps = (int)std::min(most, (long long)kPromptMostSteps);
    const int D = h->cfg.head_dim, page = c->pages.page_size, k_box = page < 64 ? page : 64, v_box = page < 128 ? page : 128;
    const bool e4m3 = c->pages.format == ADASPARK_PAGES_E4M3;
    CUtensorMap tmQ, tmK, tmV;
    if (!encode_bf16_rows(&tmQ, rq.p, c->n, g.Hq, D, rq.ts, rq.hs, 64, g.G, g.T) ||
        !encode_page_boxes(&tmK, p.k, e4m3, p.n_pages, g.Hkv, page, D, p.page_stride, e4m3 ? D : 64, k_box, e4m3 && D == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode_page_boxes(&tmV, p.v, e4m3, p.n_pages, g.Hkv, page, D, p.page_stride, D / 2, v_box,
                           e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B))
        return fail(h, ADASPARK_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed", who);
    const long long longest = std::min((long long)c->table_width << p.page_shift, 128ll * g.most_steps);
    const bool cut = prompt_may_cut(prompt_most_tiles(g), (int)std::min(longest, 0x7fffffffll), false, 2 * g.T, g.Hkv);
    const PromptOut o = {(__nv_bfloat16*)c->out, c->lse, cut ? (float*)c->workspace : nullptr, c->status};
    if (D == 128) return e4m3 ? launch_prompt<128, kKeysPages8>(h, g, tmQ, tmK, tmV, o, cuda_stream) : launch_prompt<128, kKeysPages>(h, g, tmQ, tmK, tmV, o, cuda_stream);
    return e4m3 ? launch_prompt<64, kKeysPages8>(h, g, tmQ, tmK, tmV, o, cuda_stream) : launch_prompt<64, kKeysPages>(h, g, tmQ, tmK, tmV, o, cuda_stream);
}

adaspark_status_t adaspark_attn_rotary_init(adaspark_attn_rotary_t* r, const double* radians, const int32_t* axis, int32_t pairs, int32_t axes, int32_t adjacent) {
    if (!r || pairs < 0 || pairs > kRotaryPairs || pairs % 8 || axes < 1 || axes > 255 || (pairs && !radians)) return ADASPARK_ERR_INVALID_ARG;
    adaspark_attn_rotary_t got;
    std::memset(&got, 0, sizeof(got));
    for (int i = 0; i < pairs; ++i) {
        if (!std::isfinite(radians[i]) || (axis && (axis[i] < 0 || axis[i] >= axes))) return ADASPARK_ERR_INVALID_ARG;
        const long double turns = (long double)radians[i] / 6.283185307179586476925286766559L, part = turns - std::floor(turns);
        got.turns[i] = part < 1.L ? (uint64_t)(part * 18446744073709551616.L) : 0;
        got.axis[i] = axis ? (uint8_t)axis[i] : 0;
    }
    got.pairs = pairs;
    got.axes = axes;
    got.adjacent = adjacent != 0;
    *r = got;
    return ADASPARK_OK;
}

adaspark_status_t adaspark_attn_rotate(adaspark_attn_t* h, const adaspark_attn_rotate_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "rotate";
    if (!c || c->n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative size", who);
    h->launches = 0;
    if (c->n == 0 || (!c->q.data && !c->k.data)) return ADASPARK_OK;
    RotateCall a;
    std::memset(&a, 0, sizeof(a));
    ADASPARK_TRY(check_turned(h, who, c->n, c->q, c->q_out, c->k, c->rotary, c->q_norm, c->k_norm, c->eps, a));
    if (c->k.data) {
        Rows out;
        ADASPARK_TRY(check_rows(h, who, "k_out", c->k_out, a.Hkv, out));
        a.k_out = {out.p, out.ts, out.hs};
    }
    if (a.pairs && !c->positions) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL positions", who);
    a.positions = c->positions;
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    PageGeom none;
    std::memset(&none, 0, sizeof(none));
    return launch_rotate<0>(h, a, none, cuda_stream);
}

adaspark_status_t adaspark_attn_paged_append(adaspark_attn_t* h, const adaspark_attn_paged_append_t* c, void* cuda_stream) {
    if (!h) return ADASPARK_ERR_INVALID_ARG;
    const char* who = "paged_append";
    if (!c || c->batch < 0 || c->n < 0) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL call or negative size", who);
    h->launches = 0;
    if (c->batch == 0 || c->n == 0) return ADASPARK_OK;
    PageGeom p;
    Rows rv;
    RotateCall a;
    std::memset(&a, 0, sizeof(a));
    ADASPARK_TRY(check_pages(h, who, &c->pages, c->block_table, c->table_width, p));
    if (!c->k.data) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL k", who);
    ADASPARK_TRY(check_turned(h, who, c->n, c->q, c->q_out, c->k, c->rotary, c->q_norm, c->k_norm, c->eps, a));
    ADASPARK_TRY(check_rows(h, who, "v", c->v, a.Hkv, rv));
    if (!c->cu || !c->kv_len) return fail(h, ADASPARK_ERR_INVALID_ARG, "%s: NULL cu or kv_len", who);
    a.v = {rv.p, rv.ts, rv.hs};
    a.positions = c->positions;
    a.cu = c->cu;
    a.kv_len = c->kv_len;
    a.batch = c->batch;
    a.status = c->status;
    DeviceScope scope;
    ADASPARK_TRY(scope.enter(h, who));
    return c->pages.format == ADASPARK_PAGES_E4M3 ? launch_rotate<2>(h, a, p, cuda_stream) : launch_rotate<1>(h, a, p, cuda_stream);
}

}  // extern "C"
