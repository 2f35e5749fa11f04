// Attention of one new token per sequence over the pages of its cache, split over the cache's length and joined.
//
//   o = sum_j w_j v_j / sum_j w_j,  w_j = 2^(x_j - m),  x_j = scale_log2 q.k_j,  j < kv_len
//
// Bound by HBM: every page is read once for all heads of a group (at most 16, the rows of one mma.sync tile: the tensor work per byte
// is tiny, what matters is bytes under way).  The key tiles of all sequences and kv heads are one line, cut into equal
// runs, one per CTA: a batch of any lengths loads every SM alike, and one long sequence is spread over all of them.  Lengths are
// read on the device; a CTA finds its run by a prefix sum over the batch.  A (sequence, kv head) that lies in one run is
// finished there; of one that is cut, each part leaves (maxima, sum, unnormalised output) and paged_join_kernel puts them together, in
// the order of the runs: the result does not depend on who is faster.
//   warp 4      producer: page numbers (32 columns of the table at a time, the next 32 ahead), TMA tiles of K and V from
//               their pages and the bytes of the powers of two into a ring, the next (sequence, head)'s q; the new token into its page
//   warps 0-3   each a quarter of a tile's keys: S = Q K^T, softmax, O += P V, with a state of its own, merged at the end of a run's part
//
// 8-bit pages go through the tensor cores as f16, which holds every e4m3 value.  q is brought to f16 by a power of two per row (largest
// magnitude 2^14 ..: what falls below 2^-29 of it loses bits, 2^-39 of it at most); a key's power of two multiplies its score.  A
// value's power of two e_j joins its weight: the weights of the product are 2^(x_j + e_j - m') with their own maximum m', so that they stay within f16
// whatever the rows' sizes, and beside them the sum of 2^(x_j - m) is kept.
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"
#include "tc_common.cuh"

namespace adaspark {

constexpr int kPagedThreads = 160;
constexpr int kPagedCtas = 296;              // two per SM of a B200
constexpr int kPagedRing = 96 * 1024;        // bytes of a CTA's ring
constexpr float kPagedBias = 14.f;           // f16 weights are at most 2^14: 2^-28 of the largest one is still a normal number

__host__ __device__ constexpr int paged_tile(bool e4m3) { return e4m3 ? 128 : 64; }   // keys of a tile
__host__ __device__ constexpr int paged_row_floats(int D) { return D + 4; }           // m, l, m', -, o[D]
__host__ __device__ constexpr size_t paged_partial_bytes(int D, int G) { return (size_t)kPagedCtas * 2 * G * paged_row_floats(D) * sizeof(float); }

// The new token's row of one kv head (keys: which = 0, values: 1) into its place; by the 32 lanes of a warp.
template <int D, bool kE4m3>
__device__ __forceinline__ void append_row(const PageGeom& p, int page, int head, int place, int which, const __nv_bfloat16* src, int lane) {
    constexpr int kLanes = D / 8;
    const long long row = ((long long)head << p.page_shift) + place;
    const int part = lane % kLanes;
    const uint4 x = *reinterpret_cast<const uint4*>(src + part * 8);
    if (kE4m3) {
        bool odd;
        uint32_t top = chunk_top(x, odd);
#pragma unroll
        for (int s = 1; s < kLanes; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
        const uint32_t s = scale_byte(top);
        if (lane < kLanes) *reinterpret_cast<uint2*>((which ? p.v : p.k) + (long long)page * p.page_stride + row * D + part * 8) = chunk_codes(x, s, odd);
        if (lane == 0) (which ? p.vs : p.ks)[(long long)page * p.scale_stride + row] = (uint8_t)s;
    } else if (lane < kLanes) {
        *reinterpret_cast<uint4*>((which ? p.v : p.k) + ((long long)page * p.page_stride + row * D + part * 8) * 2) = x;
    }
}

// What one call works on.
struct PagedCall {
    const int32_t* kv_len;
    int batch, Hq, G;
    const __nv_bfloat16 *q, *k_new, *v_new;
    long long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs;
    float scale_log2;
    __nv_bfloat16* out;
    float* lse;
    float* partial;                          // [cta][2][G][paged_row_floats]
    int32_t* status;
};

// The line of tiles: sequence by sequence, kv head by kv head.  Held by a whole warp, which has the tile counts of 32 sequences in its lanes.
template <int kTile>
struct TileLine {
    const PageGeom* p;
    const int32_t* kv_len;
    int batch, lane;
    int chunk, tiles;                        // first sequence of the lanes' 32, tiles of this lane's sequence (0: none, or out of range)
    __device__ __forceinline__ int count(int n) const { return n > 0 && n <= (p->table_width << p->page_shift) ? (n + kTile - 1) / kTile : 0; }
    __device__ __forceinline__ void load(int c) {
        chunk = c;
        tiles = c + lane < batch ? count(kv_len[c + lane]) : 0;
    }
    __device__ __forceinline__ long long total() {
        long long sum = 0;
        for (int c = 0; c < batch; c += 32) {
            load(c);
            sum += (long long)__reduce_add_sync(0xffffffffu, (unsigned)(tiles & 0xffff)) + ((long long)__reduce_add_sync(0xffffffffu, (unsigned)(tiles >> 16)) << 16);
        }
        return sum * p->Hkv;
    }
};

// The line's total tiles are cut into runs of at least one tile: how many, the first tile of run c, and the run that holds tile x.
__device__ __forceinline__ int run_count(long long total, int n_ctas) { return (int)min(total, (long long)n_ctas); }
__device__ __forceinline__ long long run_begin(long long total, int n_runs, int c) { return total * c / n_runs; }
__device__ __forceinline__ int run_of(long long total, int n_runs, long long x) { return (int)(((x + 1) * n_runs - 1) / total); }

// A place on the line: tile `tile` of `tiles` of (sequence b, kv head gk).
template <int kTile>
struct LineWalk {
    TileLine<kTile> line;
    int b, gk, tile, tiles;
    // to position x < total
    __device__ __forceinline__ void seek(long long x) {
        for (int c = 0; c < line.batch; c += 32) {
            line.load(c);
            long long upto = (long long)line.tiles * line.p->Hkv;
            const long long mine = upto;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, upto, s);
                if (line.lane >= s) upto += y;
            }
            const long long all = __shfl_sync(0xffffffffu, upto, 31);
            if (x < all) {
                const int who = __ffs(__ballot_sync(0xffffffffu, upto > x)) - 1;
                const int rest = (int)(x - __shfl_sync(0xffffffffu, upto - mine, who));
                b = c + who;
                tiles = __shfl_sync(0xffffffffu, line.tiles, who);
                gk = rest / tiles;
                tile = rest - gk * tiles;
                return;
            }
            x -= all;
        }
    }
    // to the first tile of the next (sequence, kv head); there has to be one
    __device__ __forceinline__ void next() {
        tile = 0;
        if (++gk < line.p->Hkv) return;
        gk = 0;
        int from = b + 1 - line.chunk;
        while (true) {
            const uint32_t there = from < 32 ? __ballot_sync(0xffffffffu, line.tiles > 0) >> from << from : 0u;
            if (there) {
                const int who = __ffs(there) - 1;
                b = line.chunk + who;
                tiles = __shfl_sync(0xffffffffu, line.tiles, who);
                return;
            }
            if (line.chunk + 32 >= line.batch) return;
            line.load(line.chunk + 32);
            from = 0;
        }
    }
};

template <int D, bool kE4m3>
struct PagedSmem {
    static constexpr int kTile = paged_tile(kE4m3), kRowBytes = kE4m3 ? D : 2 * D;
    static constexpr int kTileBytes = kTile * kRowBytes;       // of K, and of V
    static constexpr int kStages = kPagedRing / (2 * kTileBytes);
    unsigned char kv[kStages][2][kTileBytes];                 // bf16: [panel of 64 d][key][128 bytes]; e4m3: [key][D bytes]; swizzled by TMA
    float red[16][D];
    __nv_bfloat16 q[16][D + 8];                               // of one part at a time (read into registers when it begins)
    unsigned char scale[kStages][2][kE4m3 ? kTile : 16];
    float stat[4][16][4];
    uint64_t full[kStages], empty[kStages], q_full, q_empty;
    int bad[2];                                               // number + 1 of a part with a page that is not there
    int abort_flag;
};

static_assert(sizeof(PagedSmem<128, true>) <= 115712 && sizeof(PagedSmem<128, false>) <= 115712, "two CTAs share an SM");

__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3, const void* smem_ptr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(smem_u32(smem_ptr)));
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {   // 16-byte aligned, a multiple of 16 bytes
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(smem_u32(smem_dst)), "l"(src), "r"(bytes),
                 "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;\n" ::: "memory"); }

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kPagedThreads, 2) paged_decode_kernel(PageGeom p, PagedCall a, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV) {
    using Smem = PagedSmem<D, kE4m3>;
    extern __shared__ __align__(1024) unsigned char paged_smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(paged_smem_raw);
    constexpr int kTile = Smem::kTile, kStages = Smem::kStages, kTileBytes = Smem::kTileBytes, kRowBytes = Smem::kRowBytes;
    constexpr int kWarpKeys = kTile / 4, kNTiles = kWarpKeys / 8, kKSteps = D / 16, kDTiles = D / 8, kRowF = paged_row_floats(D);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    launch_dependents();
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&sm.full[s], 1);
            tc::mbar_init(&sm.empty[s], 4);
        }
        tc::mbar_init(&sm.q_full, 1);
        tc::mbar_init(&sm.q_empty, 4);
        sm.bad[0] = sm.bad[1] = 0;
        sm.abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tensormap(&tmK);
        tc::prefetch_tensormap(&tmV);
    }
    __syncthreads();
    volatile int* abort_flag = &sm.abort_flag;
    wait_for_previous_kernel();

    LineWalk<kTile> w;
    w.line.p = &p;
    w.line.kv_len = a.kv_len;
    w.line.batch = a.batch;
    w.line.lane = lane;
    const long long total = w.line.total();
    const int n_runs = run_count(total, gridDim.x);
    if ((int)blockIdx.x >= n_runs) return;                    // (the whole CTA)
    const long long it0 = run_begin(total, n_runs, blockIdx.x), it1 = run_begin(total, n_runs, blockIdx.x + 1);
    w.seek(it0);
    const int page_shift = p.page_shift, page_size = 1 << page_shift;

    if (warp == 4) {
        // ------------------------------------------------------------ producer
        const int sub = min(page_size, kTile), n_sub = kTile / sub;        // tokens of a box, boxes of a tile
        int st = 0, ph = 1, part = 0;
        bool ok = true;
        for (long long it = it0; it < it1 && ok; ++part) {
            const int n_here = (int)min((long long)(w.tiles - w.tile), it1 - it), n = a.kv_len[w.b];
            const int32_t* table = p.table + (size_t)w.b * p.table_width;
            // page numbers: this lane's of the 32 columns from `cols` on, and of the 32 behind them
            const int last_col = (n - 1) >> page_shift;
            int cols = (w.tile * kTile) >> page_shift;
            auto page_at = [&](int col) -> int { return col <= last_col ? table[col] : 0; };
            int pages = page_at(cols + lane), pages_next = page_at(cols + 32 + lane);
            // q of the heads, a row each
            if (!(ok = tc::mbar_wait_warp(&sm.q_empty, (part & 1) ^ 1, abort_flag))) break;
            if (lane == 0) tc::mbar_arrive_expect_tx(&sm.q_full, (uint32_t)a.G * D * 2);
            __syncwarp();
            if (lane < a.G) bulk_load(&sm.q[lane][0], a.q + w.b * a.q_ts + (w.gk * a.G + lane) * a.q_hs, D * 2, &sm.q_full);
            for (int i = 0; i < n_here; ++i) {
                const int tile = w.tile + i, pos0 = tile * kTile, col0 = pos0 >> page_shift;
                while (col0 >= cols + 32) {
                    cols += 32;
                    pages = pages_next;
                    pages_next = page_at(cols + 32 + lane);
                }
                const int boxes = min((n - pos0 + sub - 1) / sub, n_sub);  // those that hold a token
                int page = __shfl_sync(0xffffffffu, pages, min(col0 - cols + lane, 31));
                const int over = __shfl_sync(0xffffffffu, pages_next, max(col0 - cols + lane - 32, 0) & 31);
                if (col0 - cols + lane >= 32) page = over;
                const bool there = page >= 0 && page < p.n_pages;
                if (__any_sync(0xffffffffu, lane < boxes && !there)) {
                    if (lane == 0) {
                        sm.bad[part & 1] = part + 1;
                        if (a.status != nullptr) atomicExch(a.status, 1);
                    }
                } else if (a.k_new != nullptr && tile == w.tiles - 1) {    // the new token: the last of this tile
                    const int pg = __shfl_sync(0xffffffffu, page, boxes - 1), place = (n - 1) & (page_size - 1);
                    append_row<D, kE4m3>(p, pg, w.gk, place, 0, a.k_new + w.b * a.k_ts + w.gk * a.k_hs, lane);
                    append_row<D, kE4m3>(p, pg, w.gk, place, 1, a.v_new + w.b * a.v_ts + w.gk * a.v_hs, lane);
                    asm volatile("fence.proxy.async;\n" ::: "memory");     // it is read by the copies below
                    __syncwarp();
                }
                if (!(ok = tc::mbar_wait_warp(&sm.empty[st], ph, abort_flag))) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&sm.full[st], (uint32_t)(boxes * sub * 2 * (kRowBytes + (kE4m3 ? 1 : 0))));
                __syncwarp();
                if (lane < boxes) {
                    const int slot = pos0 & (page_size - 1);               // (0 where a page is no larger than a tile)
                    const int at = there ? page : p.n_pages;               // a box outside the tensor reads zeros
                    if (kE4m3) {
                        tc::tma_load_4d(&sm.kv[st][0][lane * sub * kRowBytes], &tmK, 0, slot, w.gk, at, &sm.full[st]);
                        tc::tma_load_4d(&sm.kv[st][1][lane * sub * kRowBytes], &tmV, 0, slot, w.gk, at, &sm.full[st]);
                        const long long s_at = (long long)(there ? page : 0) * p.scale_stride + ((long long)w.gk << page_shift) + slot;
                        bulk_load(&sm.scale[st][0][lane * sub], p.ks + s_at, sub, &sm.full[st]);
                        bulk_load(&sm.scale[st][1][lane * sub], p.vs + s_at, sub, &sm.full[st]);
                    } else {
#pragma unroll
                        for (int x = 0; x < D / 64; ++x) {
                            tc::tma_load_4d(&sm.kv[st][0][x * kTile * 128 + lane * sub * 128], &tmK, x * 64, slot, w.gk, at, &sm.full[st]);
                            tc::tma_load_4d(&sm.kv[st][1][x * kTile * 128 + lane * sub * 128], &tmV, x * 64, slot, w.gk, at, &sm.full[st]);
                        }
                    }
                }
                __syncwarp();
                if (++st == kStages) { st = 0; ph ^= 1; }
            }
            it += n_here;
            if (it < it1) w.next();
        }
        return;
    }
    // ---------------------------------------------------------------- consumers (they keep to their barriers when a wait has expired)
    const int rA = lane >> 2, rB = rA + 8, t4 = lane & 3;
    int st = 0, ph = 0, part = 0;
    for (long long it = it0; it < it1; ++part) {
        const int n_here = (int)min((long long)(w.tiles - w.tile), it1 - it), n = a.kv_len[w.b];
        // ---- q fragments: rows = heads (zero beyond the group)
        uint32_t qf[kKSteps][4];
        float fA = a.scale_log2, fB = a.scale_log2;           // what a row's products are multiplied by
        tc::mbar_wait(&sm.q_full, part & 1, abort_flag);
        {
            const __nv_bfloat16 *qa = sm.q[rA], *qb = sm.q[rB];
            const bool hasA = rA < a.G, hasB = rB < a.G;
            if (!kE4m3) {
#pragma unroll
                for (int ks = 0; ks < kKSteps; ++ks) {
                    const int c = ks * 16 + 2 * t4;
                    qf[ks][0] = hasA ? *reinterpret_cast<const uint32_t*>(qa + c) : 0u;
                    qf[ks][1] = hasB ? *reinterpret_cast<const uint32_t*>(qb + c) : 0u;
                    qf[ks][2] = hasA ? *reinterpret_cast<const uint32_t*>(qa + c + 8) : 0u;
                    qf[ks][3] = hasB ? *reinterpret_cast<const uint32_t*>(qb + c + 8) : 0u;
                }
            } else {
                // Thread t of a quad has the 16-byte chunks t (D = 64) or 2 t, 2 t + 1 (D = 128) of a key's codes: step (chunk j, word i)
                // takes d = 16 * chunk + 4 i .. + 3 as the k indexes 2t, 2t + 1, 2t + 8, 2t + 9
                uint32_t top[2] = {0u, 0u};
#pragma unroll
                for (int ks = 0; ks < kKSteps; ++ks) {
                    const int d = 16 * (D == 128 ? 2 * t4 + (ks >> 2) : t4) + 4 * (ks & 3);
                    const uint2 x = hasA ? *reinterpret_cast<const uint2*>(qa + d) : make_uint2(0u, 0u);
                    const uint2 y = hasB ? *reinterpret_cast<const uint2*>(qb + d) : make_uint2(0u, 0u);
                    qf[ks][0] = x.x; qf[ks][2] = x.y; qf[ks][1] = y.x; qf[ks][3] = y.y;
                    top[0] = __vmaxu2(top[0], __vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu));
                    top[1] = __vmaxu2(top[1], __vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu));
                }
                float mul[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    uint32_t m = max(top[r] & 0xffffu, top[r] >> 16);
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                    const int e = max((int)(m >> 7), 30);                  // biased exponent of the largest; 2^14 is 141
                    mul[r] = __uint_as_float((uint32_t)(127 + 141 - e) << 23);       // e = 255 (no number): 2^-... and stays one
                    (r ? fB : fA) = a.scale_log2 * __uint_as_float((uint32_t)min(127 + e - 141, 254) << 23);
                }
#pragma unroll
                for (int ks = 0; ks < kKSteps; ++ks)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float f = mul[e & 1];
                        qf[ks][e] = pack_f16x2(__uint_as_float(qf[ks][e] << 16) * f, __uint_as_float(qf[ks][e] & 0xffff0000u) * f);
                    }
            }
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sm.q_empty);

        // running maxima and sums of rows A and B; with e4m3 pages mv is the maximum of the weights of the products
        float mA = -INFINITY, mB = -INFINITY, lA = 0.f, lB = 0.f, mvA = -INFINITY, mvB = -INFINITY;
        float o[kDTiles][4];
#pragma unroll
        for (int i = 0; i < kDTiles; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        for (int i = 0; i < n_here; ++i) {
            const int n_vis = n - (w.tile + i) * kTile - warp * kWarpKeys;      // keys of this warp's quarter that are there
            tc::mbar_wait(&sm.full[st], ph, abort_flag);
            if (n_vis > 0) {
                unsigned char* kst = sm.kv[st][0];
                unsigned char* vst = sm.kv[st][1];
                const int row0 = warp * kWarpKeys;
                if (n_vis < kWarpKeys) {                      // what lies behind the last token may be anything: 0 * it is not 0
                    constexpr int kChunks = kRowBytes / 16;
                    for (int c = lane; c < (kWarpKeys - n_vis) * kChunks; c += 32) {
                        const int r = row0 + n_vis + c / kChunks, x = c % kChunks;
                        unsigned char* dst = kE4m3 ? vst + r * kRowBytes + x * 16 : vst + (x >> 3) * (kTile * 128) + r * 128 + (x & 7) * 16;
                        *reinterpret_cast<uint4*>(dst) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");   // TMA writes there again
                    __syncwarp();
                }
                float sc[kNTiles][4];
#pragma unroll
                for (int nt = 0; nt < kNTiles; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
                if (!kE4m3) {
#pragma unroll
                    for (int ks = 0; ks < kKSteps; ++ks) {
                        const int row = row0 + (lane & 7) + ((lane >> 4) << 3), chunk = ks * 2 + ((lane >> 3) & 1);
                        uint32_t b0, b1, b2, b3;
                        ldmatrix_x4(b0, b1, b2, b3, kst + (chunk >> 3) * (kTile * 128) + sw128(row, chunk & 7));
                        mma_bf16_16816(sc[0], qf[ks], b0, b1);
                        mma_bf16_16816(sc[1], qf[ks], b2, b3);
                    }
                } else {
#pragma unroll
                    for (int nt = 0; nt < kNTiles; ++nt) {
                        const int row = row0 + nt * 8 + rA;
#pragma unroll
                        for (int j = 0; j < D / 64; ++j) {
                            const uint4 x = D == 128 ? *reinterpret_cast<const uint4*>(kst + row * 128 + (((2 * t4 + j) ^ (row & 7)) << 4))
                                                     : *reinterpret_cast<const uint4*>(kst + row * 64 + ((t4 ^ ((row >> 1) & 3)) << 4));
                            const uint32_t c[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) mma_f16_16816(sc[nt], qf[j * 4 + e], codes_to_f16x2(c[e] & 0xffffu), codes_to_f16x2(c[e] >> 16));
                        }
                    }
                }
                // ---- x_j, their maxima, and with e4m3 x_j + e_j and theirs
                float ve[kNTiles][2];                         // e_j of this thread's keys
                float mxA = -INFINITY, mxB = -INFINITY, mxvA = -INFINITY, mxvB = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < kNTiles; ++nt) {
                    float k0 = 1.f, k1 = 1.f;
                    if (kE4m3) {
                        const uint32_t ks2 = *reinterpret_cast<const uint16_t*>(&sm.scale[st][0][row0 + nt * 8 + 2 * t4]);
                        const uint32_t vs2 = *reinterpret_cast<const uint16_t*>(&sm.scale[st][1][row0 + nt * 8 + 2 * t4]);
                        k0 = pow2_of_byte(ks2 & 0xffu);
                        k1 = pow2_of_byte(ks2 >> 8);
                        ve[nt][0] = (float)(int)(vs2 & 0xffu) - 127.f;
                        ve[nt][1] = (float)(int)(vs2 >> 8) - 127.f;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bool seen = nt * 8 + 2 * t4 + e < n_vis;
                        const float kf = e ? k1 : k0;
                        const float xa = seen ? (kE4m3 ? sc[nt][e] * fA * kf : sc[nt][e] * fA) : -INFINITY;
                        const float xb = seen ? (kE4m3 ? sc[nt][2 + e] * fB * kf : sc[nt][2 + e] * fB) : -INFINITY;
                        sc[nt][e] = xa;
                        sc[nt][2 + e] = xb;
                        mxA = fmaxf(mxA, xa);
                        mxB = fmaxf(mxB, xb);
                        if (kE4m3) {
                            mxvA = fmaxf(mxvA, xa + ve[nt][e]);
                            mxvB = fmaxf(mxvB, xb + ve[nt][e]);
                        }
                    }
                }
#pragma unroll
                for (int x = 1; x < 4; x <<= 1) {
                    mxA = fmaxf(mxA, __shfl_xor_sync(0xffffffffu, mxA, x));
                    mxB = fmaxf(mxB, __shfl_xor_sync(0xffffffffu, mxB, x));
                    if (kE4m3) {
                        mxvA = fmaxf(mxvA, __shfl_xor_sync(0xffffffffu, mxvA, x));
                        mxvB = fmaxf(mxvB, __shfl_xor_sync(0xffffffffu, mxvB, x));
                    }
                }
                if (!kE4m3) {
                    mxvA = mxA;
                    mxvB = mxB;
                }
                if (__any_sync(0xffffffffu, mxA > mA || mxB > mB || mxvA > mvA || mxvB > mvB)) {
                    const float nA = fmaxf(mA, mxA), nB = fmaxf(mB, mxB), nvA = fmaxf(mvA, mxvA), nvB = fmaxf(mvB, mxvB);
                    lA = mA == -INFINITY ? 0.f : lA * fast_exp2(mA - nA);
                    lB = mB == -INFINITY ? 0.f : lB * fast_exp2(mB - nB);
                    const float cA = mvA == -INFINITY ? 0.f : fast_exp2(mvA - nvA), cB = mvB == -INFINITY ? 0.f : fast_exp2(mvB - nvB);
#pragma unroll
                    for (int dt = 0; dt < kDTiles; ++dt) {
                        o[dt][0] *= cA; o[dt][1] *= cA;
                        o[dt][2] *= cB; o[dt][3] *= cB;
                    }
                    mA = nA; mB = nB; mvA = nvA; mvB = nvB;
                }
                // (a maximum of -inf: every score of the row is; 2^(-inf - 0) = 0 then)
                const float refA = mA == -INFINITY ? 0.f : mA, refB = mB == -INFINITY ? 0.f : mB;
                const float refvA = (mvA == -INFINITY ? 0.f : mvA) - kPagedBias, refvB = (mvB == -INFINITY ? 0.f : mvB) - kPagedBias;
                uint32_t pf[kNTiles / 2][4];
#pragma unroll
                for (int nt = 0; nt < kNTiles; ++nt) {
                    const float p0 = fast_exp2(sc[nt][0] - refA), p1 = fast_exp2(sc[nt][1] - refA), p2 = fast_exp2(sc[nt][2] - refB), p3 = fast_exp2(sc[nt][3] - refB);
                    lA += p0 + p1;
                    lB += p2 + p3;
                    if (kE4m3) {
                        pf[nt / 2][(nt & 1) * 2] = pack_f16x2(fast_exp2(sc[nt][0] + ve[nt][0] - refvA), fast_exp2(sc[nt][1] + ve[nt][1] - refvA));
                        pf[nt / 2][(nt & 1) * 2 + 1] = pack_f16x2(fast_exp2(sc[nt][2] + ve[nt][0] - refvB), fast_exp2(sc[nt][3] + ve[nt][1] - refvB));
                    } else {
                        pf[nt / 2][(nt & 1) * 2] = pack_bf16x2(p0, p1);
                        pf[nt / 2][(nt & 1) * 2 + 1] = pack_bf16x2(p2, p3);
                    }
                }
                if (!kE4m3) {
#pragma unroll
                    for (int dp = 0; dp < kDTiles / 2; ++dp) {
                        const int row = row0 + (lane & 7) + (((lane >> 3) & 1) << 3), chunk = dp * 2 + (lane >> 4);
                        uint32_t b0, b1, b2, b3;
                        ldmatrix_x4_trans(b0, b1, b2, b3, vst + (chunk >> 3) * (kTile * 128) + sw128(row, chunk & 7));
                        mma_bf16_16816(o[dp * 2], pf[0], b0, b1);
                        mma_bf16_16816(o[dp * 2 + 1], pf[0], b2, b3);
                    }
                } else {
                    // Lane group g has the bytes [g * D / 8, (g + 1) * D / 8) of a key's values: column g of d tile i is d = g * D / 8 + i
#pragma unroll
                    for (int s = 0; s < kNTiles / 2; ++s) {
                        uint32_t v[4][D / 32];
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int row = row0 + s * 16 + 2 * t4 + (y & 1) + (y >> 1) * 8;
                            if (D == 128) {
                                const uint4 x = *reinterpret_cast<const uint4*>(vst + row * 128 + ((rA ^ (row & 7)) << 4));
                                v[y][0] = x.x; v[y][1] = x.y; v[y][D / 64] = x.z; v[y][D / 32 - 1] = x.w;
                            } else {
                                const uint2 x = *reinterpret_cast<const uint2*>(vst + row * 64 + (((rA >> 1) ^ ((row >> 1) & 3)) << 4) + (rA & 1) * 8);
                                v[y][0] = x.x; v[y][1] = x.y;
                            }
                        }
#pragma unroll
                        for (int x = 0; x < D / 32; ++x) {
                            const uint32_t lo0 = __byte_perm(v[0][x], v[1][x], 0x5140), hi0 = __byte_perm(v[0][x], v[1][x], 0x7362);
                            const uint32_t lo1 = __byte_perm(v[2][x], v[3][x], 0x5140), hi1 = __byte_perm(v[2][x], v[3][x], 0x7362);
                            mma_f16_16816(o[4 * x], pf[s], codes_to_f16x2(lo0 & 0xffffu), codes_to_f16x2(lo1 & 0xffffu));
                            mma_f16_16816(o[4 * x + 1], pf[s], codes_to_f16x2(lo0 >> 16), codes_to_f16x2(lo1 >> 16));
                            mma_f16_16816(o[4 * x + 2], pf[s], codes_to_f16x2(hi0 & 0xffffu), codes_to_f16x2(hi1 & 0xffffu));
                            mma_f16_16816(o[4 * x + 3], pf[s], codes_to_f16x2(hi0 >> 16), codes_to_f16x2(hi1 >> 16));
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm.empty[st]);
            if (++st == kStages) { st = 0; ph ^= 1; }
        }

        // ---- the four warps' states, one after the other into one (always in the same order)
        lA += __shfl_xor_sync(0xffffffffu, lA, 1);
        lA += __shfl_xor_sync(0xffffffffu, lA, 2);
        lB += __shfl_xor_sync(0xffffffffu, lB, 1);
        lB += __shfl_xor_sync(0xffffffffu, lB, 2);
        if (t4 == 0) {
            *reinterpret_cast<float4*>(sm.stat[warp][rA]) = make_float4(mA, lA, mvA, 0.f);
            *reinterpret_cast<float4*>(sm.stat[warp][rB]) = make_float4(mB, lB, mvB, 0.f);
        }
        consumer_sync();
        float allvA = -INFINITY, allvB = -INFINITY;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            allvA = fmaxf(allvA, sm.stat[x][rA][2]);
            allvB = fmaxf(allvB, sm.stat[x][rB][2]);
        }
        const float cA = mvA == -INFINITY ? 0.f : fast_exp2(mvA - allvA), cB = mvB == -INFINITY ? 0.f : fast_exp2(mvB - allvB);
#pragma unroll 1
        for (int x = 0; x < 4; ++x) {
            if (warp == x) {
#pragma unroll
                for (int dt = 0; dt < kDTiles; ++dt) {
                    float2* da = reinterpret_cast<float2*>(&sm.red[rA][(dt * 8 + 2 * t4) ^ ((rA & 3) << 3)]);
                    float2* db = reinterpret_cast<float2*>(&sm.red[rB][(dt * 8 + 2 * t4) ^ ((rB & 3) << 3)]);
                    const float2 wasA = x ? *da : make_float2(0.f, 0.f);
                    *da = make_float2(wasA.x + o[dt][0] * cA, wasA.y + o[dt][1] * cA);
                    if (a.G > 8) {
                        const float2 wasB = x ? *db : make_float2(0.f, 0.f);
                        *db = make_float2(wasB.x + o[dt][2] * cB, wasB.y + o[dt][3] * cB);
                    }
                }
            }
            consumer_sync();
        }
        const bool whole = w.tile == 0 && n_here == w.tiles;
        const bool bad = *(volatile int*)&sm.bad[part & 1] == part + 1;
        const int slot = w.tile > 0 ? 0 : 1;                  // a part that goes on from an earlier run, one that begins here
        float* dst = a.partial + ((size_t)(blockIdx.x * 2 + slot) * a.G) * kRowF;
        for (int idx = tid; idx < a.G * (D / 2); idx += 128) {
            const int row = idx / (D / 2), d = (idx % (D / 2)) * 2;
            float m = -INFINITY, mv = -INFINITY, l = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                m = fmaxf(m, sm.stat[x][row][0]);
                mv = fmaxf(mv, sm.stat[x][row][2]);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float mx = sm.stat[x][row][0], lx = sm.stat[x][row][1];
                if (lx != 0.f) l += lx * fast_exp2(mx == -INFINITY ? 0.f : mx - m);
            }
            // e4m3: column c of d tile i is d = c * D / 8 + i
            const int c0 = kE4m3 ? (d % (D / 8)) * 8 + d / (D / 8) : d, c1 = kE4m3 ? ((d + 1) % (D / 8)) * 8 + (d + 1) / (D / 8) : d + 1;
            const float o0 = sm.red[row][c0 ^ ((row & 3) << 3)], o1 = sm.red[row][c1 ^ ((row & 3) << 3)];
            if (whole) {
                const float f = kE4m3 ? exp2f(mv - m - kPagedBias) : 1.f, inv = 1.f / l;
                const size_t at = (size_t)w.b * a.Hq + w.gk * a.G + row;
                *reinterpret_cast<uint32_t*>(a.out + at * D + d) = bad ? 0u : pack_bf16x2(o0 * inv * f, o1 * inv * f);
                if (d == 0 && a.lse != nullptr) a.lse[at] = bad ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            } else {
                float* r = dst + row * kRowF;
                *reinterpret_cast<float2*>(r + 4 + d) = make_float2(o0, o1);
                if (d == 0) *reinterpret_cast<float4*>(r) = make_float4(m, bad ? -1.f : l, kE4m3 ? mv - kPagedBias : m, 0.f);
            }
        }
        consumer_sync();                                      // the statistics and the sums may be overwritten
        it += n_here;
        if (it < it1) w.next();
    }
    if (tid == 0 && sm.abort_flag && a.status != nullptr) atomicExch(a.status, 6);
}

// grid (Hq, batch), 512 threads: the parts of one row in the order of the runs, 512 / D groups of threads a share each.  Rows of sequences
// that are not there (or whose length is out of range: status 1) become zeros.  n_ctas: of the kernel before.
template <int D, bool kE4m3>
__global__ void __launch_bounds__(512) paged_join_kernel(PageGeom p, PagedCall a, int n_ctas) {
    constexpr int kTile = paged_tile(kE4m3), kGroups = 512 / D, kRowF = paged_row_floats(D);
    __shared__ float weight[kPagedCtas];
    __shared__ float red[kGroups][D];
    __shared__ float all[4];                                  // m, l, m', bad
    __shared__ int range[2];                                  // first and last run; first < 0: nothing to join, -2: zeros
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gk = h / a.G, row = h - gk * a.G;
    launch_dependents();
    wait_for_previous_kernel();
    if (warp == 0) {
        TileLine<kTile> line;
        line.p = &p;
        line.kv_len = a.kv_len;
        line.batch = a.batch;
        line.lane = lane;
        long long before = 0, total = 0;
        for (int c = 0; c < a.batch; c += 32) {
            line.load(c);
            long long t = line.tiles, u = c + lane < b ? t : 0;
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) {
                t += __shfl_xor_sync(0xffffffffu, t, x);
                u += __shfl_xor_sync(0xffffffffu, u, x);
            }
            total += t;
            before += u;
        }
        if (lane == 0) {
            const int n = a.kv_len[b], tiles = line.count(n);
            if (tiles == 0) {
                range[0] = -2;
                if (n != 0 && h == 0 && a.status != nullptr) atomicExch(a.status, 1);
            } else {
                total *= p.Hkv;
                const long long begin = before * p.Hkv + (long long)gk * tiles;
                const int n_runs = run_count(total, n_ctas), c0 = run_of(total, n_runs, begin), c1 = run_of(total, n_runs, begin + tiles - 1);
                range[0] = c0 == c1 ? -1 : c0;
                range[1] = c1;
            }
        }
    }
    __syncthreads();
    const int c0 = range[0], c1 = range[1];
    const size_t at = (size_t)b * a.Hq + h;
    if (c0 == -1) return;
    if (c0 == -2) {
        if (tid < D / 2) *reinterpret_cast<uint32_t*>(a.out + at * D + 2 * tid) = 0u;
        if (tid == 0 && a.lse != nullptr) a.lse[at] = -INFINITY;
        return;
    }
    const int n = c1 - c0 + 1;
    // part i lies with run c0 + i: the first in its slot 1, the others in slot 0
    auto part = [&](int i) -> const float* { return a.partial + ((size_t)((c0 + i) * 2 + (i == 0 ? 1 : 0)) * a.G + row) * kRowF; };
    if (warp == 0) {
        float m = -INFINITY, mv = -INFINITY, l = 0.f;
        bool bad = false;
        for (int i = lane; i < n; i += 32) {
            const float4 s = *reinterpret_cast<const float4*>(part(i));
            m = fmaxf(m, s.x);
            mv = fmaxf(mv, s.z);
            bad = bad || s.y == -1.f;
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
            mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, x));
        }
        for (int i = lane; i < n; i += 32) {
            const float4 s = *reinterpret_cast<const float4*>(part(i));
            if (s.y != 0.f) l += s.y * fast_exp2(s.x == -INFINITY ? 0.f : s.x - m);
            weight[i] = s.z == -INFINITY ? 0.f : fast_exp2(s.z - mv);
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) {
            all[0] = m;
            all[1] = l;
            all[2] = mv;
            all[3] = bad ? 1.f : 0.f;
        }
    }
    __syncthreads();
    const int d = tid & (D - 1), grp = tid / D;
    float acc = 0.f;
#pragma unroll 8
    for (int i = grp; i < n; i += kGroups) acc = fmaf(part(i)[4 + d], weight[i], acc);
    red[grp][d] = acc;
    __syncthreads();
    if (grp == 0) {
#pragma unroll
        for (int i = 1; i < kGroups; ++i) acc += red[i][d];
        const float f = kE4m3 ? exp2f(all[2] - all[0]) : 1.f;
        const bool bad = all[3] != 0.f;
        a.out[at * D + d] = __float2bfloat16(bad ? 0.f : acc / all[1] * f);
        if (d == 0 && a.lse != nullptr) a.lse[at] = bad ? -INFINITY : (all[0] + log2f(all[1])) * 0.6931471805599453f;
    }
}

}  // namespace adaspark
