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
// The scores are S = q K^T with the heads as rows (an 8-row half of the m16 tile where the group has at most 8), the outputs
// O^T = V^T P^T with the heads as columns: S's accumulators are P^T's operand as they stand, and O takes half the registers and products.
//
// 8-bit pages go through the tensor cores as f16, which holds every e4m3 value.  q is brought to f16 by a power of two per row (largest
// magnitude 2^14 ..: what falls below 2^-28 of it loses bits, 2^-39 of it at most); a key's power of two multiplies its score.  A value's
// power of two e_j joins its weight: the weights of the product are 2^(x_j + e_j - m') with their own maximum m', so that they stay
// within f16 whatever the rows' sizes, and beside them the sum of 2^(x_j - m) is kept.  A score is multiplied by the powers of two of q and key
// one after the other, the one below 1 first where q is large: they may lie at opposite ends of the range.  (K as e4m3 against q in two e4m3 parts: no faster, the
// legacy 8-bit products are converted, too, and half as fast with more than 8 heads.)
//
// With a window (kWin) of the last `window` tokens and the `sinks` first ones, a sequence's line holds the tiles of the first ones and those from the
// window's first on, as if they were neighbours; tiles at the two borders are masked as the last one is.  Pages that hold nothing that is
// seen are not read, and their numbers may be any.
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"
#include "tc_common.cuh"

namespace adaspark {

constexpr int kPagedThreads = 160;
constexpr int kPagedCtas = 296;              // two per SM of a B200
constexpr int kPagedRing = 96 * 1024;        // bytes of a CTA's ring
// What a part costs beside its tiles, in tiles (24 sequences of up to 8192 tokens, bf16, at 0 / 1 / 2 / 3: 35.9 / 28.7 / 25.2 / 24.2 us, 128 of 20 to
// 1000 at 2 / 3: 30.4 / 31.4; 64 of 16 to 8192 in 8 bits, tiles of twice the keys, at 1 / 2 / 4: 39.7 / 40.5 / 43.2).
__host__ __device__ constexpr int paged_part_cost(int tile) { return tile == 64 ? 2 : 1; }
constexpr int kPagedFewSequences = 16;       // up to so many (sequence, kv head)s, 18 runs each on average where there are tiles enough: a CTA joins a row
constexpr float kPagedBias = 14.f;           // f16 weights are at most 2^14: 2^-28 of the largest one is still a normal number

__host__ __device__ constexpr int paged_tile(bool e4m3) { return e4m3 ? 128 : 64; }   // keys of a tile
// Tiles of n tokens, and pieces of `size` that the first tile of n > 0 tokens holds keys in; a table may have room for 2^31 - 1 tokens.
__host__ __device__ constexpr int paged_tiles(int n, int tile) { return n > 0 ? (n - 1) / tile + 1 : 0; }
__host__ __device__ constexpr int paged_pieces(int n, int tile, int size) { return ((n < tile ? n : tile) + size - 1) / size; }
__host__ __device__ constexpr int paged_row_floats(int D) { return D + 4; }           // m, l, m', -, o[D]
__host__ __device__ constexpr size_t paged_partial_bytes(int D, int G) { return (size_t)kPagedCtas * 2 * G * paged_row_floats(D) * sizeof(float); }

// The new token's rows of one kv head into their place; by the 32 lanes of a warp, of which lane % (D / 8) holds k and v, 8 values each.
template <int D, bool kE4m3>
__device__ __forceinline__ void append_rows(const PageGeom& p, int page, int head, int place, uint4 k, uint4 v, int lane) {
    constexpr int kLanes = D / 8;
    const long long row = ((long long)head << p.page_shift) + place, at = (long long)page * p.page_stride + row * D + lane % kLanes * 8;
    if (kE4m3) {
        uint32_t tops = row_tops<kLanes>(chunk_tops(k), chunk_tops(v));
        if (__any_sync(0xffffffffu, any_odd(tops))) {
            tops = row_tops<kLanes>(chunk_finite_tops(k), chunk_finite_tops(v));
            k = infinities_to_nan(k);
            v = infinities_to_nan(v);
        }
        const uint32_t sk = scale_byte(tops & 0xffffu), sv = scale_byte(tops >> 16);
        if (lane < kLanes) {
            *reinterpret_cast<uint2*>(p.k + at) = chunk_codes(k, sk);
            *reinterpret_cast<uint2*>(p.v + at) = chunk_codes(v, sv);
        }
        if (lane == 0) {
            p.ks[(long long)page * p.scale_stride + row] = (uint8_t)sk;
            p.vs[(long long)page * p.scale_stride + row] = (uint8_t)sv;
        }
    } else if (lane < kLanes) {
        *reinterpret_cast<uint4*>(p.k + at * 2) = k;
        *reinterpret_cast<uint4*>(p.v + at * 2) = v;
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
    int window, sinks;                       // kWin
};

// The line of tiles: sequence by sequence, kv head by kv head, in front of each (sequence, kv head) paged_part_cost places for what a part costs
// beside its tiles (q, the merge of the warps, the output).  Held by a whole warp, which has the lengths of 32 sequences in its lanes.
template <int kTile, bool kWin>
struct PageLine {
    const PageGeom* p;
    const PagedCall* a;
    const int32_t* kv_len;
    int batch, lane;
    int chunk, len;                          // first sequence of the lanes' 32, tokens of this lane's sequence (0: none, or out of range)
    __device__ __forceinline__ bool in_range(int n) const { return n >= 0 && n <= (p->table_width << p->page_shift); }
    __device__ __forceinline__ void load(int c) {
        chunk = c;
        const int n = c + lane < batch ? kv_len[c + lane] : 0;
        len = in_range(n) ? n : 0;
    }
    // tiles of n tokens that hold something that is seen
    __device__ __forceinline__ int tiles_of(int n) const {
        const int all = paged_tiles(n, kTile);
        return kWin ? all - max(max(n - a->window, 0) / kTile - paged_tiles(a->sinks, kTile), 0) : all;
    }
    // where tile t of those lies in the sequence
    __device__ __forceinline__ int tile_at(int n, int tiles, int t) const { return kWin && t >= paged_tiles(a->sinks, kTile) ? t + paged_tiles(n, kTile) - tiles : t; }
    // places of one (sequence, kv head) of n tokens
    __device__ __forceinline__ int places(int n) const { return n > 0 ? tiles_of(n) + paged_part_cost(kTile) : 0; }
    __device__ __forceinline__ long long total() {
        long long sum = 0;
        for (int c = 0; c < batch; c += 32) {
            load(c);
            const unsigned x = (unsigned)places(len);
            sum += (long long)__reduce_add_sync(0xffffffffu, x & 0xffffu) + ((long long)__reduce_add_sync(0xffffffffu, x >> 16) << 16);
        }
        return sum * p->Hkv;
    }
};

// The line's places are cut into runs of at least one: how many, the first place of run c, and the run that holds place x.
__device__ __forceinline__ int run_count(long long total, int n_ctas) { return (int)min(total, (long long)n_ctas); }
__device__ __forceinline__ long long run_begin(long long total, int n_runs, int c) { return total * c / n_runs; }
__device__ __forceinline__ int run_of(long long total, int n_runs, long long x) { return (int)(((x + 1) * n_runs - 1) / total); }

// A walk along a run, part by part: the tiles [tile, end) of (sequence b, kv head gk), which has n tokens in `tiles` tiles.
template <int kTile, bool kWin>
struct RunWalk {
    PageLine<kTile, kWin> line;
    long long place, stop;                   // first place of the (sequence, kv head); first place behind the run
    int b, gk, n, tiles, tile, end;
    // to place x < total; false: no tile there (only the places in front of one)
    __device__ __forceinline__ bool seek(long long x, long long run_end) {
        stop = run_end;
        long long before = 0;
        for (int c = 0; c < line.batch; c += 32) {
            line.load(c);
            const long long mine = (long long)line.places(line.len) * line.p->Hkv;
            long long upto = mine;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, upto, s);
                if (line.lane >= s) upto += y;
            }
            const long long all = __shfl_sync(0xffffffffu, upto, 31);
            if (x < before + all) {
                const int who = __ffs(__ballot_sync(0xffffffffu, before + upto > x)) - 1;
                const long long first = before + __shfl_sync(0xffffffffu, upto - mine, who);
                b = c + who;
                n = __shfl_sync(0xffffffffu, line.len, who);
                tiles = line.tiles_of(n);
                const int per = tiles + paged_part_cost(kTile), rest = (int)(x - first);
                gk = rest / per;
                place = first + (long long)gk * per;
                return begin(max(rest - gk * per - paged_part_cost(kTile), 0));
            }
            before += all;
        }
        return false;
    }
    // to the first place of (sequence b, kv head gk); false: it has none
    __device__ __forceinline__ bool seek_sequence(int seq, int head, long long total) {
        stop = total;
        place = 0;
        for (int c = 0; c <= seq; c += 32) {
            line.load(c);
            long long x = c + line.lane < seq ? line.places(line.len) : 0;
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
            place += x * line.p->Hkv;
        }
        n = __shfl_sync(0xffffffffu, line.len, seq & 31);
        b = seq;
        gk = head;
        tiles = line.tiles_of(n);
        place += (long long)head * line.places(n);
        return begin(0);
    }
    // the part that begins with tile t; false: the run ends in front of it
    __device__ __forceinline__ bool begin(int t) {
        tile = t;
        end = (int)min((long long)tiles, max(stop - place - paged_part_cost(kTile), 0ll));
        return end > tile;
    }
    // the next part
    __device__ __forceinline__ bool next() {
        place += tiles + paged_part_cost(kTile);
        if (place >= stop) return false;
        if (++gk < line.p->Hkv) return begin(0);
        gk = 0;
        int from = b + 1 - line.chunk;
        while (true) {
            const uint32_t there = from < 32 ? __ballot_sync(0xffffffffu, line.len > 0) >> from << from : 0u;
            if (there) {
                const int who = __ffs(there) - 1;
                b = line.chunk + who;
                n = __shfl_sync(0xffffffffu, line.len, who);
                tiles = line.tiles_of(n);
                return begin(0);
            }
            if (line.chunk + 32 >= line.batch) return false;
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
    float red[16][D + 4];                                     // outputs of a part: 16 heads, or 8 of two halves
    __nv_bfloat16 q[16][D + 8];                               // of one part (16 heads), or two (8 heads)
    unsigned char scale[kStages][2][kE4m3 ? kTile : 16];
    float stat[4][16][4];
    uint64_t full[kStages], empty[kStages], q_full[2], q_empty[2];
    int bad[4];                                               // number + 1 of a part with a page that is not there
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
// four codes -> two f16 pairs
__device__ __forceinline__ void codes_to_f16x4(uint32_t c, uint32_t& a, uint32_t& b) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}\n" : "=r"(a), "=r"(b) : "r"(c));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;\n" ::: "memory"); }

// kGroups: groups of 8 heads, (G + 7) / 8.
template <int D, bool kE4m3, int kGroups, bool kWin>
__global__ void __launch_bounds__(kPagedThreads, 2) paged_decode_kernel(PageGeom p, PagedCall a, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV) {
    using Smem = PagedSmem<D, kE4m3>;
    extern __shared__ __align__(1024) unsigned char paged_smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>(paged_smem_raw);
    constexpr int kTile = Smem::kTile, kStages = Smem::kStages, kRowBytes = Smem::kRowBytes;
    constexpr int kWarpKeys = kTile / 4, kNTiles = kWarpKeys / 8, kRowF = paged_row_floats(D);
    constexpr int kMTiles = D / 16;                           // O^T: tiles of 16 d
    constexpr int kQSlots = kGroups == 1 ? 2 : 1;             // parts whose q is held
    constexpr int kQSteps = D / 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(&sm.full[s], 1);
            tc::mbar_init(&sm.empty[s], 4);
        }
        for (int s = 0; s < 2; ++s) {
            tc::mbar_init(&sm.q_full[s], 1);
            tc::mbar_init(&sm.q_empty[s], 4);
        }
        for (int s = 0; s < 4; ++s) sm.bad[s] = 0;
        sm.abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tensormap(&tmK);
        tc::prefetch_tensormap(&tmV);
    }
    __syncthreads();
    volatile int* abort_flag = &sm.abort_flag;
    wait_for_previous_kernel();
    launch_dependents();                                      // (after the wait: the next kernel reads kv_len before its own)

    RunWalk<kTile, kWin> w;
    w.line.p = &p;
    w.line.a = &a;
    w.line.kv_len = a.kv_len;
    w.line.batch = a.batch;
    w.line.lane = lane;
    const long long total = w.line.total();
    const int n_runs = run_count(total, gridDim.x);
    bool more = (int)blockIdx.x < n_runs && w.seek(run_begin(total, n_runs, blockIdx.x), run_begin(total, n_runs, blockIdx.x + 1));
    const int page_shift = p.page_shift, page_size = 1 << page_shift;

    if (warp == 4) {
        // ------------------------------------------------------------ producer
        const int sub = min(page_size, kTile);               // tokens of a box
        int st = 0, ph = 1;
        // page numbers: this lane's of the 32 columns from `cols` on of sequence `cols_b`, and of the 32 behind them
        int cols_b = -1, cols = 0, pages = 0, pages_next = 0;
        bool ok = true;
        for (int part = 0; more && ok; ++part, more = w.next()) {
            const int32_t* table = p.table + (size_t)w.b * p.table_width;
            const int last_col = (w.n - 1) >> page_shift, col_begin = (w.line.tile_at(w.n, w.tiles, w.tile) * kTile) >> page_shift;
            auto page_at = [&](int col) -> int { return col <= last_col ? table[col] : 0; };
            if (cols_b != w.b || col_begin < cols) {
                cols_b = w.b;
                cols = col_begin;
                pages = page_at(cols + lane);
                pages_next = page_at(cols + 32 + lane);
            }
            uint4 new_k = make_uint4(0u, 0u, 0u, 0u), new_v = new_k;
            if (a.k_new != nullptr && w.end == w.tiles) {     // (asked for here, beside the page numbers)
                new_k = *reinterpret_cast<const uint4*>(a.k_new + w.b * a.k_ts + w.gk * a.k_hs + lane % (D / 8) * 8);
                new_v = *reinterpret_cast<const uint4*>(a.v_new + w.b * a.v_ts + w.gk * a.v_hs + lane % (D / 8) * 8);
            }
            // q of the heads, a row each
            const int qs = part % kQSlots;
            if (!(ok = tc::mbar_wait_warp(&sm.q_empty[qs], ((part / kQSlots) & 1) ^ 1, abort_flag))) break;
            if (lane == 0) tc::mbar_arrive_expect_tx(&sm.q_full[qs], (uint32_t)a.G * D * 2);
            __syncwarp();
            if (lane < a.G) tc::bulk_load(&sm.q[qs * 8 + lane][0], a.q + w.b * a.q_ts + (w.gk * a.G + lane) * a.q_hs, D * 2, &sm.q_full[qs]);
            for (int tile = w.tile; tile < w.end; ++tile) {
                const int pos0 = w.line.tile_at(w.n, w.tiles, tile) * kTile, col0 = pos0 >> page_shift;
                if (kWin && col0 >= cols + 64) {              // over what lies between the first tokens and the window
                    cols = col0;
                    pages = page_at(cols + lane);
                    pages_next = page_at(cols + 32 + lane);
                }
                while (col0 >= cols + 32) {
                    cols += 32;
                    pages = pages_next;
                    pages_next = page_at(cols + 32 + lane);
                }
                const int boxes = paged_pieces(w.n - pos0, kTile, sub);   // those that hold a token
                int page = __shfl_sync(0xffffffffu, pages, min(col0 - cols + lane, 31));
                const int over = __shfl_sync(0xffffffffu, pages_next, max(col0 - cols + lane - 32, 0) & 31);
                if (col0 - cols + lane >= 32) page = over;
                bool there = page >= 0 && page < p.n_pages;
                // a box of tokens that are not seen is not read: zeros
                const int box0 = pos0 + lane * sub;
                const bool seen = !kWin || box0 < a.sinks || box0 + sub > w.n - a.window;
                if (kWin && !seen) there = false;
                if (__any_sync(0xffffffffu, lane < boxes && seen && !there)) {
                    if (lane == 0) {
                        sm.bad[part & 3] = part + 1;
                        if (a.status != nullptr) atomicExch(a.status, 1);
                    }
                }
                if (a.k_new != nullptr && tile == w.tiles - 1) {           // the new token: the last of this tile
                    const int pg = __shfl_sync(0xffffffffu, page, boxes - 1), place = (w.n - 1) & (page_size - 1);
                    if (pg >= 0 && pg < p.n_pages) {                       // (whatever the other pages are)
                        append_rows<D, kE4m3>(p, pg, w.gk, place, new_k, new_v, lane);
                        asm volatile("fence.proxy.async;\n" ::: "memory");    // it is read by the copies below
                        __syncwarp();
                    }
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
                        tc::bulk_load(&sm.scale[st][0][lane * sub], p.ks + s_at, sub, &sm.full[st]);
                        tc::bulk_load(&sm.scale[st][1][lane * sub], p.vs + s_at, sub, &sm.full[st]);
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
        }
        return;
    }
    // ---------------------------------------------------------------- consumers (they keep to their barriers when a wait has expired)
    const int g8 = lane >> 2, t4 = lane & 3;                  // the lane's row and column pair of a fragment
    int st = 0, ph = 0;
    for (int part = 0; more; ++part, more = w.next()) {
        const int n = w.n, qs = part % kQSlots;
        // ---- q fragments: rows = heads
        uint32_t qf[kQSteps][4];
        float f[kGroups];                                     // what the products of head g8 (g8 + 8) are multiplied by
        tc::mbar_wait(&sm.q_full[qs], (part / kQSlots) & 1, abort_flag);
        {
            const __nv_bfloat16* qr[2] = {sm.q[qs * 8 + g8], sm.q[(kGroups == 2 ? 8 : 0) + g8]};
            const bool has[2] = {g8 < a.G, kGroups == 2 && g8 + 8 < a.G};
#pragma unroll
            for (int ks = 0; ks < kQSteps; ++ks)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    // e4m3: thread t4 of a quad has the 16-byte chunks 2 t4, 2 t4 + 1 (D = 64: t4) of a key's codes; step (chunk, word w) takes
                    // d = 16 * chunk + 4 w + 0, 1 and + 2, 3 as the k indexes 2 t4, + 1 and 2 t4 + 8, + 9
                    const int d = kE4m3 ? 16 * (D == 128 ? 2 * t4 + (ks >> 2) : t4) + 4 * (ks & 3) : ks * 16 + 2 * t4;
                    qf[ks][r] = has[r] ? *reinterpret_cast<const uint32_t*>(qr[r] + d) : 0u;
                    qf[ks][2 + r] = has[r] ? *reinterpret_cast<const uint32_t*>(qr[r] + d + (kE4m3 ? 2 : 8)) : 0u;
                }
#pragma unroll
            for (int r = 0; r < kGroups; ++r) {
                f[r] = a.scale_log2;
                if (kE4m3) {
                    uint32_t top = 0u;
#pragma unroll
                    for (int ks = 0; ks < kQSteps; ++ks) top = __vmaxu2(top, __vmaxu2(qf[ks][r] & 0x7fff7fffu, qf[ks][2 + r] & 0x7fff7fffu));
                    top = max(top & 0xffffu, top >> 16);
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const int e = max((int)(top >> 7), 30);                // biased exponent of the largest: it becomes 2^14
                    const float mul = __uint_as_float((uint32_t)(127 + 141 - e) << 23);
                    f[r] *= __uint_as_float((uint32_t)min(127 + e - 141, 254) << 23);     // (e = 255, no number: it stays one)
#pragma unroll
                    for (int ks = 0; ks < kQSteps; ++ks)
#pragma unroll
                        for (int y = 0; y < 4; y += 2)
                            qf[ks][y + r] = pack_f16x2(__uint_as_float(qf[ks][y + r] << 16) * mul, __uint_as_float(qf[ks][y + r] & 0xffff0000u) * mul);
                }
            }
        }
        // a factor above 1 (queries above 2^16) comes behind the keys' powers of two, which may be as far at the other end of the range
        const bool large = kE4m3 && __any_sync(0xffffffffu, f[0] > 1.f || f[kGroups - 1] > 1.f);
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sm.q_empty[qs]);

        // running maximum and sum of head g8 (g8 + 8); with e4m3 pages mv is the maximum of the weights of the products
        float m[kGroups], l[kGroups], mv[kGroups], o[kGroups][kMTiles][4];
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            m[r] = mv[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int i = 0; i < kMTiles; ++i) o[r][i][0] = o[r][i][1] = o[r][i][2] = o[r][i][3] = 0.f;
        }
        for (int tile = w.tile; tile < w.end; ++tile) {
            const int key0 = w.line.tile_at(n, w.tiles, tile) * kTile + warp * kWarpKeys;
            const int n_vis = n - key0;                                    // keys of this warp's quarter that are there
            // of these, [hide0, hide1) lie between the first ones and the window
            const int hide0 = kWin ? max(a.sinks - key0, 0) : 0, hide1 = kWin ? min(n - a.window - key0, kWarpKeys) : 0;
            const bool hides = kWin && hide0 < hide1;
            tc::mbar_wait(&sm.full[st], ph, abort_flag);
            if (n_vis > 0 && !(kWin && hide0 == 0 && hide1 == kWarpKeys)) {
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
                if (hides) {                                  // what is hidden may be anything, too
                    constexpr int kChunks = kRowBytes / 16;
                    for (int c = lane; c < (hide1 - hide0) * kChunks; c += 32) {
                        const int r = row0 + hide0 + c / kChunks, x = c % kChunks;
                        unsigned char* dst = kE4m3 ? vst + r * kRowBytes + x * 16 : vst + (x >> 3) * (kTile * 128) + r * 128 + (x & 7) * 16;
                        *reinterpret_cast<uint4*>(dst) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                }
                float x[kGroups][kNTiles][2];                 // scores of keys 8 nt + 2 t4, + 1, times scale_log2
                float ve[kNTiles][2];                         // their values' e_j
                {
                    float sc[kNTiles][4];
#pragma unroll
                    for (int nt = 0; nt < kNTiles; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
                    if (!kE4m3) {
#pragma unroll
                        for (int ks = 0; ks < kQSteps; ++ks) {
                            const int row = row0 + (lane & 7) + ((lane >> 4) << 3), chunk = ks * 2 + ((lane >> 3) & 1);
                            uint32_t b0, b1, b2, b3;
                            ldmatrix_x4(b0, b1, b2, b3, kst + (chunk >> 3) * (kTile * 128) + sw128(row, chunk & 7));
                            mma_bf16_16816(sc[0], qf[ks], b0, b1);
                            mma_bf16_16816(sc[1], qf[ks], b2, b3);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < D / 64; ++j) {
                            uint4 c[kNTiles];
#pragma unroll
                            for (int nt = 0; nt < kNTiles; ++nt) {
                                const int row = row0 + nt * 8 + g8;
                                c[nt] = D == 128 ? *reinterpret_cast<const uint4*>(kst + row * 128 + (((2 * t4 + j) ^ (row & 7)) << 4))
                                                 : *reinterpret_cast<const uint4*>(kst + row * 64 + ((t4 ^ ((row >> 1) & 3)) << 4));
                            }
#pragma unroll
                            for (int y = 0; y < 4; ++y)
#pragma unroll
                                for (int nt = 0; nt < kNTiles; ++nt) {
                                    uint32_t b0, b1;
                                    codes_to_f16x4(y == 0 ? c[nt].x : y == 1 ? c[nt].y : y == 2 ? c[nt].z : c[nt].w, b0, b1);
                                    mma_f16_16816(sc[nt], qf[j * 4 + y], b0, b1);
                                }
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < kNTiles; ++nt) {
                        float kf[2] = {1.f, 1.f};
                        if (kE4m3) {
                            const uint32_t ks2 = *reinterpret_cast<const uint16_t*>(&sm.scale[st][0][row0 + nt * 8 + 2 * t4]);
                            const uint32_t vs2 = *reinterpret_cast<const uint16_t*>(&sm.scale[st][1][row0 + nt * 8 + 2 * t4]);
                            kf[0] = __uint_as_float(max((ks2 & 0xffu) << 23, 0x00400000u));   // (byte 0: 2^-127, a subnormal number)
                            kf[1] = __uint_as_float(max((ks2 >> 8) << 23, 0x00400000u));
                            ve[nt][0] = (float)(int)(vs2 & 0xffu) - 127.f;
                            ve[nt][1] = (float)(int)(vs2 >> 8) - 127.f;
                        }
#pragma unroll
                        for (int r = 0; r < kGroups; ++r)
#pragma unroll
                            for (int e = 0; e < 2; ++e) x[r][nt][e] = kE4m3 ? sc[nt][2 * r + e] * fminf(f[r], 1.f) * kf[e] : sc[nt][2 * r + e] * f[r];
                    }
                    if (kE4m3 && large) {
#pragma unroll
                        for (int r = 0; r < kGroups; ++r)
#pragma unroll
                            for (int nt = 0; nt < kNTiles; ++nt) {
                                x[r][nt][0] *= fmaxf(f[r], 1.f);
                                x[r][nt][1] *= fmaxf(f[r], 1.f);
                            }
                    }
                }
                if (n_vis < kWarpKeys) {
#pragma unroll
                    for (int r = 0; r < kGroups; ++r)
#pragma unroll
                        for (int nt = 0; nt < kNTiles; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (nt * 8 + 2 * t4 + e >= n_vis) x[r][nt][e] = -INFINITY;
                }
                if (hides) {
#pragma unroll
                    for (int r = 0; r < kGroups; ++r)
#pragma unroll
                        for (int nt = 0; nt < kNTiles; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (nt * 8 + 2 * t4 + e >= hide0 && nt * 8 + 2 * t4 + e < hide1) x[r][nt][e] = -INFINITY;
                }
                uint32_t pf[kGroups][kNTiles];                // P^T: two keys of a head
#pragma unroll
                for (int r = 0; r < kGroups; ++r) {
                    float mx = -INFINITY, mxv = -INFINITY;
#pragma unroll
                    for (int nt = 0; nt < kNTiles; ++nt) {
                        mx = fmax3(mx, x[r][nt][0], x[r][nt][1]);
                        if (kE4m3) mxv = fmax3(mxv, x[r][nt][0] + ve[nt][0], x[r][nt][1] + ve[nt][1]);
                    }
#pragma unroll
                    for (int y = 1; y < 4; y <<= 1) {
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, y));
                        if (kE4m3) mxv = fmaxf(mxv, __shfl_xor_sync(0xffffffffu, mxv, y));
                    }
                    if (!kE4m3) mxv = mx;
                    if (__any_sync(0xffffffffu, mx > m[r] || mxv > mv[r])) {
                        const float nm = fmaxf(m[r], mx), nmv = fmaxf(mv[r], mxv);
                        if (m[r] != -INFINITY) l[r] *= fast_exp2(m[r] - nm);   // (else it is zero, or no number and stays that)
                        const float c = mv[r] == -INFINITY ? 0.f : fast_exp2(mv[r] - nmv);
                        // of heads 2 t4 and 2 t4 + 1, the columns of O^T
                        const float c0 = __shfl_sync(0xffffffffu, c, 8 * t4), c1 = __shfl_sync(0xffffffffu, c, 8 * t4 + 4);
#pragma unroll
                        for (int i = 0; i < kMTiles; ++i) {
                            o[r][i][0] *= c0; o[r][i][2] *= c0;
                            o[r][i][1] *= c1; o[r][i][3] *= c1;
                        }
                        m[r] = nm;
                        mv[r] = nmv;
                    }
                    // (a maximum of -inf: every score of the head is; 2^(-inf - 0) = 0 then)
                    const float ref = m[r] == -INFINITY ? 0.f : m[r], refv = (mv[r] == -INFINITY ? 0.f : mv[r]) - kPagedBias;
#pragma unroll
                    for (int nt = 0; nt < kNTiles; ++nt) {
                        const float p0 = fast_exp2(x[r][nt][0] - ref), p1 = fast_exp2(x[r][nt][1] - ref);
                        l[r] += p0 + p1;
                        pf[r][nt] = kE4m3 ? pack_f16x2(fast_exp2(x[r][nt][0] + (ve[nt][0] - refv)), fast_exp2(x[r][nt][1] + (ve[nt][1] - refv))) : pack_bf16x2(p0, p1);
                    }
                }
                if (!kE4m3) {
#pragma unroll
                    for (int i = 0; i < kMTiles; ++i) {       // rows d of V^T: (keys 0..7, d lo), (keys 0..7, d hi), (keys 8..15, d lo), (keys 8..15, d hi)
                        const int row = row0 + (lane & 7) + ((lane >> 4) << 3), chunk = i * 2 + ((lane >> 3) & 1);
                        uint32_t v[4];
                        ldmatrix_x4_trans(v[0], v[1], v[2], v[3], vst + (chunk >> 3) * (kTile * 128) + sw128(row, chunk & 7));
#pragma unroll
                        for (int r = 0; r < kGroups; ++r) mma_bf16_16816(o[r][i], v, pf[r][0], pf[r][1]);
                    }
                } else {
                    // Lane group g8 has the bytes [g8 * D / 8, (g8 + 1) * D / 8) of a key's values: rows g8 and g8 + 8 of d tile i are
                    // d = g8 * D / 8 + 2 i and + 1
#pragma unroll
                    for (int s = 0; s < kNTiles / 2; ++s) {
                        uint32_t v[4][D / 32];
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int row = row0 + s * 16 + 2 * t4 + (y & 1) + (y >> 1) * 8;
                            if (D == 128) {
                                const uint4 c = *reinterpret_cast<const uint4*>(vst + row * 128 + ((g8 ^ (row & 7)) << 4));
                                v[y][0] = c.x; v[y][1] = c.y; v[y][D / 64] = c.z; v[y][D / 32 - 1] = c.w;
                            } else {
                                const uint2 c = *reinterpret_cast<const uint2*>(vst + row * 64 + (((g8 >> 1) ^ ((row >> 1) & 3)) << 4) + (g8 & 1) * 8);
                                v[y][0] = c.x; v[y][1] = c.y;
                            }
                        }
#pragma unroll
                        for (int c = 0; c < D / 32; ++c)
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                const uint32_t sel = y ? 0x7362 : 0x5140;
                                uint32_t vf[4];
                                codes_to_f16x4(__byte_perm(v[0][c], v[1][c], sel), vf[0], vf[1]);
                                codes_to_f16x4(__byte_perm(v[2][c], v[3][c], sel), vf[2], vf[3]);
#pragma unroll
                                for (int r = 0; r < kGroups; ++r) mma_f16_16816(o[r][2 * c + y], vf, pf[r][2 * s], pf[r][2 * s + 1]);
                            }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm.empty[st]);
            if (++st == kStages) { st = 0; ph ^= 1; }
        }

        // ---- the warps' states into one, always in the same order: with 8 heads two halves at a time, (0 and 1) + (2 and 3)
        float c[kGroups];
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            if (t4 == 0) *reinterpret_cast<float4*>(sm.stat[warp][r * 8 + g8]) = make_float4(m[r], l[r], mv[r], 0.f);
        }
        // warps that had a key of the part (the first ones, where it is one tile)
        const int live = w.end - w.tile > 1 ? 4 : paged_pieces(n - w.line.tile_at(n, w.tiles, w.tile) * kTile, kTile, kWarpKeys);
        consumer_sync();
#pragma unroll
        for (int r = 0; r < kGroups; ++r) {
            float all = -INFINITY;
#pragma unroll
            for (int y = 0; y < 4; ++y) all = fmaxf(all, sm.stat[y][r * 8 + g8][2]);
            c[r] = mv[r] == -INFINITY ? 0.f : fast_exp2(mv[r] - all);
        }
        constexpr int kHalves = kGroups == 1 ? 2 : 1;
#pragma unroll 1
        for (int y = 0; y < live; y += kHalves) {
            if (warp >= y && warp < y + kHalves && warp < live) {
#pragma unroll
                for (int r = 0; r < kGroups; ++r) {
                    const float c0 = __shfl_sync(0xffffffffu, c[r], 8 * t4), c1 = __shfl_sync(0xffffffffu, c[r], 8 * t4 + 4);
                    float* d0 = sm.red[(kGroups == 1 ? warp & 1 : r) * 8 + 2 * t4];
                    float* d1 = d0 + (D + 4);
#pragma unroll
                    for (int i = 0; i < kMTiles; ++i) {
                        if (kE4m3) {
                            const int at = (g8 * (D / 8) + 2 * i) ^ ((g8 << 1) & (D / 8 - 1));
                            const float2 a0 = y ? *reinterpret_cast<float2*>(d0 + at) : make_float2(0.f, 0.f), a1 = y ? *reinterpret_cast<float2*>(d1 + at) : make_float2(0.f, 0.f);
                            *reinterpret_cast<float2*>(d0 + at) = make_float2(a0.x + o[r][i][0] * c0, a0.y + o[r][i][2] * c0);
                            *reinterpret_cast<float2*>(d1 + at) = make_float2(a1.x + o[r][i][1] * c1, a1.y + o[r][i][3] * c1);
                        } else {
                            const int at = i * 16 + g8;
                            d0[at] = (y ? d0[at] : 0.f) + o[r][i][0] * c0;
                            d1[at] = (y ? d1[at] : 0.f) + o[r][i][1] * c1;
                            d0[at + 8] = (y ? d0[at + 8] : 0.f) + o[r][i][2] * c0;
                            d1[at + 8] = (y ? d1[at + 8] : 0.f) + o[r][i][3] * c1;
                        }
                    }
                }
            }
            consumer_sync();
        }
        const bool whole = w.tile == 0 && w.end == w.tiles;
        const bool bad = *(volatile int*)&sm.bad[part & 3] == part + 1;
        const int slot = w.tile > 0 ? 0 : 1;                  // a part that goes on from an earlier run, one that begins here
        float* dst = a.partial + ((size_t)(blockIdx.x * 2 + slot) * a.G) * kRowF;
        for (int idx = tid; idx < a.G * (D / 2); idx += 128) {
            const int row = idx / (D / 2), d = (idx % (D / 2)) * 2;
            float am = -INFINITY, amv = -INFINITY, al = 0.f;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                am = fmaxf(am, sm.stat[y][row][0]);
                amv = fmaxf(amv, sm.stat[y][row][2]);
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float my = sm.stat[y][row][0], ly = sm.stat[y][row][1];
                if (ly != 0.f) al += ly * fast_exp2(my == -INFINITY ? 0.f : my - am);
            }
            const int at = kE4m3 ? d ^ (((d / (D / 8)) << 1) & (D / 8 - 1)) : d;
            float2 v = *reinterpret_cast<const float2*>(&sm.red[row][at]);
            if (kGroups == 1 && live > 1) {
                const float2 u = *reinterpret_cast<const float2*>(&sm.red[8 + row][at]);
                v = make_float2(v.x + u.x, v.y + u.y);
            }
            if (whole) {
                // (every score -inf: the maxima are, sum and outputs are zeros, or none where a value is none)
                const float fo = kE4m3 && am != -INFINITY ? exp2f(amv - am - kPagedBias) : 1.f, inv = al != 0.f ? 1.f / al : 0.f;
                const size_t out_at = (size_t)w.b * a.Hq + w.gk * a.G + row;
                *reinterpret_cast<uint32_t*>(a.out + out_at * D + d) = bad ? 0u : pack_bf16x2(v.x * inv * fo, v.y * inv * fo);
                if (d == 0 && a.lse != nullptr) a.lse[out_at] = bad ? -INFINITY : (am + log2f(al)) * 0.6931471805599453f;
            } else {
                float* r = dst + row * kRowF;
                *reinterpret_cast<float2*>(r + 4 + d) = v;
                if (d == 0) *reinterpret_cast<float4*>(r) = make_float4(am, bad ? -1.f : al, kE4m3 ? amv - kPagedBias : am, 0.f);
            }
        }
        consumer_sync();                                      // the statistics and the sums may be overwritten
    }
    // rows of sequences that are not there, or whose length is out of range
    for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
        const int n = a.kv_len[b];
        if (n > 0 && w.line.in_range(n)) continue;
        for (int i = tid; i < a.Hq * (D / 8); i += 128) *reinterpret_cast<uint4*>(a.out + (size_t)b * a.Hq * D + i * 8) = make_uint4(0u, 0u, 0u, 0u);
        if (a.lse != nullptr)
            for (int i = tid; i < a.Hq; i += 128) a.lse[(size_t)b * a.Hq + i] = -INFINITY;
        if (tid == 0 && n != 0 && a.status != nullptr) atomicExch(a.status, 1);
    }
    if (tid == 0 && sm.abort_flag && a.status != nullptr) atomicExch(a.status, 6);
    tc::settle_after_abort(abort_flag);                       // (the producer has stopped, or finds the flag at its next wait)
}

// Joins what is cut.  Many (sequence, kv head)s: grid (runs - 1), CTA i joins the one that is cut by the end of run i and has its first tile in
// that run; there are as many as cuts at most, however large the batch (a CTA for every row of 256 sequences: 55 us instead of 21 for the
// step).  Few, of many parts each: grid (batch * Hkv, G), a CTA a row.  The kernel before lets this one in when kv_len is
// there: what comes before the wait runs beside it.  Up to 16 parts, a warp joins a row by itself; more are shared out over the CTA's warps.
// Statistics and values of the first parts are loaded together, one round trip to the L2.
constexpr int kJoinThreads = 256;
constexpr int kJoinBlocks = 4, kJoinWarpAhead = 8;

template <int D, bool kE4m3, bool kFew, bool kWin>
__global__ void __launch_bounds__(kJoinThreads, kFew ? 2 : kJoinBlocks) paged_join_kernel(PageGeom p, PagedCall a, int n_ctas) {
    constexpr int kTile = paged_tile(kE4m3), kLanes = D / 4, kShares = kJoinThreads / kLanes, kRowF = paged_row_floats(D), kAhead = kFew ? 8 : 4;
    __shared__ float weight[kPagedCtas];
    __shared__ float4 red[kShares / 2][kLanes];
    __shared__ float tops[8][2], sums[8];
    __shared__ int bads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    RunWalk<kTile, kWin> w;
    w.line.p = &p;
    w.line.a = &a;
    w.line.kv_len = a.kv_len;
    w.line.batch = a.batch;
    w.line.lane = lane;
    const long long total = w.line.total();
    const int n_runs = run_count(total, n_ctas);
    int run = blockIdx.x, n = 0;                              // first of the n runs that hold its tiles; n < 2: not this CTA's
    if (kFew) {
        const int b = blockIdx.x / p.Hkv, gk = blockIdx.x - b * p.Hkv;
        if (w.seek_sequence(b, gk, total)) {
            run = run_of(total, n_runs, w.place + paged_part_cost(kTile));
            n = run_of(total, n_runs, w.place + paged_part_cost(kTile) + w.tiles - 1) - run + 1;
        }
    } else if (run + 1 < n_runs) {
        const long long cut = run_begin(total, n_runs, run + 1);
        w.seek(cut, total);
        const long long first = w.place + paged_part_cost(kTile);
        if (first < cut && run_of(total, n_runs, first) == run) n = run_of(total, n_runs, first + w.tiles - 1) - run + 1;
    }
    launch_dependents();
    wait_for_previous_kernel();
    if (n < 2) return;                                        // (finished where it was computed)
    // part i lies with run + i: the first in its slot 1, the others in slot 0
    const size_t step = (size_t)2 * a.G * kRowF;
    const float* parts = a.partial + (size_t)run * step;
    auto part = [&](int i, int row) -> const float* { return parts + i * step + ((i == 0 ? a.G : 0) + row) * kRowF; };
    auto add = [](float4& acc, const float4& y, float f) {
        acc.x = fmaf(y.x, f, acc.x);
        acc.y = fmaf(y.y, f, acc.y);
        acc.z = fmaf(y.z, f, acc.z);
        acc.w = fmaf(y.w, f, acc.w);
    };
    auto finish = [&](int row, int d4, const float4& acc, float m, float mv, float l, bool bad) {
        const size_t at = (size_t)w.b * a.Hq + w.gk * a.G + row;
        const float f = (kE4m3 && m != -INFINITY ? exp2f(mv - m) : 1.f) * (l != 0.f ? 1.f / l : 0.f);   // (every score -inf: as in a whole part)
        *reinterpret_cast<uint2*>(a.out + at * D + 4 * d4) = bad ? make_uint2(0u, 0u) : make_uint2(pack_bf16x2(acc.x * f, acc.y * f), pack_bf16x2(acc.z * f, acc.w * f));
        if (d4 == 0 && a.lse != nullptr) a.lse[at] = bad ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    };
    if (n <= 16) {
        constexpr int kPer = 32 / kLanes;                     // parts that a warp takes at a time
        const int d4 = lane % kLanes, sub = lane / kLanes;
        for (int row = blockIdx.y + warp * gridDim.y; row < a.G; row += 8 * gridDim.y) {
            float4 st = make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
            if (lane < n) st = *reinterpret_cast<const float4*>(part(lane, row));
            float4 v[kJoinWarpAhead];
#pragma unroll
            for (int i = 0; i < kJoinWarpAhead; ++i) {
                const int x = sub + i * kPer;
                v[i] = x < n ? *reinterpret_cast<const float4*>(part(x, row) + 4 + 4 * d4) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float m = st.x, mv = st.z;
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, x));
            }
            float l = st.y != 0.f && lane < 16 ? st.y * fast_exp2(st.x == -INFINITY ? 0.f : st.x - m) : 0.f;
            const float wt = st.z == -INFINITY ? 0.f : fast_exp2(st.z - mv);
            const bool bad = __any_sync(0xffffffffu, st.y == -1.f);
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 16 / kPer; ++i) {
                const int x = sub + i * kPer;
                const float f = __shfl_sync(0xffffffffu, wt, x & 15);
                if (x < n) add(acc, i < kJoinWarpAhead ? v[i < kJoinWarpAhead ? i : 0] : *reinterpret_cast<const float4*>(part(x, row) + 4 + 4 * d4), f);
            }
            if (kPer == 2) {
                const float4 y = make_float4(__shfl_xor_sync(0xffffffffu, acc.x, 16), __shfl_xor_sync(0xffffffffu, acc.y, 16), __shfl_xor_sync(0xffffffffu, acc.z, 16),
                                             __shfl_xor_sync(0xffffffffu, acc.w, 16));
                add(acc, y, 1.f);
            }
            // (lanes 16 .. 31 hold no statistics of theirs: the first lane's)
            m = __shfl_sync(0xffffffffu, m, 0);
            mv = __shfl_sync(0xffffffffu, mv, 0);
            l = __shfl_sync(0xffffffffu, l, 0);
            if (lane < kLanes) finish(row, d4, acc, m, mv, l, bad);
        }
        return;
    }
    const int d4 = tid % kLanes, share = tid / kLanes;
    for (int row = blockIdx.y; row < a.G; row += gridDim.y) {
        __syncthreads();
        if (tid == 0) bads = 0;
        float4 st = make_float4(-INFINITY, 0.f, -INFINITY, 0.f), st2 = st;    // of parts tid and tid + 256
        if (tid < n) st = *reinterpret_cast<const float4*>(part(tid, row));
        if (tid + kJoinThreads < n) st2 = *reinterpret_cast<const float4*>(part(tid + kJoinThreads, row));
        float4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int x = share + i * kShares;
            v[i] = x < n ? *reinterpret_cast<const float4*>(part(x, row) + 4 + 4 * d4) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float m = fmaxf(st.x, st2.x), mv = fmaxf(st.z, st2.z);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) {
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
            mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, x));
        }
        if (lane == 0) {
            tops[warp][0] = m;
            tops[warp][1] = mv;
        }
        __syncthreads();
        if (st.y == -1.f || st2.y == -1.f) bads = 1;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            m = fmaxf(m, tops[x][0]);
            mv = fmaxf(mv, tops[x][1]);
        }
        float l = 0.f;
        if (st.y != 0.f) l += st.y * fast_exp2(st.x == -INFINITY ? 0.f : st.x - m);
        if (st2.y != 0.f) l += st2.y * fast_exp2(st2.x == -INFINITY ? 0.f : st2.x - m);
        if (tid < n) weight[tid] = st.z == -INFINITY ? 0.f : fast_exp2(st.z - mv);
        if (tid + kJoinThreads < n) weight[tid + kJoinThreads] = st2.z == -INFINITY ? 0.f : fast_exp2(st2.z - mv);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
        if (lane == 0) sums[warp] = l;
        __syncthreads();
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (share + i * kShares < n) add(acc, v[i], weight[share + i * kShares]);
#pragma unroll 4
        for (int x = share + kAhead * kShares; x < n; x += kShares) add(acc, *reinterpret_cast<const float4*>(part(x, row) + 4 + 4 * d4), weight[x]);
        if (share >= kShares / 2) red[share - kShares / 2][d4] = acc;
        __syncthreads();
        if (share < kShares / 2) {
            add(acc, red[share][d4], 1.f);
            red[share][d4] = acc;
        }
        __syncthreads();
        if (tid < kLanes) {
            for (int x = 1; x < kShares / 2; ++x) add(acc, red[x][d4], 1.f);
            l = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) l += sums[x];
            finish(row, d4, acc, m, mv, l, bads != 0);
        }
    }
}

}  // namespace adaspark
