// Causal attention over whole prompts, packed one behind the other, on the 5th-generation tensor cores.
//
//   o_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = 2^(scale_log2 q_i.k_j - m_i),  j <= n_k - n_q + i
//
// One pass over the keys with a reference m_i and running sum, scores and weights in tensor memory alone.  The reference is the largest of the
// row's first 128 scores (itself, so that its weight, 1, is not rounded: with the next whole number the outputs were 1.2 times as far from 64 bits)
// and moves only when the weights of 64 keys sum up to more than 2^40: weights, sums and outputs are
// floating-point numbers, whose relative precision does not depend on it, and 2^40 is far from where they end.  So no step but the first
// takes a maximum (9 % of the time of a long prompt).  (A row whose first scores are all -inf has the lowest float as its reference, so that
// the first step with any other score moves it.)  Where they sum up to 2^100 and more, infinity included, that half step's scores, which
// the weights have overwritten, are computed once more by the threads themselves.  A reference moves by a
// whole number: the weights that stand are multiplied by a power of two, which rounds nothing (a second rounding took outputs of two keys
// near 2^100 past the bound of one).
//
// Work is dealt out in tiles of 256 rows, a CTA pair (cta_group::2) each: the rows are (token, head of the group) pairs, 128 / G tokens
// per CTA, so that K and V are read once for all heads of a group, a sequence of a few tokens fills rows that it would leave empty head by
// head, and the diagonal wastes little (256 rows of a group of 7 are 36 tokens: 2 % of the scores of 8192 tokens lie above it, 256 tokens of
// one head: 4.7 %).
//
// Roles of a CTA (640 threads), coupled by barriers alone, so that set-up, loads and first scores of the next tile overlap the end of
// the present one:
//   warps 0-15  softmax, two teams of two warpgroups that take the steps of 128 keys in turn; a row's keys are shared by two threads
//   warp  16    TMA producer of K; masked steps: looks for values that are no numbers (below)
//   warp  17    MMA issuer (CTA 0): S = Q K^T, O += P V (P in TMEM, V with its rows along d); CTA 1: passes on that its Q is there
//   warp  18    TMA producer of V
//   warp  19    planner: the next tiles and their Q
// TMEM (512 columns): three score tiles of 128 columns, each with the weights (bf16 pairs) over the first 32 of either half, and O.  The
// waits are those of the prefill kernel (attn_prefill_tc.cuh): the issuer never waits for a tile that it has not begun while a product of
// an earlier one is still to be issued.  A step takes 0.9 to 1.0 us (head_dim 64: 0.73) and a tile about 2 us beside its steps, fitted over calls of
// 9 to 33 tiles a pair with 1.4 to 18 steps each: 512 + 512 cycles of a step's 1800 at full clock are products (head_dim 64: half as many of
// 1400), the others the softmax's share of the chain scores -> weights -> product, which three score tiles and two teams work on at a time.
// (Three warpgroups with a row each per thread: 10 % longer.)
//
// Tiles are dealt longest first and back and forth over the pairs of CTAs.  Every planner works the order out for itself from cu_q and
// cu_k, level by level of the number of steps: no list in memory, no counter, one launch, and nothing to be cleared before it.
//
// A weight of zero does not hide a value that is no number: 0 * inf is one too.  Steps in which a row of the tile does not see a key
// (the last one to three of a tile) therefore go over V in shared memory before the tensor core reads it: what is infinite or no
// number is replaced by zero, and if it belongs to the sequence, the rows that do see it get it added at the end.
#pragma once
#include <type_traits>

#include "tc_common.cuh"

namespace adaspark {

constexpr int kPromptTeams = 2;                               // softmax teams, of two warpgroups each
constexpr int kPromptThreads = (2 * kPromptTeams + 1) * 128;
constexpr int kPromptPlans = 4;                               // tiles planned at once
constexpr int kPromptBufs = 3;                                // score tiles in TMEM
constexpr int kPromptRefSlots = 4;
constexpr float kPromptBig = 0x1p40f;                         // a reference moves when a half step's weights sum up to more
constexpr float kPromptLowest = -3.402823466e38f;             // a reference below any score
// A planner that walks past levels of a long prompt looks at every sequence for each: 16 ns a sequence and level, 150 levels and more from one of
// a pair's tiles to its next (where a level has one tile).  Waits for its plans last so much longer.
constexpr uint64_t kPromptPlanNs = 10000;                     // a sequence
constexpr int kPromptOddSlots = 8;                            // more than tiles whose V can be under way at once (a step each)
__host__ __device__ constexpr int prompt_k_stages(int D) { return D == 64 ? 6 : 3; }   // steps whose K, V are under way
__host__ __device__ constexpr int prompt_v_stages(int D) { return D == 64 ? 6 : 3; }
static_assert(prompt_v_stages(64) + 1 < kPromptOddSlots, "a slot is not written again before it has been read");

// q.k of two rows in global memory
template <int D>
__device__ __noinline__ float prompt_dot(const __nv_bfloat16* q, const __nv_bfloat16* key) {
    float sum = 0.f;
#pragma unroll 1
    for (int c = 0; c < D; c += 8) {
        const uint4 a = *reinterpret_cast<const uint4*>(q + c), b = *reinterpret_cast<const uint4*>(key + c);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sum = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), sum));
    }
    return sum;
}

// What one call works on.
struct PromptGeom {
    const int32_t *cu_q, *cu_k;
    int batch, n_q, n_k;
    int Hq, Hkv, G;
    int T;                      // tokens of a CTA: 128 / G
    FastDiv div_w, div_g, div_kv;   // by 2 T, G, Hkv
    float scale_log2;
    const __nv_bfloat16 *q, *k, *v; // for scores that leave the range of a step's reference, values that are no numbers
    long long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs;
};

struct PromptTile {
    int q0, n_tok;              // this CTA's first row of q and its tokens (the pair's first CTA may have all)
    int k0;                     // first key row of the sequence
    int last0;                  // last key that this CTA's first token sees (-1 and less: none)
    int gk;
    int n_steps, first_masked;  // steps of 128 keys; from this one on rows are masked
    int part;                   // number of the part of a tile whose keys are cut, -1: a whole tile
};

// A sequence as a planner sees it; one that leaves the tensors has no tiles.
struct PromptSeq {
    int q0, k0, nq, nk, off, nt;
    __device__ __forceinline__ bool load(const PromptGeom& g, int b) {
        const int a0 = g.cu_q[b], a1 = g.cu_q[b + 1], b0 = g.cu_k[b], b1 = g.cu_k[b + 1];
        const bool valid = 0 <= a0 && a0 <= a1 && a1 <= g.n_q && 0 <= b0 && b0 <= b1 && b1 <= g.n_k;
        q0 = a0;
        k0 = b0;
        nq = valid ? a1 - a0 : 0;
        nk = valid ? b1 - b0 : 0;
        off = nk - nq;
        nt = nq > 0 ? g.div_w.div(nq + 2 * g.T - 1) : 0;
        return valid;
    }
    // tiles whose last row sees at most x keys
    __device__ __forceinline__ int tiles_up_to(const PromptGeom& g, int x) const {
        return x >= nk ? nt : x <= off ? 0 : min(g.div_w.div(x - off), nt);
    }
};

// Few tiles over many keys (a turn that continues a long conversation) would leave most pairs of CTAs without work: a tile whose steps are
// 1.5 times and more what a pair has to do on average (`unit`, no less than kPromptMinUnit) is cut into parts of about that.  Each part
// leaves its outputs, references and sums, and prompt_join_kernel puts them together.  There are at most 4/3 as many as pairs.
constexpr int kPromptPairs = 74, kPromptMinUnit = 8;
constexpr int kPromptParts = 100;
// Rows of the cut tiles' parts: outputs [part][CTA][128][D], then (reference, sum) [part][CTA][128]
__host__ __device__ constexpr size_t prompt_partial_bytes(int D) { return (size_t)kPromptParts * 256 * (D + 2) * sizeof(float); }
// Could a call have tiles to cut?  (If not, there is nothing to join either: 36.1 against 37.9 us for 4301 tokens in 5 prompts, 16 heads of 64.)  More
// tiles than 4 a pair: no one is long enough to matter.  Whole prompts: the n / W tiles of a prompt of n tokens, W to a tile, average half
// of its n / 128 steps; that is 1.5 times what a pair has to do only up to n = 99 W / Hkv, and no tile of less than 12 steps is cut.
inline bool prompt_may_cut(long long most_tiles, int n_k, bool whole, int W, int Hkv) {
    return most_tiles <= 4 * kPromptPairs && n_k > 128 * 3 * kPromptMinUnit / 2 && (!whole || W > 16 * Hkv);
}

// The order of the items (tiles, or parts of them): levels from many steps to few, sequences in order, tiles, kv heads, parts.  A warp walks
// it, with 32 sequences in its lanes.  Parts come first: an item's number is its part's.
struct PromptWalk {
    int level, unit;                                          // unit 0: nothing is cut
    int below;                                                // most steps of a tile of fewer than `level`, among the sequences seen so far
    int chunk, base;                                          // number of the first item of (level, chunk)
    int held;                                                 // chunk of `mine`, this lane's sequence
    PromptSeq mine;
    // what find() found
    PromptSeq seq;
    int tile, gk, part, parts;

    // false: a sequence leaves the tensors
    __device__ __forceinline__ bool begin(const PromptGeom& g, bool cut, int n_pairs, int lane) {
        bool fine = true;
        long long steps = 0;                                  // at least as many as there are
        level = chunk = base = below = 0;
        for (held = 0; held * 32 < g.batch; ++held) {
            mine.nt = 0;
            if (held * 32 + lane < g.batch) {
                fine = mine.load(g, held * 32 + lane) && fine;
                if (mine.nt > 0) {
                    level = max(level, max(1, (mine.nk + 127) >> 7));
                    steps += (long long)mine.nt * (max(mine.off, 0) / 128 + 2) + (long long)g.T * mine.nt * (mine.nt + 1) / 128;
                }
            }
        }
        --held;
        level = (int)__reduce_max_sync(0xffffffffu, (unsigned)level);
        unit = 0;
        if (cut) {
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, x);
            unit = (int)max((steps * g.Hkv + n_pairs - 1) / n_pairs, (long long)kPromptMinUnit);
        }
        return fine;
    }
    __device__ __forceinline__ int parts_of(int steps) const { return unit > 0 ? max((2 * steps + unit) / (2 * unit), 1) : 1; }
    // item `number`, which is no smaller than the one before; false: there are not so many (of cut tiles)
    __device__ __forceinline__ bool find(const PromptGeom& g, int number, int lane, bool cut_only = false) {
        while (level > 0) {
            parts = parts_of(level);
            if (cut_only && parts == 1) return false;
            if (held != chunk) {                              // (up to 32 sequences: never)
                held = chunk;
                mine.nt = 0;
                if (chunk * 32 + lane < g.batch) mine.load(g, chunk * 32 + lane);
            }
            int first = 0, n = 0;
            if (mine.nt > 0) {
                first = level == 1 ? 0 : mine.tiles_up_to(g, 128 * (level - 1));
                n = (mine.tiles_up_to(g, 128 * level) - first) * g.Hkv * parts;
            }
            int upto = n;
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, upto, x);
                if (lane >= x) upto += y;
            }
            const int total = __shfl_sync(0xffffffffu, upto, 31);
            if (number < base + total) {
                const int who = __ffs(__ballot_sync(0xffffffffu, base + upto > number)) - 1;
                int i = __shfl_sync(0xffffffffu, number - base - (upto - n), who);
                seq.q0 = __shfl_sync(0xffffffffu, mine.q0, who);
                seq.k0 = __shfl_sync(0xffffffffu, mine.k0, who);
                seq.nq = __shfl_sync(0xffffffffu, mine.nq, who);
                seq.nk = __shfl_sync(0xffffffffu, mine.nk, who);
                seq.off = __shfl_sync(0xffffffffu, mine.off, who);
                part = i % parts;
                i /= parts;
                g.div_kv.divmod(i, tile, gk);
                tile += __shfl_sync(0xffffffffu, first, who);
                return true;
            }
            base += total;
            // the next level is that of the longest tile left: levels without a tile are passed over
            if (first > 0) below = max(below, max((min(mine.off + 2 * g.T * first, mine.nk) + 127) >> 7, 1));
            if (++chunk * 32 >= g.batch) {
                chunk = 0;
                level = min((int)__reduce_max_sync(0xffffffffu, (unsigned)below), level - 1);   // (down in any case: the walk ends)
                below = 0;
            }
        }
        return false;
    }
    // first token of CTA `rank` of the tile, and how many it has
    __device__ __forceinline__ int first_token(const PromptGeom& g, int rank) const { return (2 * tile + rank) * g.T; }
    __device__ __forceinline__ int tokens(const PromptGeom& g, int rank) const { return min(max(seq.nq - first_token(g, rank), 0), g.T); }
};

template <int D>
struct PromptSmem {
    __nv_bfloat16 q[2][D / 64][128][64];                      // [tile & 1][d panel][row][64 d]
    __nv_bfloat16 k[prompt_k_stages(D)][64 * D];              // [d panel][this CTA's 64 keys][64 d]
    __nv_bfloat16 v[prompt_v_stages(D)][64 * D];              // [128 keys][this CTA's half of d]
    unsigned char out[128][2 * D + 16];
    float ref[kPromptRefSlots][128], first_ref[2][128];      // reference of a row after a step, after the first 128 keys of a tile
    float part_l[2][2][128], part_m[2][2][128];             // sums and reference of the team that does not finish a tile, by half
    float other_l[kPromptTeams][2][128], other_ref[kPromptTeams][2][128];   // between the halves of a row
    uint64_t q_full[2], q_peer[2], q_empty[2], k_full[prompt_k_stages(D)], k_empty[prompt_k_stages(D)], v_full[prompt_v_stages(D)], v_empty[prompt_v_stages(D)];
    uint64_t v_raw[prompt_v_stages(D)], s_full[kPromptBufs], p_full[kPromptBufs], ref_done[kPromptRefSlots][4], first_done[2][4], o_full, o_free;
    uint64_t plan_full[kPromptPlans], plan_empty[kPromptPlans], part_full[2], part_free[2], out_free;
    PromptTile tile[kPromptPlans];
    int odd_tile[kPromptOddSlots];                            // number + 1 of a tile with masked values that are no numbers
    uint32_t tmem_base;
    int abort_flag;
};

template <int D>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPromptThreads, 1) attn_prompt_kernel(
    PromptGeom g, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    __nv_bfloat16* out, float* lse, float* partial, int32_t* status) {
    extern __shared__ unsigned char prompt_smem_raw[];
    PromptSmem<D>& sm = *reinterpret_cast<PromptSmem<D>*>((reinterpret_cast<uintptr_t>(prompt_smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kPanels = D / 64, kQKSteps = D / 16, kKStages = prompt_k_stages(D), kVStages = prompt_v_stages(D);
    constexpr uint32_t kIdescS = tc::make_idesc_bf16(256, 128);
    constexpr uint32_t kIdescO = tc::make_idesc_bf16(256, D) | (1u << 16);   // B = V: rows along N
    constexpr uint32_t kTileBytes = 64 * D * 2;               // a CTA's share of the K or V of a step
    constexpr int kVRow = D;                                  // bytes of a key in a CTA's share of V (half of d)
    constexpr int kKWarp = kPromptTeams * 8, kMmaWarp = kKWarp + 1, kVWarp = kKWarp + 2, kPlanWarp = kKWarp + 3;
    constexpr uint32_t kOCol = kPromptBufs * 128;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x & 1u), n_pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1);

    // ---------------------------------------------------------------- set-up
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&sm.q_full[i], 1);
            tc::mbar_init(&sm.q_peer[i], 1);
            tc::mbar_init(&sm.q_empty[i], 1);
            tc::mbar_init(&sm.part_full[i], 8);
            tc::mbar_init(&sm.part_free[i], 8);
        }
        for (int i = 0; i < kPromptPlans; ++i) {
            tc::mbar_init(&sm.plan_full[i], 1);
            tc::mbar_init(&sm.plan_empty[i], 4 + kPromptTeams * 8);
        }
        for (int i = 0; i < kKStages; ++i) {
            tc::mbar_init(&sm.k_full[i], 1);
            tc::mbar_init(&sm.k_empty[i], 1);
        }
        for (int i = 0; i < kVStages; ++i) {
            tc::mbar_init(&sm.v_full[i], 2);                  // of both CTAs
            tc::mbar_init(&sm.v_raw[i], 1);
            tc::mbar_init(&sm.v_empty[i], 1);
        }
        for (int i = 0; i < kPromptBufs; ++i) {
            tc::mbar_init(&sm.s_full[i], 1);
            tc::mbar_init(&sm.p_full[i], 16);
        }
        for (int i = 0; i < kPromptRefSlots; ++i)
            for (int w = 0; w < 4; ++w) tc::mbar_init(&sm.ref_done[i][w], 1);
        for (int i = 0; i < 2; ++i)
            for (int w = 0; w < 4; ++w) tc::mbar_init(&sm.first_done[i][w], 1);
        for (int i = 0; i < kPromptOddSlots; ++i) sm.odd_tile[i] = 0;
        tc::mbar_init(&sm.o_full, 1);
        tc::mbar_init(&sm.o_free, 16);
        tc::mbar_init(&sm.out_free, 8);
        sm.abort_flag = 0;
        tc::fence_barrier_init();
        tc::prefetch_tensormap(&tmQ);
        tc::prefetch_tensormap(&tmK);
        tc::prefetch_tensormap(&tmV);
    }
    __syncwarp();
    wait_for_previous_kernel();
    launch_dependents();                                      // (after the wait: the next kernel reads cu_q and cu_k before its own)
    // (not before the wait: a CTA of the previous kernel that is still to allocate would wait for this one)
    if (warp == kMmaWarp) tc::tmem_alloc_pair<512>(&sm.tmem_base);
    tc::tc_fence_before_sync();
    cluster_sync();
    tc::tc_fence_after_sync();
    const uint32_t tbase = sm.tmem_base;
    volatile int* abort_flag = &sm.abort_flag;
    const uint64_t plan_limit = tc::kWaitLimitNs + (uint64_t)g.batch * kPromptPlanNs;

    if (warp == kPlanWarp) {
        // ------------------------------------------------------------ planner
        PromptWalk w;
        if (!w.begin(g, partial != nullptr, n_pairs, lane) && blockIdx.x == 0 && status != nullptr) atomicExch(status, 1);
        for (int k = 0;; ++k) {
            const int slot = k % kPromptPlans, qs = k & 1;
            if (!tc::mbar_wait(&sm.plan_empty[slot], ((k / kPromptPlans) & 1) ^ 1u, abort_flag)) break;
            const int number = k * n_pairs + ((k & 1) ? n_pairs - 1 - pair : pair);
            const bool found = w.find(g, number, lane);
            PromptTile t;
            if (found) {
                const int tok = w.first_token(g, rank), begin = w.part * w.level / w.parts;
                t.q0 = w.seq.q0 + tok;
                t.n_tok = w.tokens(g, rank);
                t.k0 = w.seq.k0 + begin * 128;                // a part counts its keys from its own first one
                t.last0 = w.seq.off + tok - begin * 128;
                t.gk = w.gk;
                t.n_steps = (w.part + 1) * w.level / w.parts - begin;
                t.first_masked = max((max(w.seq.off + w.first_token(g, 0) + 1, 0) >> 7) - begin, 0);
                t.part = w.parts > 1 ? number : -1;
                if (lane == 0) sm.tile[slot] = t;
            }
            if (!found) {
                if (lane == 0) {
                    sm.tile[slot].n_steps = 0;                // no more
                    tc::mbar_arrive(&sm.plan_full[slot]);
                }
                break;
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm.plan_full[slot]);
            if (!tc::mbar_wait(&sm.q_empty[qs], ((k >> 1) & 1) ^ 1, abort_flag)) break;
            __syncwarp();
            if (lane == 0) {
                // rows (token, head of the group); tokens behind the tensor read zeros, those of the next sequence are not stored
                tc::mbar_arrive_expect_tx(&sm.q_full[qs], (uint32_t)(g.T * g.G) * D * 2);
                for (int p = 0; p < kPanels; ++p) tc::tma_load_3d(&sm.q[qs][p][0][0], &tmQ, p * 64, t.gk * g.G, t.q0, &sm.q_full[qs]);
            }
            __syncwarp();
        }
    } else if (warp == kKWarp) {
        // ------------------------------------------------------------ K: CTA r fetches the keys r * 64 .. of a step.  And masked steps:
        // values that are no numbers.  Whichever is ready, so that neither waits for the other.
        const uint32_t bar0 = cluster_address(sm.k_full, 0), v_bar0 = cluster_address(sm.v_full, 0);
        const uint32_t odd0 = cluster_address(sm.odd_tile, 0), odd1 = cluster_address(sm.odd_tile, 1);
        auto ready = [&](uint64_t* bar, uint32_t phase) -> bool { return __all_sync(0xffffffffu, tc::mbar_test(bar, phase)); };
        struct { int k = 0, j = 0, n = 0, st = 0; bool done = false; } kp, look;      // tile, step, steps of the tile (0: not begun), stage
        int k_ph = 1, row0 = 0, gk = 0, first_masked = 0;
        uint32_t raw_phases = 0, idle = 0;                    // (of v_raw, a bit each)
        uint64_t since = 0;
        while (!kp.done || !look.done) {
            bool moved = false;
            if (!kp.done) {
                const int slot = kp.k % kPromptPlans;
                if (kp.n == 0 && ready(&sm.plan_full[slot], (kp.k / kPromptPlans) & 1)) {
                    kp.n = sm.tile[slot].n_steps;
                    row0 = sm.tile[slot].k0 + rank * 64;
                    gk = sm.tile[slot].gk;
                    kp.done = kp.n == 0;
                    moved = true;
                }
                if (kp.n > 0 && ready(&sm.k_empty[kp.st], k_ph)) {
                    if (tc::elect_one()) {
                        if (rank == 0) tc::mbar_arrive_expect_tx(&sm.k_full[kp.st], 2 * kTileBytes);
                        for (int p = 0; p < kPanels; ++p)
                            tc::tma_load_3d_pair(&sm.k[kp.st][p * 64 * 64], &tmK, p * 64, gk, row0 + kp.j * 128, bar0 + kp.st * 8);
                    }
                    __syncwarp();
                    if (++kp.st == kKStages) { kp.st = 0; k_ph ^= 1; }
                    if (++kp.j == kp.n) {
                        if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
                        kp.j = kp.n = 0;
                        ++kp.k;
                    }
                    moved = true;
                }
            }
            if (!look.done) {
                const int slot = look.k % kPromptPlans;
                if (look.n == 0 && ready(&sm.plan_full[slot], (look.k / kPromptPlans) & 1)) {
                    look.n = sm.tile[slot].n_steps;
                    first_masked = sm.tile[slot].first_masked;
                    look.done = look.n == 0;
                    look.j = min(first_masked, look.n);
                    look.st = (look.st + look.j) % kVStages;
                    moved = true;
                }
                if (look.n > 0 && look.j < look.n && ready(&sm.v_raw[look.st], (raw_phases >> look.st) & 1)) {
                    raw_phases ^= 1u << look.st;
                    // exponents of all ones: adding 0x80 to (x & 0x7f80) carries into bit 15
                    uint4* chunks = reinterpret_cast<uint4*>(&sm.v[look.st][0]);
                    uint32_t any = 0;
#pragma unroll 8
                    for (int i = lane; i < (int)kTileBytes / 16; i += 32) {
                        const uint4 x = chunks[i];
                        any |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u) | ((x.z & 0x7f807f80u) + 0x00800080u) |
                               ((x.w & 0x7f807f80u) + 0x00800080u);
                    }
                    if (__any_sync(0xffffffffu, (any & 0x80008000u) != 0u)) {
                        for (int i = lane; i < (int)kTileBytes / 16; i += 32) {
                            uint32_t x[4] = {chunks[i].x, chunks[i].y, chunks[i].z, chunks[i].w};
                            for (int e = 0; e < 4; ++e) {
                                if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
                                if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
                            }
                            chunks[i] = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                        if (lane < 2)                         // (keys of other sequences among them: the rows look for themselves)
                            asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"((lane ? odd1 : odd0) + (look.k % kPromptOddSlots) * 4), "r"(look.k + 1) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("fence.acq_rel.cluster;\n" ::: "memory");
                        tc::mbar_arrive_release_cluster(v_bar0 + look.st * 8);
                    }
                    __syncwarp();
                    if (++look.st == kVStages) look.st = 0;
                    ++look.j;
                    moved = true;
                }
                if (look.n > 0 && look.j == look.n) {
                    if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
                    look.n = 0;
                    ++look.k;
                    moved = true;
                }
            }
            if (moved) {
                idle = 0;
            } else if ((++idle & 0xff) == 0) {                // bounded, as every wait
                const uint64_t now = tc::global_timer_ns();
                if (idle == 0x100) since = now;
                if (now - since > plan_limit) *abort_flag = 1;
                if (__any_sync(0xffffffffu, *abort_flag != 0)) break;
            }
        }
    } else if (warp == kVWarp) {
        // ------------------------------------------------------------ V: CTA r fetches half r of d of a step's 128 keys
        if (tc::elect_one()) {
            const uint32_t bar0 = cluster_address(sm.v_full, 0);
            int st = 0, ph = 1;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                const int slot = k % kPromptPlans;
                if (!(ok = tc::mbar_wait(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit))) break;
                const int n_steps = sm.tile[slot].n_steps, k0 = sm.tile[slot].k0, gk = sm.tile[slot].gk, first_masked = sm.tile[slot].first_masked;
                if (n_steps == 0) break;
                for (int j = 0; j < n_steps; ++j) {
                    if (!(ok = tc::mbar_wait(&sm.v_empty[st], ph, abort_flag))) break;
                    if (j < first_masked) {
                        if (rank == 0) tc::mbar_arrive_expect_tx(&sm.v_full[st], 2 * kTileBytes);
                        else tc::mbar_arrive_cluster(bar0 + st * 8);
                        tc::tma_load_3d_pair(&sm.v[st][0], &tmV, rank * (D / 2), gk, k0 + j * 128, bar0 + st * 8);
                    } else {                                  // K's warp looks for what is no number and says that it is there
                        tc::mbar_arrive_expect_tx(&sm.v_raw[st], kTileBytes);
                        tc::tma_load_3d(&sm.v[st][0], &tmV, rank * (D / 2), gk, k0 + j * 128, &sm.v_raw[st]);
                    }
                    if (++st == kVStages) { st = 0; ph ^= 1; }
                }
                tc::mbar_arrive(&sm.plan_empty[slot]);
            }
        }
    } else if (warp == kMmaWarp && rank == 1) {
        // ------------------------------------------------------------ CTA 1: Q is there, said to the issuing warp of CTA 0
        if (lane == 0) {
            for (int k = 0;; ++k) {
                const int slot = k % kPromptPlans;
                if (!tc::mbar_wait(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit) || sm.tile[slot].n_steps == 0) break;
                if (!tc::mbar_wait(&sm.q_full[k & 1], (k >> 1) & 1, abort_flag)) break;
                asm volatile("fence.acq_rel.cluster;\n" ::: "memory");
                tc::mbar_arrive_cluster(cluster_address(&sm.q_peer[k & 1], 0));
                tc::mbar_arrive(&sm.plan_empty[slot]);
            }
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ MMA issuer
        constexpr uint32_t kKStep = 32 >> 4;                                        // 16 elements of a 128-byte row
        constexpr uint32_t kQPanelStep = (128 * 128) >> 4, kKPanelStep = (64 * 128) >> 4, kVStep = (16 * kVRow) >> 4;
        constexpr uint32_t kQSlotStep = (uint32_t)sizeof(sm.q[0]) >> 4, kStageStep = (uint32_t)sizeof(sm.k[0]) >> 4;
        // V: rows of a key's 64 (D = 64: 32) values with the 128- (64-) byte swizzle, groups of 8 keys kVRow * 8 bytes apart
        constexpr uint32_t kVDescHi = (uint32_t)((8 * kVRow) >> 4) | (1u << 14) | ((D == 128 ? 2u : 4u) << 29);
        const uint32_t q_lo0 = __shfl_sync(0xffffffffu, tc::smem_desc_lo_sw128(smem_u32(&sm.q[0][0][0][0])), 0);
        const uint32_t k_lo0 = __shfl_sync(0xffffffffu, tc::smem_desc_lo_sw128(smem_u32(&sm.k[0][0])), 0);
        const uint32_t v_lo0 = __shfl_sync(0xffffffffu, tc::smem_desc_lo_sw128(smem_u32(&sm.v[0][0])), 0);
        const uint32_t tb = __shfl_sync(0xffffffffu, tbase, 0);
        if (tc::elect_one()) {
            bool ok = true, ended = false;
            int ks = -1, s_left = 0, sbuf = 0, kst = 0, kph = 0, ahead = 0;
            int n_steps0 = 0, n_steps1 = 0, n_steps2 = 0;         // steps of tiles ks, ks - 1, ks - 2
            // S of the next step, if there is one (must: nothing else is left to issue, so the next tile is waited for)
            auto next_scores = [&](bool must) -> bool {
                if (s_left == 0) {
                    if (ended) return false;
                    const int kn = ks + 1, slot = kn % kPromptPlans;
                    auto there = [&](uint64_t* bar, uint32_t phase) -> bool { return must ? (ok = tc::mbar_wait(bar, phase, abort_flag, plan_limit)) : tc::mbar_test(bar, phase); };
                    if (!there(&sm.plan_full[slot], (kn / kPromptPlans) & 1)) return false;
                    if ((ended = sm.tile[slot].n_steps == 0)) return false;
                    if (!there(&sm.q_full[kn & 1], (kn >> 1) & 1) || !there(&sm.q_peer[kn & 1], (kn >> 1) & 1)) return false;
                    ks = kn;
                    n_steps2 = n_steps1;
                    n_steps1 = n_steps0;
                    s_left = n_steps0 = sm.tile[slot].n_steps;
                    tc::mbar_arrive(&sm.plan_empty[slot]);
                }
                if (!(ok = tc::mbar_wait(&sm.k_full[kst], kph, abort_flag))) return false;
                tc::tc_fence_after_sync();
                const uint32_t qa = q_lo0 + (ks & 1) * kQSlotStep, kb = k_lo0 + kst * kStageStep, dst = tb + sbuf * 128;
#pragma unroll
                for (int x = 0; x < kQKSteps; ++x)
                    tc::umma_ss_pair(dst, tc::smem_desc_from_halves(qa + (x >> 2) * kQPanelStep + (x & 3) * kKStep, tc::kSmemDescHiSw128),
                                     tc::smem_desc_from_halves(kb + (x >> 2) * kKPanelStep + (x & 3) * kKStep, tc::kSmemDescHiSw128), kIdescS, x > 0);
                tc::umma_commit_pair(&sm.s_full[sbuf]);
                tc::umma_commit_pair(&sm.k_empty[kst]);
                if (--s_left == 0) tc::umma_commit_pair(&sm.q_empty[ks & 1]);
                if (++sbuf == kPromptBufs) sbuf = 0;
                if (++kst == kKStages) { kst = 0; kph ^= 1; }
                ++ahead;
                return true;
            };
            int buf = 0, buf_ph = 0, vst = 0, vph = 0;
            for (int k = 0; ok; ++k) {
                int steps = 1;
                for (int j = 0; j < steps; ++j) {
                    while (ahead < kPromptBufs && next_scores(ahead == 0)) {}
                    if (!ok || ahead == 0) { ok = false; break; }  // no more
                    if (j == 0) steps = ks == k ? n_steps0 : ks == k + 1 ? n_steps1 : n_steps2;
                    if (!(ok = tc::mbar_wait(&sm.v_full[vst], vph, abort_flag))) break;
                    if (j == 0 && k > 0 && !(ok = tc::mbar_wait(&sm.o_free, (k - 1) & 1, abort_flag))) break;
                    if (!(ok = tc::mbar_wait(&sm.p_full[buf], buf_ph, abort_flag))) break;
                    tc::tc_fence_after_sync();
                    const uint32_t vb = v_lo0 + vst * kStageStep, src = tb + buf * 128;
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        tc::umma_ts_pair(tb + kOCol, src + (x >> 2) * 64 + (x & 3) * 8, tc::smem_desc_from_halves(vb + x * kVStep, kVDescHi), kIdescO, x > 0 || j > 0);
                    tc::umma_commit_pair(&sm.v_empty[vst]);
                    if (j == steps - 1) tc::umma_commit_pair(&sm.o_full);
                    if (++vst == kVStages) { vst = 0; vph ^= 1; }
                    if (++buf == kPromptBufs) { buf = 0; buf_ph ^= 1; }
                    --ahead;
                }
            }
        }
    } else if (warp < kKWarp) {
        // ------------------------------------------------------------ softmax warps
        // Warpgroups 2 t and 2 t + 1 are team t, which takes every second step; a thread has half the keys of a row (TMEM lane).
        const int wg = warp >> 2, team = wg >> 1, half = wg & 1, quad = warp & 3;
        const int row = quad * 32 + lane;
        const uint32_t lane_addr = tbase + ((uint32_t)(quad * 32) << 16);
        const uint32_t p_bar0 = cluster_address(&sm.p_full[0], 0), o_free_bar = cluster_address(&sm.o_free, 0);
        const float scale_log2 = g.scale_log2;
        const unsigned long long scale2 = pack_f32x2(scale_log2, scale_log2);
        const int pair_bar = 1 + team * 4 + quad;              // the two warps that share 32 rows
        auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;\n" ::"r"(pair_bar) : "memory"); };
        auto pair_any = [&](bool x) -> bool {
            int r;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 64, p;\n\tselp.s32 %0, 1, 0, q;\n\t}\n" : "=r"(r) : "r"((int)x), "r"(pair_bar) : "memory");
            return r != 0;
        };
        int tok, head;                                        // of the row
        g.div_g.divmod(row, tok, head);
        bool ok = true;
        int g0 = 0;                                           // steps of the tiles before this one
        bool out_pending = false;                             // the rows of an epilogue leave shared memory while this team goes on
        auto release_out = [&]() {
            if (out_pending) {
                asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.out_free);
                out_pending = false;
            }
        };
        // A wait that has expired does not end the loops below at once, for the two warps of a row meet in barriers: ok says so, and the
        // loops end with the tile (further waits return quickly).
        for (int k = 0;; ++k) {
            const int slot = k % kPromptPlans;
            if (!tc::mbar_wait(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit)) ok = false;
            if (pair_any(!ok)) break;
            const PromptTile t = sm.tile[slot];
            if (t.n_steps == 0) break;
            const int last = t.last0 + tok;                   // the last key that the row sees
            const bool valid = tok < t.n_tok;                 // (the tile's last rows may be none, tokens behind the sequence not its own)
            const int j0 = (team + g0) & 1;
            const bool finishes = ((g0 + t.n_steps - 1) & 1) == team;
            float m_ref = 0.f, l_sum = 0.f;
            for (int j = j0; j < t.n_steps; j += kPromptTeams) {
                const int gs = g0 + j, rs = gs & (kPromptRefSlots - 1), buf = gs % kPromptBufs;
                const uint32_t s_addr = lane_addr + buf * 128 + half * 64;
                const bool masked = j >= t.first_masked;
                const int n_vis = masked ? last + 1 - j * 128 - half * 64 : 64;    // keys of the half step that the row sees (any number)
                if (!tc::mbar_wait(&sm.s_full[buf], (gs / kPromptBufs) & 1, abort_flag)) ok = false;
                tc::tc_fence_after_sync();
                auto hide = [&](uint32_t (&s)[32], int c) {
                    const int n = n_vis - c * 32;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (i >= n) s[i] = 0xff800000u;
                };
                // what the warp's rows see of a chunk of 32 keys: nothing, all of it, or each its own (hide).  Most chunks of masked steps are of
                // the first two kinds
                auto sees_none = [&](int c) -> bool { return masked && __all_sync(0xffffffffu, !valid || n_vis - c * 32 <= 0); };
                auto sees_all = [&](int c) -> bool { return !masked || __all_sync(0xffffffffu, !valid || n_vis - c * 32 >= 32); };
                auto largest = [&](const uint32_t (&s)[32]) -> float {
                    float a0 = -INFINITY, a1 = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        a0 = fmax3(a0, __uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
                        a1 = fmax3(a1, __uint_as_float(s[16 + 2 * i]), __uint_as_float(s[17 + 2 * i]));
                    }
                    return fmaxf(a0, a1);
                };
                if (j == 0) {
                    // ---- the reference of the tile: the largest of the first 128 scores
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        if (sees_none(c)) break;
                        uint32_t s[32];
                        tc::tmem_ld_32x32(s_addr + c * 32, s);
                        tc::tmem_wait_ld_for(s);
                        if (!sees_all(c)) hide(s, c);
                        top = fmaxf(top, largest(s));
                    }
                    sm.other_ref[team][half][row] = top;
                    pair_sync();
                    top = fmaxf(top, sm.other_ref[team][half ^ 1][row]) * scale_log2;    // scale > 0
                    // (-inf: so far the row sees nothing, or scores of -inf alone; the lowest reference there is, above which any score is
                    // far, and the first step that has one moves it.  An overflow of the product with the scale ends there, too)
                    m_ref = fmaxf(top, kPromptLowest);
                    if (half == 0) {
                        sm.first_ref[k & 1][row] = m_ref;
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(&sm.first_done[k & 1][quad]);
                    }
                    pair_sync();                               // (other_ref is written again below)
                } else if (j == j0) {
                    if (!tc::mbar_wait(&sm.first_done[k & 1][quad], (k >> 1) & 1, abort_flag)) ok = false;
                    m_ref = sm.first_ref[k & 1][row];
                }
                // ---- weights, 32 keys at a time over the scores
                const float ref = m_ref;
                const unsigned long long add2 = pack_f32x2(-ref, -ref);
                unsigned long long psA = 0ull, psB = 0ull;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t s[32], pk[16];
                    if (sees_none(c)) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) pk[i] = 0u;
                        tc::tmem_st_32x16(s_addr + c * 16, pk);
                        continue;
                    }
                    tc::tmem_ld_32x32(s_addr + c * 32, s);
                    tc::tmem_wait_ld_for(s);
                    if (!sees_all(c)) hide(s, c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const unsigned long long x01 = fma_f32x2(pack_f32x2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), scale2, add2);
                        const unsigned long long x23 = fma_f32x2(pack_f32x2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3])), scale2, add2);
                        float x0, x1, x2, x3;
                        unpack_f32x2(x01, x0, x1);
                        unpack_f32x2(x23, x2, x3);
                        const float p0 = fast_exp2(x0), p1 = fast_exp2(x1), p2 = fast_exp2(x2), p3 = fast_exp2(x3);
                        psA = add_f32x2(psA, pack_f32x2(p0, p1));
                        psB = add_f32x2(psB, pack_f32x2(p2, p3));
                        pk[2 * i] = pack_bf16x2(p0, p1);
                        pk[2 * i + 1] = pack_bf16x2(p2, p3);
                    }
                    tc::tmem_st_32x16(s_addr + c * 16, pk);
                }
                float a0, a1, b0, b1;
                unpack_f32x2(psA, a0, a1);
                unpack_f32x2(psB, b0, b1);
                float l_step = (a0 + a1) + (b0 + b1);
                // ---- the steps' references in order: it only grows
                float m_prev = ref;
                if (gs > 0 && !tc::mbar_wait(&sm.ref_done[(gs - 1) & (kPromptRefSlots - 1)][quad], ((gs - 1) / kPromptRefSlots) & 1, abort_flag)) ok = false;
                if (j > 0) m_prev = sm.ref[(gs - 1) & (kPromptRefSlots - 1)][row];
                float m_new = m_prev;
                const bool over = valid && l_step > kPromptBig;   // (no number: some score is none, and so will the row be)
                if (pair_any(over || ref != m_prev)) {
                    // rare: the reference of one half has to move, or that of the step before has
                    const bool lost = over && !(l_step < 0x1p100f);   // (weights near 2^128 are infinite, their factors near 2^-126 zero)
                    const __nv_bfloat16* q_row = g.q + (long long)(t.q0 + tok) * g.q_ts + (t.gk * g.G + head) * g.q_hs;
                    const int key0 = j * 128 + half * 64, n_keys = lost ? min(last + 1 - key0, 64) : 0;
                    const __nv_bfloat16* keys = g.k + (long long)(t.k0 + key0) * g.k_ts + t.gk * g.k_hs;
                    float mine = ref;
                    if (over && !lost) mine += ceilf(log2f(l_step));
                    for (int i = 0; i < n_keys; ++i) mine = fmaxf(mine, prompt_dot<D>(q_row, keys + i * g.k_ts) * scale_log2);
                    // up by a whole number, as above; so far (or from the lowest reference) that what stood before is zero: to the score itself
                    if (lost && mine - ref < 512.f) mine = ref + ceilf(mine - ref);
                    sm.other_ref[team][half][row] = mine;
                    pair_sync();
                    m_new = fmaxf(m_prev, fmaxf(mine, sm.other_ref[team][half ^ 1][row]));
                    const float f = fast_exp2(ref - m_new);
                    l_step = lost ? 0.f : l_step * f;
                    l_sum *= fast_exp2(m_ref - m_new);
                    tc::tmem_wait_st();
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[8];
                        tc::tmem_ld_32x8(s_addr + c * 8, w);
                        tc::tmem_wait_ld();
                        if (lost) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float p[2];
#pragma unroll
                                for (int y = 0; y < 2; ++y) {
                                    const int i = c * 16 + 2 * e + y;
                                    p[y] = i < n_keys ? fast_exp2(fmaf(prompt_dot<D>(q_row, keys + i * g.k_ts), scale_log2, -m_new)) : 0.f;
                                    l_step += p[y];
                                }
                                w[e] = pack_bf16x2(p[0], p[1]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(__uint_as_float(w[e] << 16) * f, __uint_as_float(w[e] & 0xffff0000u) * f);
                        }
                        __syncwarp();
                        tc::tmem_st_32x8(s_addr + c * 8, w);
                    }
                    if (j > 0 && __any_sync(0xffffffffu, m_new != m_prev)) {
                        // O holds the products of all steps up to the last one, and no later one starts before this step's weights are
                        // reported; half its columns each
                        const float factor = fast_exp2(m_prev - m_new);
                        if (!tc::mbar_wait(&sm.v_empty[(gs - 1) % kVStages], ((gs - 1) / kVStages) & 1, abort_flag)) ok = false;
                        tc::tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < D / 64; ++c) {
                            uint32_t o0[32];
                            const uint32_t at = lane_addr + kOCol + half * (D / 2) + c * 32;
                            tc::tmem_ld_32x32(at, o0);
                            tc::tmem_wait_ld_for(o0);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o0[e] = __float_as_uint(__uint_as_float(o0[e]) * factor);
                            tc::tmem_st_32x32(at, o0);
                        }
                    }
                    pair_sync();                               // other_ref has been read
                }
                if (half == 0) {
                    sm.ref[rs][row] = m_new;
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sm.ref_done[rs][quad]);
                }
                l_sum += l_step;
                m_ref = m_new;
                tc::tmem_wait_st();
                tc::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive_cluster(p_bar0 + buf * 8);
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
            // ---- the teams' sums meet in the one that took the last step; the other goes on to the next tile
            release_out();
            const int ps = k & 1, p_ph = (k >> 1) & 1;
            if (!finishes) {
                if (!tc::mbar_wait(&sm.part_free[ps], p_ph ^ 1, abort_flag)) ok = false;
                sm.part_l[ps][half][row] = l_sum;
                sm.part_m[ps][half][row] = m_ref;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.part_full[ps]);
            } else {
                sm.other_l[team][half][row] = l_sum;
                if (!tc::mbar_wait(&sm.part_full[ps], p_ph, abort_flag)) ok = false;
                pair_sync();
                // first halves first: both of a row's threads add in the same order.  The reference only grows: the last step's is the largest
                float l_fin = sm.other_l[team][0][row] + sm.other_l[team][1][row];
                const float l_part = sm.part_l[ps][0][row] + sm.part_l[ps][1][row];
                if (l_part != 0.f) l_fin += l_part * fast_exp2(sm.part_m[ps][0][row] - m_ref);
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.part_free[ps]);
                const float inv = l_fin != 0.f ? 1.f / l_fin : 0.f;
                const bool mine = valid;
                const long long at = (long long)(t.q0 + tok) * g.Hq + t.gk * g.G + head;
                float* part_o = nullptr;                      // this thread's outputs of a part
                if (t.part >= 0) {
                    const size_t part_row = ((size_t)t.part * 2 + rank) * 128 + row;
                    part_o = partial + part_row * D + half * (D / 2);
                    if (half == 0) reinterpret_cast<float2*>(partial + (size_t)kPromptParts * 256 * D)[part_row] = make_float2(m_ref, l_fin);
                } else if (mine && half == 0 && lse != nullptr) lse[at] = (m_ref + log2f(l_fin)) * 0.6931471805599453f;
                if (k > 0 && !tc::mbar_wait(&sm.out_free, (k - 1) & 1, abort_flag)) ok = false;
                if (!tc::mbar_wait(&sm.o_full, k & 1, abort_flag)) ok = false;
                tc::tc_fence_after_sync();
                const bool odd = *(volatile int*)&sm.odd_tile[k % kPromptOddSlots] == k + 1;
                unsigned char* srow = sm.out[row] + half * D;     // half the row's bytes
#pragma unroll 1
                for (int c = 0; c < D / 64; ++c) {
                    uint32_t o[32];
                    tc::tmem_ld_32x32(lane_addr + kOCol + half * (D / 2) + c * 32, o);
                    tc::tmem_wait_ld_for(o);
                    if (c == D / 64 - 1) {
                        tc::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive_cluster(o_free_bar);
                    }
                    if (part_o != nullptr) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(part_o + c * 32 + e * 4) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint4 val;
                        val.x = pack_bf16x2(__uint_as_float(o[8 * e + 0]) * inv, __uint_as_float(o[8 * e + 1]) * inv);
                        val.y = pack_bf16x2(__uint_as_float(o[8 * e + 2]) * inv, __uint_as_float(o[8 * e + 3]) * inv);
                        val.z = pack_bf16x2(__uint_as_float(o[8 * e + 4]) * inv, __uint_as_float(o[8 * e + 5]) * inv);
                        val.w = pack_bf16x2(__uint_as_float(o[8 * e + 6]) * inv, __uint_as_float(o[8 * e + 7]) * inv);
                        *reinterpret_cast<uint4*>(srow + (c * 4 + e) * 16) = val;
                    }
                }
                if (odd && mine) {                            // rare: values that are no numbers and that this row sees
                    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(srow);
                    for (int key = t.first_masked * 128; key <= last; ++key) {
                        const __nv_bfloat16* vr = g.v + (long long)(t.k0 + key) * g.v_ts + t.gk * g.v_hs + half * (D / 2);
                        for (int d = 0; d < D / 2; ++d) {
                            const float x = __bfloat162float(vr[d]);
                            if (fabsf(x) < INFINITY) continue;
                            if (part_o != nullptr) part_o[d] += x;
                            else o[d] = __float2bfloat16(__bfloat162float(o[d]) + x);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                if (mine && part_o == nullptr) asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n" ::"l"(out + at * D + half * (D / 2)), "r"(smem_u32(srow)), "n"(D) : "memory");
                asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
                out_pending = true;
                pair_sync();                                  // other_l has been read
            }
            g0 += t.n_steps;
        }
        release_out();
    }
    // ---------------------------------------------------------------- teardown
    __syncwarp();
    tc::settle_after_abort(abort_flag);
    __syncwarp();
    tc::tc_fence_before_sync();
    cluster_sync();                                           // nothing of the other CTA reaches this one any more
    if (tid == 0 && sm.abort_flag && status != nullptr) atomicExch(status, 6);   // a bounded wait expired
    if (warp == kMmaWarp) tc::tmem_dealloc_pair<512>(tbase);
}

// Puts the parts of cut tiles together: grid (kPromptParts, 256 / kPromptJoinRows), CTA (i, y) kPromptJoinRows rows of the tile whose first
// part is item i.
constexpr int kPromptJoinThreads = 256, kPromptJoinRows = 16;

template <int D>
__global__ void __launch_bounds__(kPromptJoinThreads) prompt_join_kernel(PromptGeom g, int n_pairs, const float* partial, __nv_bfloat16* out, float* lse) {
    constexpr int kLanes = D / 4, kRows = 32 / kLanes;        // threads of a row, rows of a warp
    __shared__ PromptWalk found;
    __shared__ int mine;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp == 0) {
        PromptWalk w;
        w.begin(g, true, n_pairs, lane);
        const bool x = w.find(g, blockIdx.x, lane, true) && w.part == 0;
        if (lane == 0) {
            found = w;
            mine = x;
        }
    }
    __syncthreads();
    launch_dependents();
    wait_for_previous_kernel();
    if (!mine) return;
    const PromptWalk& w = found;
    const float2* stats = reinterpret_cast<const float2*>(partial + (size_t)kPromptParts * 256 * D);
    const int d4 = lane % kLanes;
    for (int r = warp * kRows + lane / kLanes; r < kPromptJoinRows; r += kRows * (kPromptJoinThreads / 32)) {
        const int row = blockIdx.y * kPromptJoinRows + r, rank = row >> 7;
        int tok, head;
        g.div_g.divmod(row & 127, tok, head);
        if (tok >= w.tokens(g, rank)) continue;
        // statistics and outputs of four parts are asked for together; more are joined to what these gave
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = 0; p0 < w.parts; p0 += 4) {
            float2 s[4];
            float4 o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const size_t at = (size_t)(blockIdx.x + min(p0 + i, w.parts - 1)) * 256 + row;
                s[i] = stats[at];
                o[i] = *reinterpret_cast<const float4*>(partial + at * D + 4 * d4);
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p0 + i < w.parts && s[i].y != 0.f) top = fmaxf(top, s[i].x);      // (0: the row sees none of the part's keys)
            const float c = l != 0.f ? fast_exp2(m - top) : 0.f;
            l *= c;
            acc.x *= c; acc.y *= c; acc.z *= c; acc.w *= c;
            m = top;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (p0 + i >= w.parts || s[i].y == 0.f) continue;
                const float f = fast_exp2(s[i].x - m);
                l = fmaf(s[i].y, f, l);
                acc.x = fmaf(o[i].x, f, acc.x);
                acc.y = fmaf(o[i].y, f, acc.y);
                acc.z = fmaf(o[i].z, f, acc.z);
                acc.w = fmaf(o[i].w, f, acc.w);
            }
        }
        const float inv = l != 0.f ? 1.f / l : 0.f;
        const long long at = (long long)(w.seq.q0 + w.first_token(g, rank) + tok) * g.Hq + w.gk * g.G + head;
        *reinterpret_cast<uint2*>(out + at * D + 4 * d4) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        if (d4 == 0 && lse != nullptr) lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace adaspark
