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
//   warp  17    MMA issuer (CTA 0): S = Q K^T, O += P V (P in TMEM, V with its rows along d); CTA 1: passes on that its Q (8-bit pages: its V) is there
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
//
// Keys and values in the pages of a cache (kKeysPages): several new tokens a sequence, all of its tokens or a window of the last ones and the first few.
// The steps of a tile are those of the first ones and those from the window's beginning on, which start with the box of its first key (not at a
// multiple of 128 keys: 47.0 -> 44.4 us for 5874 tokens and a window of 300); what only some of its rows see is masked by 32 bits a row and chunk.  A row whose first steps show it nothing begins with the first that does.  Boxes that no row sees are read as zeros, whatever
// the table says of them.  A page's number is asked for a step ahead.  With few tiles a pair (PromptLine) they are one line cut into
// equal runs: 2048 tokens over 65536 2.64 -> 2.13 ms, a mixed batch of chunks and single tokens 105 -> 88 us against tiles dealt longest first.
//
// Pages of e4m3 (kKeysPages8): K goes to the tensor cores as it lies in the pages (kind::f8f6f4), against q in two parts of four bits each whose sum
// q is; the products are multiplied by the row's power of two and, four keys a load, by the keys' before they are weighed.  V is brought to bf16 in
// shared memory by four more warps (20-23), with its powers of two in it: the weights need more bits than an 8-bit operand has.  (K brought to
// bf16, too: 2.89 against 2.75 ms of 2048 tokens over 65536 then.)  What bounds it is issue and fetch of instructions: 5300 instructions of warps a
// step and CTA against 3100 of bf16 pages, and the stall that leads is that none is there (2.4 of 9.9 cycles an instruction; bf16 1.1); loops
// that are rolled up are faster than the same unrolled.  24 warps leave a thread 80 registers: 94 bytes of it are spilled with heads of 64, 86 with heads of
// 128 (bf16 pages, 20 warps and 96 registers: 18 bytes; packed rows: none).  Tried without gain: rows of few tokens twice, each copy with half of the keys; 8 warps for
// the codes and registers moved between warpgroups (spills); more or fewer stages of K, V and codes; the keys' powers of two a step ahead.
#pragma once
#include <type_traits>

#include "paged_cache.cuh"
#include "tc_common.cuh"

namespace adaspark {

// Where keys and values are: packed rows, pages of bf16, pages of e4m3.
constexpr int kKeysPacked = 0, kKeysPages = 1, kKeysPages8 = 2;

constexpr int kPromptTeams = 2;                               // softmax teams, of two warpgroups each
constexpr int kPromptCodeWarps = 4;                           // 8-bit pages: warps that see to codes and queries
__host__ __device__ constexpr int prompt_threads(int keys) { return (2 * kPromptTeams + (keys == kKeysPages8 ? 2 : 1)) * 128; }
constexpr int kPromptPlans = 4;                               // tiles planned at once
constexpr int kPromptBufs = 3;                                // score tiles in TMEM
constexpr int kPromptRefSlots = 4;
constexpr float kPromptBig = 0x1p40f;                         // a reference moves when a half step's weights sum up to more
constexpr float kPromptLowest = -3.402823466e38f;             // a reference below any score
// A planner that walks past levels of a long prompt looks at every sequence for each: 16 ns a sequence and level, 150 levels and more from one of
// a pair's tiles to its next (where a level has one tile).  Waits for its plans last so much longer.
constexpr uint64_t kPromptPlanNs = 10000;                     // a sequence
constexpr int kPromptOddSlots = 8;                            // more than tiles whose V can be under way at once (a step each)
__host__ __device__ constexpr int prompt_k_stages(int D, int keys) { return D == 64 ? 6 : keys == kKeysPages8 ? 4 : 3; }   // steps whose K, V are under way
__host__ __device__ constexpr int prompt_v_stages(int D) { return D == 64 ? 6 : 3; }
__host__ __device__ constexpr int prompt_raw_stages(int D, int keys) { return keys != kKeysPages8 ? 0 : D == 64 ? 6 : 3; }   // steps whose codes of V are under way
constexpr int kPromptFactorSlots = 8;                         // steps whose keys' powers of two are kept
static_assert(prompt_v_stages(64) + 2 <= kPromptFactorSlots, "a step's are written when the values of the step before have their place");
static_assert(prompt_v_stages(64) + 1 < kPromptOddSlots, "a slot is not written again before it has been read");

// Shared memory by its 32-bit address
__device__ __forceinline__ uint4 load_shared_16(uint32_t at) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at) : "memory");
    return r;
}
// (not held to its place among other accesses)
__device__ __forceinline__ uint4 load_shared_16_free(uint32_t at) {
    uint4 r;
    asm("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(at));
    return r;
}
__device__ __forceinline__ void store_shared_8(uint32_t at, const uint2& v) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" ::"r"(at), "r"(v.x), "r"(v.y) : "memory");
}
__device__ __forceinline__ uint32_t load_shared_byte(uint32_t at) {
    uint32_t r;
    asm volatile("ld.shared.u8 %0, [%1];\n" : "=r"(r) : "r"(at) : "memory");
    return r;
}
__device__ __forceinline__ void store_shared_16(uint32_t at, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// sum += 0 * x, of two bf16 each
__device__ __forceinline__ void add_times_zero(uint32_t& sum, uint32_t x) { asm("fma.rn.bf16x2 %0, %1, %2, %0;\n" : "+r"(sum) : "r"(x), "r"(0u)); }
// 8 codes that are numbers times 2^(s - 127), s in 8 .. 134, as bf16: exact.  A code's exponent and mantissa four bits below bf16's are the same number
// times 2^-120, subnormal ones too; f is 2^(s - 7) twice.  Bytes are made four at a time: the low ones of the bf16 numbers, the high ones, then
// these beside those.  top: the largest magnitudes so far, before f; a code that is no number shows as 0x7f0 and is 480 here.  (Codes to f16, to f32, multiplied and
// rounded: as many instructions, but a chain of conversions.)
constexpr uint32_t kNoNumberTop = 0x07f0u;
__device__ __forceinline__ uint4 codes_to_bf16x8(uint32_t a, uint32_t b, uint32_t f, uint32_t& top) {
    uint32_t r[4];
    const uint32_t w[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t low = (w[i] << 4) & 0xf0f0f0f0u, high = ((w[i] >> 4) & 0x07070707u) | (w[i] & 0x80808080u);
        r[2 * i] = __byte_perm(low, high, 0x5140);
        r[2 * i + 1] = __byte_perm(low, high, 0x7362);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        asm("max.xorsign.abs.bf16x2 %0, %0, %1;\n" : "+r"(top) : "r"(r[i]));
        asm("mul.rn.bf16x2 %0, %0, %1;\n" : "+r"(r[i]) : "r"(f));
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// What a reference that grows by -d does to what stands: times 2^d, in two factors, for a weight of up to 2^100 may meet a d below -126.
struct MovedBy {
    float a, b;
    __device__ __forceinline__ explicit MovedBy(float d) : a(fast_exp2(fmaxf(d, -120.f))), b(fast_exp2(fminf(d + 120.f, 0.f))) {}
    __device__ __forceinline__ float of(float x) const { return x * b * a; }
};

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

// Chunk c (8 values) of a key's or value's row in its page, as bf16; zeros where the page is not there.
template <int D, bool kCodes>
__device__ __noinline__ uint4 paged_chunk(const PageGeom& p, const uint8_t* pages, const uint8_t* scales, int seq, int head, int key, int c) {
    const long long page = page_of(p, seq, key);
    if (page < 0) return make_uint4(0u, 0u, 0u, 0u);
    const long long row = ((long long)head << p.page_shift) + (key & ((1 << p.page_shift) - 1)), at = page * p.page_stride + row * D + c * 8;
    if (!kCodes) return *reinterpret_cast<const uint4*>(pages + at * 2);
    return chunk_values(*reinterpret_cast<const uint2*>(pages + at), min((uint32_t)scales[page * p.scale_stride + row], 254u));
}
// q.k of a row in global memory and one in its page
template <int D, bool kCodes>
__device__ __noinline__ float paged_dot(const PageGeom& p, int seq, int head, int key, const __nv_bfloat16* q) {
    float sum = 0.f;
#pragma unroll 1
    for (int c = 0; c < D / 8; ++c) {
        const uint4 a = *reinterpret_cast<const uint4*>(q + c * 8), b = paged_chunk<D, kCodes>(p, p.k, p.ks, seq, head, key, c);
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
    // keys in pages
    PageGeom pages;
    const int32_t* kv_len;
    int window, sinks;          // window 0: none
    int most_steps;             // a bound on the steps of a tile (by the window, if there is one)
};

struct PromptTile {
    int q0, n_tok;              // this CTA's first row of q and its tokens (the pair's first CTA may have all)
    int k0;                     // first key row of the sequence
    int last0;                  // last key that this CTA's first token sees (-1 and less: none)
    int gk;
    int n_steps, first_masked;  // steps of 128 keys; from this one on rows are masked
    int part;                   // number of the part of a tile whose keys are cut, -1: a whole tile
    // keys in pages (last0 counts from the sequence's first token then)
    int seq;
    int step0, sink_steps, base;    // of the tile's steps, the first sink_steps hold the keys from 0 on, the others those from `base` on; j = 0 is number step0
    int low_first, low_masked;      // steps [low_first, low_masked) are masked, too
    int lo, hi;                     // some row sees something of [lo, hi) and of the first ones; of nothing else
    __device__ __forceinline__ int key_of(int j) const { return step0 + j < sink_steps ? (step0 + j) << 7 : base + ((step0 + j - sink_steps) << 7); }
    __device__ __forceinline__ bool masked(int j) const { return j >= first_masked || (j >= low_first && j < low_masked); }
    // the first masked step from step j on (n_steps: none)
    __device__ __forceinline__ int next_masked(int j) const {
        const int low = max(j, low_first), tail = max(j, first_masked);      // (a tile that begins among the first tokens: its tail in front of the border)
        return min(low < low_masked ? min(low, tail) : tail, n_steps);
    }
};

// A sequence as a planner sees it; one that leaves the tensors has no tiles, one whose length is none no keys.
template <bool kPaged>
struct PromptSeq {
    int q0, k0, nq, nk, off, nt, b;
    __device__ __forceinline__ bool load(const PromptGeom& g, int i) {
        const int a0 = g.cu_q[i], a1 = g.cu_q[i + 1], b0 = kPaged ? 0 : g.cu_k[i];
        int b1 = kPaged ? g.kv_len[i] : g.cu_k[i + 1];
        bool valid = 0 <= a0 && a0 <= a1 && a1 <= g.n_q && (kPaged || (0 <= b0 && b0 <= b1 && b1 <= g.n_k)), fine = valid;
        if (kPaged) {
            const bool there = b1 >= 0 && b1 <= (g.pages.table_width << g.pages.page_shift);
            fine = valid && (a0 == a1 || (there && b1 >= a1 - a0));
            if (!there) b1 = 0;
            b = i;
        }
        q0 = a0;
        k0 = b0;
        nq = valid ? a1 - a0 : 0;
        nk = valid ? b1 - b0 : 0;
        off = nk - nq;
        nt = nq > 0 ? g.div_w.div(nq + 2 * g.T - 1) : 0;
        return fine;
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
constexpr int kPromptSlots = 2 * kPromptPairs;                // of parts (pages: two a pair, PromptLine)
static_assert(kPromptParts <= kPromptSlots, "room for either");
// Rows of the cut tiles' parts: outputs [part][CTA][128][D], then (reference, sum) [part][CTA][128]
__host__ __device__ constexpr size_t prompt_partial_bytes(int D) { return (size_t)kPromptSlots * 256 * (D + 2) * sizeof(float); }
// Could a call have tiles to cut?  (If not, there is nothing to join either: 36.1 against 37.9 us for 4301 tokens in 5 prompts, 16 heads of 64.)  More
// tiles than 4 a pair: no one is long enough to matter.  Whole prompts: the n / W tiles of a prompt of n tokens, W to a tile, average half
// of its n / 128 steps; that is 1.5 times what a pair has to do only up to n = 99 W / Hkv, and no tile of less than 12 steps is cut.
inline bool prompt_may_cut(long long most_tiles, int n_k, bool whole, int W, int Hkv) {
    return most_tiles <= 4 * kPromptPairs && n_k > 128 * 3 * kPromptMinUnit / 2 && (!whole || W > 16 * Hkv);
}

// Steps of n keys; a table may have room for nearly 2^31.
constexpr int kPromptMostSteps = 1 << 24;
__host__ __device__ constexpr int prompt_steps(int n) { return ((n - 1) >> 7) + 1; }

// The order of the items (tiles, or parts of them): levels from many steps to few, sequences in order, tiles, kv heads, parts.  A warp walks
// it, with 32 sequences in its lanes.  Parts come first: an item's number is its part's.  (Pages: whole tiles alone, cut ones are PromptLine's; with a
// window a tile's level is the bound on its steps where it would be more.)
template <bool kPaged>
struct PromptWalk {
    int level, unit;                                          // unit 0: nothing is cut (packed rows alone, as part and parts are)
    int below;                                                // most steps of a tile of fewer than `level`, among the sequences seen so far
    int chunk, base;                                          // number of the first item of (level, chunk)
    int held;                                                 // chunk of `mine`, this lane's sequence
    PromptSeq<kPaged> mine;
    // what find() found
    PromptSeq<kPaged> seq;
    int tile, gk, part, parts;

    // false: a sequence leaves the tensors
    __device__ __forceinline__ bool begin(const PromptGeom& g, [[maybe_unused]] bool cut, [[maybe_unused]] int n_pairs, int lane) {
        bool fine = true;
        [[maybe_unused]] long long steps = 0;                 // at least as many as there are
        level = chunk = base = below = 0;
        for (held = 0; held * 32 < g.batch; ++held) {
            mine.nt = 0;
            if (held * 32 + lane < g.batch) {
                fine = mine.load(g, held * 32 + lane) && fine;
                if (mine.nt > 0) {
                    const int longest = max(1, prompt_steps(mine.nk));
                    level = max(level, kPaged ? min(longest, g.most_steps) : longest);
                    if constexpr (!kPaged) steps += (long long)mine.nt * (max(mine.off, 0) / 128 + 2) + (long long)g.T * mine.nt * (mine.nt + 1) / 128;
                }
            }
        }
        --held;
        level = (int)__reduce_max_sync(0xffffffffu, (unsigned)level);
        if constexpr (!kPaged) {
            unit = 0;
            if (cut) {
#pragma unroll
                for (int x = 16; x > 0; x >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, x);
                unit = (int)max((steps * g.Hkv + n_pairs - 1) / n_pairs, (long long)kPromptMinUnit);
            }
        }
        return fine;
    }
    __device__ __forceinline__ int parts_of(int steps) const { return !kPaged && unit > 0 ? max((2 * steps + unit) / (2 * unit), 1) : 1; }
    // item `number`, which is no smaller than the one before; false: there are not so many (of cut tiles)
    __device__ __forceinline__ bool find(const PromptGeom& g, int number, int lane, bool cut_only = false) {
        while (level > 0) {
            const int n_parts = parts_of(level);              // (pages: 1)
            if constexpr (!kPaged) parts = n_parts;
            if (cut_only && n_parts == 1) return false;
            if (held != chunk) {                              // (up to 32 sequences: never)
                held = chunk;
                mine.nt = 0;
                if (chunk * 32 + lane < g.batch) mine.load(g, chunk * 32 + lane);
            }
            int first = 0, n = 0;
            if (mine.nt > 0) {
                first = level == 1 ? 0 : mine.tiles_up_to(g, 128 * (level - 1));
                n = ((kPaged && level == g.most_steps ? mine.nt : mine.tiles_up_to(g, 128 * level)) - first) * g.Hkv * n_parts;
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
                if (kPaged) seq.b = chunk * 32 + who;
                if constexpr (!kPaged) {
                    part = i % n_parts;
                    i /= n_parts;
                }
                g.div_kv.divmod(i, tile, gk);
                tile += __shfl_sync(0xffffffffu, first, who);
                return true;
            }
            base += total;
            // the next level is that of the longest tile left: levels without a tile are passed over
            if (first > 0) below = max(below, max(prompt_steps(min(mine.off + 2 * g.T * first, mine.nk)), 1));   // (below `level`, whatever bounds that)
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

// What the rows of a tile see of pages: steps, and which are masked.
struct PromptSpan {
    int n;                                                    // steps
    int hi, lo, sink_steps, base, low_first, low_masked, first_masked;
    __device__ __forceinline__ PromptSpan(const PromptGeom& g, const PromptSeq<true>& seq, int tile) {
        const int tok0 = 2 * tile * g.T, m = min(seq.nq - tok0, 2 * g.T);
        const int p0 = seq.off + tok0, p1 = p0 + m - 1;      // places of the tile's first and last token
        hi = max(p1 + 1, 0);
        n = max(prompt_steps(hi), 1);
        sink_steps = base = lo = low_first = low_masked = 0;
        if (g.window > 0) {
            lo = max(max(p0, 0) + 1 - g.window, 0);          // (rows in front of token 0: a window may be 2^31 - 1)
            sink_steps = min(prompt_steps(g.sinks), n);
            // the window's steps begin with the box that holds its first key, or go on where the first ones' end
            base = max(lo & -min(1 << g.pages.page_shift, 128), sink_steps << 7);
            n = max(sink_steps + prompt_steps(max(hi - base, 0)), 1);
            const int lo1 = max(hi - g.window, 0);           // (the last row's)
            if (lo1 > g.sinks) {
                low_first = g.sinks >> 7;
                low_masked = sink_steps + prompt_steps(max(lo1 - base, 0));
            }
        }
        const int next = max(p0 + 1, 0);                     // the first key that the first row does not see
        first_masked = next < base ? next >> 7 : sink_steps + ((next - base) >> 7);
    }
};

// Few tiles over pages: all tiles, sequence by sequence, tile by tile, kv head by kv head, are one line, cut into equal runs, one a pair.
// (Whole tiles dealt longest first left a pair 2072 of an average of 1602 steps, parts of about the average 257 of 171; and a planner that
// walks levels finds its first tile 5 us later.)  Lengths are in keys: what the tile's last row sees, and in front of that kPromptAhead for what a
// tile costs beside its steps.  A pair's first tile may have begun in an earlier run, its last may go on in the next: two parts a pair,
// joined by prompt_join_kernel.  Nobody cuts off less than kPromptLeast steps.
// (Not with more than four tiles a pair, prompt_may_cut: 456 tiles of 270 steps on average gain 5 %, of 17 steps lose 17.)
constexpr int kPromptAhead = 384, kPromptLeast = 3;
struct PromptLine {
    int chunk;                                                // first sequence of the lanes' 32
    PromptSeq<true> mine;
    long long own;                                            // its length
    // the tile
    PromptSeq<true> seq;
    int tile, gk;
    long long place, cost;                                    // its beginning and length

    static __device__ __forceinline__ long long limit(const PromptGeom& g) { return g.most_steps < kPromptMostSteps ? 128ll * g.most_steps : 0x7fffffffll; }
    static __device__ __forceinline__ long long cost_of(const PromptGeom& g, const PromptSeq<true>& q, int t) {
        return kPromptAhead + min(max((long long)q.off + 2ll * g.T * (t + 1), 0ll), limit(g));
    }
    // length of the first t tiles of one head
    static __device__ __forceinline__ long long length(const PromptGeom& g, const PromptSeq<true>& q, int t) {
        const long long W = 2 * g.T, most = limit(g);
        const int none = q.off >= 0 ? 0 : min(g.div_w.div(-q.off), t);              // tiles that see nothing
        // tiles of less than the limit: W (u + 1) + off < most
        const long long room = most - q.off - 1;
        const int rising = max(min(room < 0 ? 0 : room >= 0x7fffffffll ? t : g.div_w.div((int)room), t), none);
        const long long m = rising - none;
        return (long long)t * kPromptAhead + m * q.off + W * (m * none + m * (m + 1) / 2) + (t - rising) * most;
    }
    __device__ __forceinline__ bool load(const PromptGeom& g, int c, int lane) {
        chunk = c;
        mine.nt = 0;
        const bool fine = c + lane >= g.batch || mine.load(g, c + lane);
        own = mine.nt > 0 ? length(g, mine, mine.nt) * g.Hkv : 0;
        return fine;
    }
    // length of the line; fine: no sequence leaves the tensors or its table
    __device__ __forceinline__ long long begin(const PromptGeom& g, int lane, bool& fine) {
        long long sum = 0;
        fine = true;
        for (int c = 0; c < g.batch; c += 32) {
            fine = load(g, c, lane) && fine;
            sum += own;
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
        return sum;
    }
    __device__ __forceinline__ void take(const PromptGeom& g, int who) {
        seq.q0 = __shfl_sync(0xffffffffu, mine.q0, who);
        seq.nq = __shfl_sync(0xffffffffu, mine.nq, who);
        seq.nk = __shfl_sync(0xffffffffu, mine.nk, who);
        seq.off = seq.nk - seq.nq;
        seq.nt = __shfl_sync(0xffffffffu, mine.nt, who);
        seq.k0 = 0;
        seq.b = chunk + who;
    }
    // the tile that holds place x of the line; false: there is none
    __device__ __forceinline__ bool seek(const PromptGeom& g, long long x, int lane) {
        long long before = 0;
        for (int c = 0; c < g.batch; c += 32) {
            if (c > 0 || chunk != 0) load(g, c, lane);
            long long upto = own;
#pragma unroll
            for (int y = 1; y < 32; y <<= 1) {
                const long long z = __shfl_up_sync(0xffffffffu, upto, y);
                if (lane >= y) upto += z;
            }
            const long long all = __shfl_sync(0xffffffffu, upto, 31);
            if (x < before + all) {
                const int who = __ffs(__ballot_sync(0xffffffffu, before + upto > x)) - 1;
                const long long first = before + __shfl_sync(0xffffffffu, upto - own, who), rest = x - first;
                take(g, who);
                int lo = 0, hi = seq.nt;                      // length(lo) * Hkv <= rest < length(hi) * Hkv; a lane a place to look at
                while (hi - lo > 1) {
                    const int step = (hi - lo + 31) >> 5, at = lo + step * (lane + 1);
                    const int below = __popc(__ballot_sync(0xffffffffu, at < hi && length(g, seq, at) * g.Hkv <= rest));
                    lo += step * below;
                    hi = min(lo + step, hi);
                }
                tile = lo;
                cost = cost_of(g, seq, tile);
                place = first + length(g, seq, tile) * g.Hkv;
                for (gk = 0; x - place >= cost; ++gk) place += cost;
                return true;
            }
            before += all;
        }
        return false;
    }
    __device__ __forceinline__ bool next(const PromptGeom& g, int lane) {
        place += cost;
        if (++gk < g.Hkv) return true;
        gk = 0;
        if (++tile >= seq.nt) {
            tile = 0;
            int from = seq.b + 1 - chunk;
            while (true) {
                const uint32_t there = from < 32 ? __ballot_sync(0xffffffffu, mine.nt > 0) >> from << from : 0u;
                if (there) {
                    take(g, __ffs(there) - 1);
                    break;
                }
                if (chunk + 32 >= g.batch) return false;
                load(g, chunk + 32, lane);
                from = 0;
            }
        }
        cost = cost_of(g, seq, tile);
        return true;
    }
    // steps of the tile's n that lie in front of place x
    __device__ __forceinline__ int steps_before(long long x, int n) const {
        const long long y = x - place - kPromptAhead;
        if (y >= cost - kPromptAhead) return n;
        if (y <= 0) return 0;
        // (in 32 bits: it has to grow with y and to be the same for whoever asks, no more)
        const int i = (int)((float)(int)y / (float)(int)(cost - kPromptAhead) * (float)n);
        return i < kPromptLeast ? 0 : n - i < kPromptLeast ? n : i;
    }
};
// The line's runs, of equal length but for the last one's few keys more
struct PromptRuns {
    long long total, length;
    int n_pairs;
    __device__ __forceinline__ PromptRuns(long long total_, int n) : total(total_), length(total_ >> 32 ? total_ / n : (uint32_t)total_ / (uint32_t)n), n_pairs(n) {}
    __device__ __forceinline__ long long begin(int run) const { return run == n_pairs ? total : length * run; }
};

template <int D, int kKeys>
struct PromptSmem {
    __nv_bfloat16 q[2][D / 64][128][64];                      // [tile & 1][d panel][row][64 d]
    __nv_bfloat16 k[prompt_k_stages(D, kKeys)][64 * D / (kKeys == kKeysPages8 ? 2 : 1)];   // [d panel][this CTA's 64 keys][64 d]; codes: [64 keys][D]
    __nv_bfloat16 v[prompt_v_stages(D)][64 * D];              // [128 keys][this CTA's half of d]
    unsigned char raw_v[prompt_raw_stages(D, kKeys)][64 * D]; // V's codes as they lie in the pages: [128 keys][this CTA's half of d]
    unsigned char out[128][2 * D + 16];
    uint8_t raw_ks[prompt_raw_stages(D, kKeys)][128], raw_vs[prompt_raw_stages(D, kKeys)][128];   // powers of two of the keys and values
    float key_factor[kKeys == kKeysPages8 ? kPromptFactorSlots : 0][128], row_factor[kKeys == kKeysPages8 ? kPromptPlans : 0][128];
    float ref[kPromptRefSlots][128], first_ref[2][128];      // reference of a row after a step, after the first 128 keys of a tile
    float part_l[2][2][128], part_m[2][2][128];             // sums and reference of the team that does not finish a tile, by half
    float other_l[kPromptTeams][2][128], other_ref[kPromptTeams][2][128];   // between the halves of a row
    uint64_t q_full[2], q_peer[2], q_empty[2], k_full[prompt_k_stages(D, kKeys)], k_empty[prompt_k_stages(D, kKeys)], v_full[prompt_v_stages(D)], v_empty[prompt_v_stages(D)];
    uint64_t v_raw[prompt_v_stages(D)], s_full[kPromptBufs], p_full[kPromptBufs], ref_done[kPromptRefSlots][4], first_done[2][4], o_full, o_free;
    uint64_t plan_full[kPromptPlans], plan_empty[kPromptPlans], part_full[2], part_free[2], out_free;
    uint64_t rv_full[prompt_raw_stages(D, kKeys)], rv_empty[prompt_raw_stages(D, kKeys)], key_factor_full[kKeys == kKeysPages8 ? kPromptFactorSlots : 0],
        row_factor_full[kKeys == kKeysPages8 ? kPromptPlans : 0];
    PromptTile tile[kPromptPlans];
    int odd_tile[kPromptOddSlots];                            // number + 1 of a tile with masked values that are no numbers
    uint32_t tmem_base;
    int abort_flag;
};

static_assert(sizeof(PromptSmem<128, kKeysPages8>) + 1024 <= 232448 && sizeof(PromptSmem<64, kKeysPages8>) + 1024 <= 232448, "what a CTA may have");

template <int D, int kKeys>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(prompt_threads(kKeys), 1) attn_prompt_kernel(
    const __grid_constant__ PromptGeom g, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    __nv_bfloat16* out, float* lse, float* partial, int32_t* status) {
    extern __shared__ unsigned char prompt_smem_raw[];
    using Smem = PromptSmem<D, kKeys>;
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(prompt_smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kPanels = D / 64, kQKSteps = D / 16, kKStages = prompt_k_stages(D, kKeys), kVStages = prompt_v_stages(D);
    constexpr bool kPaged = kKeys != kKeysPacked, kCodes = kKeys == kKeysPages8;
    [[maybe_unused]] constexpr int kRawStages = prompt_raw_stages(D, kKeys);
    constexpr uint32_t kIdescS = tc::make_idesc_bf16(256, 128);
    constexpr uint32_t kIdescO = tc::make_idesc_bf16(256, D) | (1u << 16);   // B = V: rows along N
    constexpr uint32_t kTileBytes = 64 * D * 2;               // a CTA's share of the K or V of a step
    constexpr uint32_t kKTileBytes = kKeys == kKeysPages8 ? kTileBytes / 2 : kTileBytes;
    constexpr int kVRow = D;                                  // bytes of a key in a CTA's share of V (half of d)
    constexpr int kKWarp = kPromptTeams * 8, kMmaWarp = kKWarp + 1, kVWarp = kKWarp + 2, kPlanWarp = kKWarp + 3;
    constexpr uint32_t kOCol = kPromptBufs * 128;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x & 1u), n_pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1);

    // ---------------------------------------------------------------- set-up
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&sm.q_full[i], 1);
            tc::mbar_init(&sm.q_peer[i], kCodes ? 2 * kPromptCodeWarps : 1);
            tc::mbar_init(&sm.q_empty[i], 1);
            tc::mbar_init(&sm.part_full[i], 8);
            tc::mbar_init(&sm.part_free[i], 8);
        }
        for (int i = 0; i < kPromptPlans; ++i) {
            tc::mbar_init(&sm.plan_full[i], 1);
            tc::mbar_init(&sm.plan_empty[i], (kCodes ? 3 + kPromptCodeWarps : 4) + kPromptTeams * 8);
        }
        for (int i = 0; i < kKStages; ++i) {
            tc::mbar_init(&sm.k_full[i], 1);
            tc::mbar_init(&sm.k_empty[i], 1);
        }
        for (int i = 0; i < kVStages; ++i) {
            tc::mbar_init(&sm.v_full[i], kCodes ? kPromptCodeWarps + 1 : 2);   // CTA 0's own, and CTA 1
            tc::mbar_init(&sm.v_raw[i], kCodes ? kPromptCodeWarps : 1);
            tc::mbar_init(&sm.v_empty[i], 1);
        }
        for (int i = 0; i < kRawStages; ++i) {
            tc::mbar_init(&sm.rv_full[i], 1);
            tc::mbar_init(&sm.rv_empty[i], kPromptCodeWarps);
        }
        for (int i = 0; i < (kCodes ? kPromptFactorSlots : 0); ++i) tc::mbar_init(&sm.key_factor_full[i], kPromptCodeWarps);
        for (int i = 0; i < (kCodes ? kPromptPlans : 0); ++i) tc::mbar_init(&sm.row_factor_full[i], kPromptCodeWarps);
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
    // The page of the `sub` keys from `key` on: its number as the table has it, asked for a step ahead; then n_pages (boxes outside the pages read
    // zeros) where `t`'s rows see none of them, or where it is not there.
    [[maybe_unused]] auto seen_by = [&](const PromptTile& t, int key, int sub) -> bool { return key < t.hi && (key + sub > t.lo || key < g.sinks); };
    [[maybe_unused]] auto entry_of = [&](const PromptTile& t, int key, int sub) -> int {
        return seen_by(t, key, sub) ? g.pages.table[(size_t)t.seq * g.pages.table_width + (key >> g.pages.page_shift)] : 0;
    };
    [[maybe_unused]] auto page_for = [&](const PromptTile& t, int key, int sub, int entry) -> int {
        if (!seen_by(t, key, sub)) return g.pages.n_pages;
        if (entry >= 0 && entry < g.pages.n_pages) return entry;
        if (status != nullptr) atomicExch(status, 1);
        return g.pages.n_pages;
    };
    if (warp == kPlanWarp) {
        // ------------------------------------------------------------ planner
        // (pages) a tile's steps [begin, end)
        [[maybe_unused]] auto tile_of_pages = [&](PromptTile& t, const PromptSeq<true>& seq, int tile, int gk, const PromptSpan& x, int begin, int end) {
            const int tok = (2 * tile + rank) * g.T;
            t.seq = seq.b;
            t.q0 = seq.q0 + tok;
            t.n_tok = min(max(seq.nq - tok, 0), g.T);
            t.k0 = 0;
            t.last0 = seq.off + tok;
            t.gk = gk;
            t.n_steps = end - begin;
            t.step0 = begin;
            t.hi = x.hi;
            t.lo = x.lo;
            t.sink_steps = x.sink_steps;
            t.base = x.base;
            t.first_masked = max(x.first_masked - begin, 0);
            t.low_first = x.low_first - begin;
            t.low_masked = x.low_masked - begin;
        };
        PromptWalk<kPaged> w;
        [[maybe_unused]] PromptLine line;
        const bool in_runs = kPaged && partial != nullptr;
        bool fine, more = false;
        long long run_end = 0, run_first = 0;
        if (in_runs) {
            const long long total = line.begin(g, lane, fine);
            const PromptRuns runs(total, n_pairs);
            run_first = runs.begin(pair);
            run_end = runs.begin(pair + 1);
            more = run_first < run_end && line.seek(g, run_first, lane);
        } else {
            fine = w.begin(g, partial != nullptr, n_pairs, lane);
        }
        if (!fine && blockIdx.x == 0 && status != nullptr) atomicExch(status, 1);
        for (int k = 0;; ++k) {
            const int slot = k % kPromptPlans, qs = k & 1;
            if (!tc::mbar_wait(&sm.plan_empty[slot], ((k / kPromptPlans) & 1) ^ 1u, abort_flag)) break;
            bool found = false;
            PromptTile t;
            if (in_runs) {
                while (more && !found) {
                    const PromptSpan x(g, line.seq, line.tile);
                    const int begin = line.steps_before(run_first, x.n), end = line.steps_before(run_end, x.n);
                    found = end > begin;
                    if (found) {
                        tile_of_pages(t, line.seq, line.tile, line.gk, x, begin, end);
                        t.part = end - begin == x.n ? -1 : 2 * pair + (begin > 0 ? 0 : 1);
                    }
                    more = line.place + line.cost < run_end && line.next(g, lane);
                }
                if (found && lane == 0) sm.tile[slot] = t;
            } else {
                const int number = k * n_pairs + ((k & 1) ? n_pairs - 1 - pair : pair);
                found = w.find(g, number, lane);
                if constexpr (kPaged) {
                    if (found) {
                        const PromptSpan x(g, w.seq, w.tile);
                        tile_of_pages(t, w.seq, w.tile, w.gk, x, 0, x.n);
                        t.part = -1;
                        if (lane == 0) sm.tile[slot] = t;
                    }
                } else if (found) {
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
    } else if (kCodes && warp == kKWarp) {
        // ------------------------------------------------------------ K: CTA r fetches the codes of the keys r * 64 .. of a step
        const uint32_t bar0 = cluster_address(sm.k_full, 0);
        const int sub = min(1 << g.pages.page_shift, 64), boxes = 64 / sub;
        int st = 0, ph = 1;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            const int slot = k % kPromptPlans;
            if (!(ok = tc::mbar_wait_warp(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit))) break;
            const PromptTile t = sm.tile[slot];
            if (t.n_steps == 0) break;
            auto key_at = [&](int j) -> int { return t.key_of(j) + rank * 64 + min(lane, boxes - 1) * sub; };
            int entry = entry_of(t, key_at(0), sub);
            for (int j = 0; j < t.n_steps; ++j) {
                const int key = key_at(j), page = page_for(t, key, sub, entry);
                if (j + 1 < t.n_steps) entry = entry_of(t, key_at(j + 1), sub);
                if (!(ok = tc::mbar_wait_warp(&sm.k_empty[st], ph, abort_flag))) break;
                if (rank == 0 && lane == 0) tc::mbar_arrive_expect_tx(&sm.k_full[st], 2 * kKTileBytes);
                __syncwarp();
                if (lane < boxes) tc::tma_load_4d_pair(reinterpret_cast<unsigned char*>(sm.k[st]) + lane * sub * D, &tmK, 0, key & ((1 << g.pages.page_shift) - 1), t.gk, page, bar0 + st * 8);
                __syncwarp();
                if (++st == kKStages) { st = 0; ph ^= 1; }
            }
            if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
        }
    } else if (kCodes && warp == kVWarp) {
        // ------------------------------------------------------------ V's codes, half `rank` of d of a step's 128 keys, and the powers of two of keys and values
        const int sub = min(1 << g.pages.page_shift, 128), boxes = 128 / sub;
        int st = 0, ph = 1;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            const int slot = k % kPromptPlans;
            if (!(ok = tc::mbar_wait_warp(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit))) break;
            const PromptTile t = sm.tile[slot];
            if (t.n_steps == 0) break;
            auto key_at = [&](int j) -> int { return t.key_of(j) + min(lane, boxes - 1) * sub; };
            int entry = entry_of(t, key_at(0), sub);
            for (int j = 0; j < t.n_steps; ++j) {
                const int key = key_at(j), page = page_for(t, key, sub, entry), in = key & ((1 << g.pages.page_shift) - 1);
                if (j + 1 < t.n_steps) entry = entry_of(t, key_at(j + 1), sub);
                if (!(ok = tc::mbar_wait_warp(&sm.rv_empty[st], ph, abort_flag))) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&sm.rv_full[st], 128 * (D / 2 + 2));
                __syncwarp();
                if (lane < boxes) {
                    tc::tma_load_4d(&sm.raw_v[st][lane * sub * (D / 2)], &tmV, rank * (D / 2), in, t.gk, page, &sm.rv_full[st]);
                    const long long at = (page < g.pages.n_pages ? page : 0) * g.pages.scale_stride + ((long long)t.gk << g.pages.page_shift) + in;
                    tc::bulk_load(&sm.raw_ks[st][lane * sub], g.pages.ks + at, sub, &sm.rv_full[st]);
                    tc::bulk_load(&sm.raw_vs[st][lane * sub], g.pages.vs + at, sub, &sm.rv_full[st]);
                }
                __syncwarp();
                if (++st == kRawStages) { st = 0; ph ^= 1; }
            }
            if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
        }
    } else if (kCodes && warp >= kPlanWarp + 1) {
        // ------------------------------------------------------------ 8-bit pages: q in two parts, the keys' powers of two, V's codes to bf16
        const int part = warp - (kPlanWarp + 1);
        // Q of tile k, of which this warp has 32 rows: q * 2^(127 - s) = a + b in e4m3, s as a row of 8-bit pages has it.  A bf16 number's 8 bits are two of
        // four, so that the sum is q itself down to 2^-10 of the row's largest magnitude; what is smaller is off by 2^-18 of that at most.  In place:
        // the row's panels become its parts (head_dim 64: the two halves of its one panel).
        const uint32_t q_peer0 = cluster_address(sm.q_peer, 0);
        auto split_q = [&](int k) -> bool {
            const int slot = k % kPromptPlans, qs = k & 1;
            if (!tc::mbar_wait_warp(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit)) return false;
            if (sm.tile[slot].n_steps == 0) return true;
            if (!tc::mbar_wait_warp(&sm.q_full[qs], (k >> 1) & 1, abort_flag)) return false;
            constexpr int kLanes = D / 8, kRows = 32 / kLanes;   // lanes of a row, rows at a time
            const uint32_t q0 = smem_u32(&sm.q[qs][0][0][0]);
            const int c = lane % kLanes;
#pragma unroll 1
            for (int r = 0; r < 32; r += kRows) {
                const int row = part * 32 + r + lane / kLanes;
                const uint4 x = load_shared_16(q0 + (c >> 3) * (128 * 128) + sw128(row, c & 7));
                uint32_t top = chunk_tops(x);
                top = max(top & 0xffffu, top >> 16);
#pragma unroll
                for (int b = 1; b < kLanes; b <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, b));
                const uint32_t s = min(scale_byte(top), 247u);
                const float inv = __uint_as_float((254u - s) << 23);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                uint32_t a[4], b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float lo = __uint_as_float(w[i] << 16) * inv, hi = __uint_as_float(w[i] & 0xffff0000u) * inv;
                    uint16_t two;
                    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(hi), "f"(lo));
                    a[i] = two;
                    const uint32_t h = codes_to_f16x2(a[i]);
                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&h));
                    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(hi - back.y), "f"(lo - back.x));
                    b[i] = two;
                }
                const uint32_t first = q0 + sw128(row, c >> 1) + (c & 1) * 8, second = D == 128 ? first + 128 * 128 : q0 + sw128(row, 4 + (c >> 1)) + (c & 1) * 8;
                store_shared_8(first, make_uint2(a[0] | (a[1] << 16), a[2] | (a[3] << 16)));   // (the row has been read by all of its lanes: the shuffles)
                store_shared_8(second, make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16)));
                // no number, or an infinity: a row without numbers
                if (c == 0) sm.row_factor[slot][row] = top >= 0x7f80u ? __uint_as_float(0x7fffffffu) : g.scale_log2 * pow2_of_byte(s);
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(&sm.row_factor_full[slot]);
                tc::mbar_arrive_release_cluster(q_peer0 + qs * 8);
            }
            __syncwarp();
            return true;
        };
        constexpr int kPieces = D / 32;                       // of 16 codes, of a thread
        constexpr int kShift = D == 128 ? 2 : 1, kRows = 32 >> kShift, kRowBytes = D;   // log2 of the pieces of a row of V
        // The thread's pieces are those of column c in the rows row0 + i * kRows; their values are the 16-byte chunks 2 c and 2 c + 1 of the row.
        const int c = lane & ((1 << kShift) - 1), row0 = part * kPieces * kRows + (lane >> kShift);
        auto place = [&](int chunk) -> uint32_t { return D == 128 ? sw128(row0, chunk) : row0 * 64 + ((chunk ^ ((row0 >> 1) & 3)) << 4); };
        const uint32_t to0 = smem_u32(sm.v[0]) + place(2 * c), to1 = smem_u32(sm.v[0]) + place(2 * c + 1);
        const uint32_t raw0 = smem_u32(sm.raw_v[0]) + (part * kPieces * 32 + lane) * 16, scale0 = smem_u32(sm.raw_vs[0]) + row0;
        uint64_t* const full = rank == 0 ? sm.v_full : sm.v_raw;   // (CTA 1's are passed on to CTA 0's issuing warp)
        const uint32_t odd0 = cluster_address(sm.odd_tile, 0), odd1 = cluster_address(sm.odd_tile, 1);
        int st = 0, ph = 1, raw = 0, raw_ph = 0, gs = 0;
        bool ok = split_q(0);
        for (int k = 0; ok; ++k) {
            const int slot = k % kPromptPlans;
            if (!(ok = tc::mbar_wait_warp(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit))) break;
            const PromptTile t = sm.tile[slot];
            if (t.n_steps == 0) break;
            bool split = false;
            for (int j = 0; j < t.n_steps; ++j, ++gs) {
                if (!(ok = tc::mbar_wait_warp(&sm.rv_full[raw], raw_ph, abort_flag))) break;
                // the keys' powers of two.  (Their slot's last readers, kPromptFactorSlots steps ago, are through: the step before this has found its
                // place for V, which products with the weights of a step of less than kPromptFactorSlots - 1 before had left)
                sm.key_factor[gs % kPromptFactorSlots][part * 32 + lane] = pow2_of_byte(min((uint32_t)sm.raw_ks[raw][part * 32 + lane], 254u));
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm.key_factor_full[gs % kPromptFactorSlots]);
                const uint32_t src = raw0 + raw * (64 * D), scales = scale0 + raw * 128, dst = st * (64 * D * 2);
                if (!(ok = tc::mbar_wait_warp(&sm.v_empty[st], ph, abort_flag))) break;
                uint32_t top = 0u, far = 0u, any = 0u;
#pragma unroll 1
                for (int i = 0; i < kPieces; i += 2) {
                    uint4 x[2];
                    uint32_t sc[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        x[y] = load_shared_16(src + (i + y) * 512);
                        sc[y] = load_shared_byte(scales + (i + y) * kRows);
                    }
                    uint4 r[2][2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint32_t f = (sc[y] + 120u) * 0x00800080u;      // 2^(s - 7) twice
                        far = max(far, sc[y] - 8u);
                        r[y][0] = codes_to_bf16x8(x[y].x, x[y].y, f, top);
                        r[y][1] = codes_to_bf16x8(x[y].z, x[y].w, f, top);
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        store_shared_16(to0 + dst + (i + y) * (kRows * kRowBytes), r[y][0]);
                        store_shared_16(to1 + dst + (i + y) * (kRows * kRowBytes), r[y][1]);
                    }
                }
                if (__any_sync(0xffffffffu, (top & 0x7fffu) >= kNoNumberTop || (top >> 16 & 0x7fffu) >= kNoNumberTop || far > 126u)) {
                    // rare: codes that are no numbers, powers of two far out
#pragma unroll 1
                    for (int i = 0; i < kPieces; ++i) {
                        const uint32_t s = min(load_shared_byte(scales + i * kRows), 254u);
                        const uint4 codes = load_shared_16(src + i * 512);
                        const uint4 lo = chunk_values(make_uint2(codes.x, codes.y), s), hi = chunk_values(make_uint2(codes.z, codes.w), s);
                        const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                        for (int e = 0; e < 8; ++e) add_times_zero(any, w[e]);
                        store_shared_16(to0 + dst + i * (kRows * kRowBytes), lo);
                        store_shared_16(to1 + dst + i * (kRows * kRowBytes), hi);
                    }
                }
                if (t.masked(j) && __any_sync(0xffffffffu, (any & 0x7fff7fffu) != 0u)) {
                    // zeros instead, and the rows add what they see (this warp's part of the keys, whole rows, as it has written them)
                    __syncwarp();
                    uint4* chunks = reinterpret_cast<uint4*>(sm.v[st]) + part * kPieces * 64;
                    for (int i = lane; i < kPieces * 64; i += 32) {
                        uint32_t x[4] = {chunks[i].x, chunks[i].y, chunks[i].z, chunks[i].w};
                        for (int e = 0; e < 4; ++e) {
                            if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
                            if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
                        }
                        chunks[i] = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                    if (lane < 2) asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"((lane ? odd1 : odd0) + (k % kPromptOddSlots) * 4), "r"(k + 1) : "memory");
                    asm volatile("fence.acq_rel.cluster;\n" ::: "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    tc::mbar_arrive(&full[st]);
                    tc::mbar_arrive(&sm.rv_empty[raw]);
                }
                __syncwarp();
                if (++st == kVStages) { st = 0; ph ^= 1; }
                if (++raw == kRawStages) { raw = 0; raw_ph ^= 1; }
                // the next tile's Q beside the first steps of this one, or where it is planned: no step waits for a plan
                if (!split && (j == t.n_steps - 1 || __all_sync(0xffffffffu, tc::mbar_test(&sm.plan_full[(k + 1) % kPromptPlans], ((k + 1) / kPromptPlans) & 1)))) {
                    if (!(ok = split_q(k + 1))) break;
                    split = true;
                }
            }
            if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
        }
    } else if (warp == kKWarp) {
        // ------------------------------------------------------------ K: CTA r fetches the keys r * 64 .. of a step.  And masked steps:
        // values that are no numbers.  Whichever is ready, so that neither waits for the other.
        const uint32_t bar0 = cluster_address(sm.k_full, 0), v_bar0 = cluster_address(sm.v_full, 0);
        const uint32_t odd0 = cluster_address(sm.odd_tile, 0), odd1 = cluster_address(sm.odd_tile, 1);
        auto ready = [&](uint64_t* bar, uint32_t phase) -> bool { return __all_sync(0xffffffffu, tc::mbar_test(bar, phase)); };
        struct { int k = 0, j = 0, n = 0, st = 0; bool done = false; } kp, look;      // tile, step, steps of the tile (0: not begun), stage
        int k_ph = 1, row0 = 0, gk = 0, first_masked = 0;
        [[maybe_unused]] PromptTile kt, lt;                   // (pages) tiles of either
        [[maybe_unused]] const int sub = kPaged ? min(1 << g.pages.page_shift, 64) : 64, boxes = 64 / sub, box = lane % boxes, panel = lane / boxes;
        [[maybe_unused]] int entry = 0;
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
                    if (kPaged) {
                        kt = sm.tile[slot];
                        if (kp.n > 0) entry = entry_of(kt, kt.key_of(0) + rank * 64 + box * sub, sub);
                    }
                    kp.done = kp.n == 0;
                    moved = true;
                }
                if (kp.n > 0 && ready(&sm.k_empty[kp.st], k_ph)) {
                    if constexpr (kPaged) {
                        const int key = kt.key_of(kp.j) + rank * 64 + box * sub, page = page_for(kt, key, sub, entry);
                        if (kp.j + 1 < kp.n) entry = entry_of(kt, kt.key_of(kp.j + 1) + rank * 64 + box * sub, sub);
                        if (rank == 0 && lane == 0) tc::mbar_arrive_expect_tx(&sm.k_full[kp.st], 2 * kTileBytes);
                        __syncwarp();
                        if (panel < kPanels)
                            tc::tma_load_4d_pair(&sm.k[kp.st][(panel * 64 + box * sub) * 64], &tmK, panel * 64, key & ((1 << g.pages.page_shift) - 1), gk, page, bar0 + kp.st * 8);
                    } else if (tc::elect_one()) {
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
                    if (kPaged) lt = sm.tile[slot];
                    look.done = look.n == 0;
                    look.j = kPaged ? lt.next_masked(0) : min(first_masked, look.n);
                    look.st = (look.st + look.j) % kVStages;
                    moved = true;
                }
                if (look.n > 0 && look.j < look.n && ready(&sm.v_raw[look.st], (raw_phases >> look.st) & 1)) {
                    raw_phases ^= 1u << look.st;
                    // zero times what is infinite or no number is none, and stays that in a sum
                    uint4* chunks = reinterpret_cast<uint4*>(&sm.v[look.st][0]);
                    uint32_t none[4] = {0u, 0u, 0u, 0u};
#pragma unroll 8
                    for (int i = lane; i < (int)kTileBytes / 16; i += 32) {
                        const uint4 x = load_shared_16(smem_u32(chunks + i));
                        add_times_zero(none[0], x.x);
                        add_times_zero(none[1], x.y);
                        add_times_zero(none[2], x.z);
                        add_times_zero(none[3], x.w);
                    }
                    if (__any_sync(0xffffffffu, ((none[0] | none[1] | none[2] | none[3]) & 0x7fff7fffu) != 0u)) {
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
                        asm volatile("fence.acq_rel.cluster;\n" ::: "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive_release_cluster(v_bar0 + look.st * 8);
                    __syncwarp();
                    if (++look.st == kVStages) look.st = 0;
                    ++look.j;
                    if (kPaged) {
                        const int next = lt.next_masked(look.j);
                        look.st = (look.st + next - look.j) % kVStages;
                        look.j = next;
                    }
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
    } else if (kPaged && warp == kVWarp) {
        // ------------------------------------------------------------ V from its pages: CTA r fetches half r of d of a step's 128 keys
        const uint32_t bar0 = cluster_address(sm.v_full, 0);
        const int sub = min(1 << g.pages.page_shift, 128), boxes = 128 / sub;
        int st = 0, ph = 1;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            const int slot = k % kPromptPlans;
            if (!(ok = tc::mbar_wait_warp(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit))) break;
            const PromptTile t = sm.tile[slot];
            if (t.n_steps == 0) break;
            auto key_at = [&](int j) -> int { return t.key_of(j) + min(lane, boxes - 1) * sub; };
            int entry = entry_of(t, key_at(0), sub);
            for (int j = 0; j < t.n_steps; ++j) {
                const int key = key_at(j), page = page_for(t, key, sub, entry), in = key & ((1 << g.pages.page_shift) - 1);
                if (j + 1 < t.n_steps) entry = entry_of(t, key_at(j + 1), sub);
                if (!(ok = tc::mbar_wait_warp(&sm.v_empty[st], ph, abort_flag))) break;
                const bool masked = t.masked(j);              // K's warp looks for what is no number and says that it is there
                if (lane == 0) {
                    if (masked) tc::mbar_arrive_expect_tx(&sm.v_raw[st], kTileBytes);
                    else if (rank == 0) tc::mbar_arrive_expect_tx(&sm.v_full[st], 2 * kTileBytes);
                    else tc::mbar_arrive_cluster(bar0 + st * 8);
                }
                __syncwarp();
                if (lane < boxes) {
                    if (masked) tc::tma_load_4d(&sm.v[st][lane * sub * (D / 2)], &tmV, rank * (D / 2), in, t.gk, page, &sm.v_raw[st]);
                    else tc::tma_load_4d_pair(&sm.v[st][lane * sub * (D / 2)], &tmV, rank * (D / 2), in, t.gk, page, bar0 + st * 8);
                }
                __syncwarp();
                if (++st == kVStages) { st = 0; ph ^= 1; }
            }
            if (lane == 0) tc::mbar_arrive(&sm.plan_empty[slot]);
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
        // ------------------------------------------------------------ CTA 1: Q is there, said to the issuing warp of CTA 0 (8-bit pages: by those that
        // split it).  8-bit pages: V is there, too.  (What a thread of this CTA has written is visible to one of the other's behind a release of the
        // cluster's scope.  It is this thread's, which has written nothing: by the four warps that write V, 350 for 268 us of proposed tokens)
        if (lane == 0) {
            [[maybe_unused]] const uint32_t v_bar0 = cluster_address(sm.v_full, 0);
            [[maybe_unused]] int st = 0, ph = 0;
            bool ok = true;
            for (int k = 0; ok; ++k) {
                const int slot = k % kPromptPlans;
                if (!tc::mbar_wait(&sm.plan_full[slot], (k / kPromptPlans) & 1, abort_flag, plan_limit)) break;
                const int n_steps = sm.tile[slot].n_steps;
                if (n_steps == 0) break;
                if (!kCodes) {
                    if (!tc::mbar_wait(&sm.q_full[k & 1], (k >> 1) & 1, abort_flag)) break;
                    asm volatile("fence.acq_rel.cluster;\n" ::: "memory");
                    tc::mbar_arrive_cluster(cluster_address(&sm.q_peer[k & 1], 0));
                }
                tc::mbar_arrive(&sm.plan_empty[slot]);
                for (int j = 0; kCodes && j < n_steps; ++j) {
                    if (!(ok = tc::mbar_wait(&sm.v_raw[st], ph, abort_flag))) break;
                    tc::mbar_arrive_release_cluster(v_bar0 + st * 8);
                    if (++st == kVStages) { st = 0; ph ^= 1; }
                }
            }
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ MMA issuer
        constexpr uint32_t kKStep = 32 >> 4;                                        // 16 elements of a 128-byte row
        constexpr uint32_t kQPanelStep = (128 * 128) >> 4, kKPanelStep = (64 * 128) >> 4, kVStep = (16 * kVRow) >> 4;
        constexpr uint32_t kQSlotStep = (uint32_t)sizeof(sm.q[0]) >> 4, kKStageStep = (uint32_t)sizeof(sm.k[0]) >> 4, kStageStep = (uint32_t)sizeof(sm.v[0]) >> 4;
        // codes of K: rows of D bytes with the 128- (64-) byte swizzle, 32 of them a step
        constexpr uint32_t kIdescCodes = tc::make_idesc_e4m3(256, 128), kCodesDescHi = (uint32_t)((8 * D) >> 4) | (1u << 14) | ((D == 128 ? 2u : 4u) << 29);
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
                    auto there = [&](uint64_t* bar, uint32_t phase, auto pair) -> bool {
                        return must ? (ok = tc::mbar_wait<pair.value>(bar, phase, abort_flag, plan_limit)) : tc::mbar_test<pair.value>(bar, phase);
                    };
                    const std::false_type own;
                    const std::true_type both;                // (both CTAs' threads arrive)
                    if (!there(&sm.plan_full[slot], (kn / kPromptPlans) & 1, own)) return false;
                    if ((ended = sm.tile[slot].n_steps == 0)) return false;
                    if ((!kCodes && !there(&sm.q_full[kn & 1], (kn >> 1) & 1, own)) || !there(&sm.q_peer[kn & 1], (kn >> 1) & 1, both)) return false;
                    ks = kn;
                    n_steps2 = n_steps1;
                    n_steps1 = n_steps0;
                    s_left = n_steps0 = sm.tile[slot].n_steps;
                    tc::mbar_arrive(&sm.plan_empty[slot]);
                }
                if (!(ok = tc::mbar_wait(&sm.k_full[kst], kph, abort_flag))) return false;
                tc::tc_fence_after_sync();
                const uint32_t qa = q_lo0 + (ks & 1) * kQSlotStep, kb = k_lo0 + kst * kKStageStep, dst = tb + sbuf * 128;
                if constexpr (kCodes) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)          // both parts of q, the products of 32 codes at a time
                        tc::umma_ss_pair_e4m3(dst, tc::smem_desc_from_halves(qa + (x >> 2) * kQPanelStep + (x & 3) * kKStep, tc::kSmemDescHiSw128),
                                              tc::smem_desc_from_halves(kb + (x % (D / 32)) * kKStep, kCodesDescHi), kIdescCodes, x > 0);
                } else {
#pragma unroll
                    for (int x = 0; x < kQKSteps; ++x)
                        tc::umma_ss_pair(dst, tc::smem_desc_from_halves(qa + (x >> 2) * kQPanelStep + (x & 3) * kKStep, tc::kSmemDescHiSw128),
                                         tc::smem_desc_from_halves(kb + (x >> 2) * kKPanelStep + (x & 3) * kKStep, tc::kSmemDescHiSw128), kIdescS, x > 0);
                }
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
                    if (!(ok = tc::mbar_wait<true>(&sm.v_full[vst], vph, abort_flag))) break;
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
            const int first = kPaged && g.window > 0 ? max(max(last, 0) + 1 - g.window, 0) : 0;   // of those behind the first ones
            const bool idle = kPaged && !__any_sync(0xffffffffu, valid);   // no row of the warp is one: nothing is computed
            [[maybe_unused]] float row_factor = 0.f;          // 8-bit pages: scores are products with codes times this and the key's power of two
            if constexpr (kCodes) {
                if (!tc::mbar_wait(&sm.row_factor_full[slot], (k / kPromptPlans) & 1, abort_flag)) ok = false;
                row_factor = sm.row_factor[slot][row];
            }
            [[maybe_unused]] const unsigned long long row_factor2 = pack_f32x2(row_factor, row_factor);
            // products of the two may leave 32 bits on the way, the score not: the key's first where the row's is large
            [[maybe_unused]] const bool large = kCodes && __any_sync(0xffffffffu, valid && row_factor > 0x1p100f);
            const int j0 = (team + g0) & 1;
            const bool finishes = ((g0 + t.n_steps - 1) & 1) == team;
            float m_ref = 0.f, l_sum = 0.f;
            for (int j = j0; j < t.n_steps; j += kPromptTeams) {
                const int gs = g0 + j, rs = gs & (kPromptRefSlots - 1), buf = gs % kPromptBufs;
                const uint32_t s_addr = lane_addr + buf * 128 + half * 64;
                const bool masked = kPaged ? t.masked(j) : j >= t.first_masked;
                const int key0 = kPaged ? t.key_of(j) + half * 64 : j * 128 + half * 64;
                // (pages) which of the 32 keys from key0 + 32 c on the row sees
                auto seen_of = [&](int c) -> uint32_t {
                    const int k = key0 + c * 32;
                    auto below = [](int n) -> uint32_t { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
                    return below(last + 1 - k) & (~below(first - k) | below(g.sinks - k));
                };
                const int n_vis = masked ? last + 1 - j * 128 - half * 64 : 64;    // keys of the half step that the row sees (any number)
                if constexpr (kCodes)
                    if (!tc::mbar_wait(&sm.key_factor_full[gs % kPromptFactorSlots], (gs / kPromptFactorSlots) & 1, abort_flag)) ok = false;
                if (!tc::mbar_wait(&sm.s_full[buf], (gs / kPromptBufs) & 1, abort_flag)) ok = false;
                tc::tc_fence_after_sync();
                // (the address as it is known behind the waits: the loads through it may go anywhere behind that)
                [[maybe_unused]] uint32_t factors = 0u;
                if constexpr (kCodes) asm volatile("add.u32 %0, %1, %2;\n" : "=r"(factors) : "r"(smem_u32(sm.key_factor[gs % kPromptFactorSlots])), "r"(half * 256) : "memory");
                // 8-bit pages: four products with codes, times the row's factor and the keys' (i: the first of them / 4, of 32 keys from chunk c on)
                [[maybe_unused]] auto scaled = [&](uint32_t (&s)[32], int c) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint4 f = load_shared_16_free(factors + c * 128 + i * 16);
                        unsigned long long a = pack_f32x2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), b = pack_f32x2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3]));
                        const unsigned long long fa = pack_f32x2(__uint_as_float(f.x), __uint_as_float(f.y)), fb = pack_f32x2(__uint_as_float(f.z), __uint_as_float(f.w));
                        a = mul_f32x2(mul_f32x2(a, large ? fa : row_factor2), large ? row_factor2 : fa);
                        b = mul_f32x2(mul_f32x2(b, large ? fb : row_factor2), large ? row_factor2 : fb);
                        s[4 * i] = (uint32_t)a;
                        s[4 * i + 1] = (uint32_t)(a >> 32);
                        s[4 * i + 2] = (uint32_t)b;
                        s[4 * i + 3] = (uint32_t)(b >> 32);
                    }
                };
                auto hide = [&](uint32_t (&s)[32], int c) {
                    const int n = n_vis - c * 32;
                    const uint32_t seen = kPaged ? seen_of(c) : 0u;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (kPaged ? (seen >> i & 1u) == 0u : i >= n) s[i] = 0xff800000u;
                };
                // what the warp's rows see of a chunk of 32 keys: nothing, all of it, or each its own (hide).  Most chunks of masked steps are of
                // the first two kinds
                auto sees_none = [&](int c) -> bool {
                    if (kPaged) return idle || (masked && __all_sync(0xffffffffu, !valid || seen_of(c) == 0u));
                    return masked && __all_sync(0xffffffffu, !valid || n_vis - c * 32 <= 0);
                };
                auto sees_all = [&](int c) -> bool {
                    if (kPaged) return !masked || __all_sync(0xffffffffu, !valid || seen_of(c) == ~0u);
                    return !masked || __all_sync(0xffffffffu, !valid || n_vis - c * 32 >= 32);
                };
                auto largest = [&](const uint32_t (&s)[32]) -> float {
                    float a0 = -INFINITY, a1 = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        a0 = fmax3(a0, __uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
                        a1 = fmax3(a1, __uint_as_float(s[16 + 2 * i]), __uint_as_float(s[17 + 2 * i]));
                    }
                    return fmaxf(a0, a1);
                };
                // ---- the largest of the step's scores, of both halves; none: the lowest reference there is, above which any score is far, and the
                // first step that has one moves it.  An overflow of the product with the scale ends there, too
                auto first_reference = [&]() -> float {
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c = 0; c < 2; ++c) {
                        if (sees_none(c)) {
                            if (kPaged) continue;             // (a window may hide the first keys alone)
                            break;
                        }
                        uint32_t s[32];
                        tc::tmem_ld_32x32(s_addr + c * 32, s);
                        tc::tmem_wait_ld_for(s);
                        if constexpr (kCodes) scaled(s, c);
                        if (!sees_all(c)) hide(s, c);
                        top = fmaxf(top, largest(s));
                    }
                    sm.other_ref[team][half][row] = top;
                    pair_sync();
                    return fmaxf(fmaxf(top, sm.other_ref[team][half ^ 1][row]) * (kCodes ? 1.f : scale_log2), kPromptLowest);    // scale > 0
                };
                if (j == 0) {
                    // ---- the reference of the tile: the largest of the first 128 scores
                    m_ref = first_reference();
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
                float ref_now = m_ref;
                if (kPaged && j > 0 && __any_sync(0xffffffffu, valid && m_ref == kPromptLowest)) {
                    // rows that have seen nothing (a window that begins behind their tile's first step): their reference is this step's.  (Both
                    // halves of a row hold the same reference)
                    const float top = first_reference();
                    if (m_ref == kPromptLowest) ref_now = top;
                    pair_sync();
                }
                // ---- weights, 32 keys at a time over the scores
                const float ref = ref_now;
                const unsigned long long add2 = pack_f32x2(-ref, -ref);
                unsigned long long psA = 0ull, psB = 0ull;
                // (8-bit pages: their warps go so many ways that instructions are what they wait for most; rolled up 254 for 281 us of proposed tokens)
                constexpr int kChunksAtOnce = kCodes ? 1 : 2;
#pragma unroll kChunksAtOnce
                for (int c = 0; c < 2; ++c) {
                    uint32_t s[32], pk[16];
                    if (sees_none(c)) {
                        if (idle) continue;                   // (rows that nobody reads)
#pragma unroll
                        for (int i = 0; i < 16; ++i) pk[i] = 0u;
                        tc::tmem_st_32x16(s_addr + c * 16, pk);
                        continue;
                    }
                    tc::tmem_ld_32x32(s_addr + c * 32, s);
                    tc::tmem_wait_ld_for(s);
                    // (one loop for either order of the factors: a branch within would part its instructions)
                    auto weigh = [&](auto key_first) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            unsigned long long x01 = pack_f32x2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), x23 = pack_f32x2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3]));
                            if constexpr (!kCodes) {
                                x01 = fma_f32x2(x01, scale2, add2);
                                x23 = fma_f32x2(x23, scale2, add2);
                            } else {
                                const uint4 f = load_shared_16_free(factors + c * 128 + i * 16);
                                const unsigned long long f01 = pack_f32x2(__uint_as_float(f.x), __uint_as_float(f.y)), f23 = pack_f32x2(__uint_as_float(f.z), __uint_as_float(f.w));
                                x01 = key_first.value ? fma_f32x2(mul_f32x2(x01, f01), row_factor2, add2) : fma_f32x2(mul_f32x2(x01, row_factor2), f01, add2);
                                x23 = key_first.value ? fma_f32x2(mul_f32x2(x23, f23), row_factor2, add2) : fma_f32x2(mul_f32x2(x23, row_factor2), f23, add2);
                            }
                            float x0, x1, x2, x3;
                            unpack_f32x2(x01, x0, x1);
                            unpack_f32x2(x23, x2, x3);
                            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1), p2 = fast_exp2(x2), p3 = fast_exp2(x3);
                            psA = add_f32x2(psA, pack_f32x2(p0, p1));
                            psB = add_f32x2(psB, pack_f32x2(p2, p3));
                            pk[2 * i] = pack_bf16x2(p0, p1);
                            pk[2 * i + 1] = pack_bf16x2(p2, p3);
                        }
                    };
                    if (!sees_all(c)) hide(s, c);
                    if (kCodes && large) weigh(std::true_type());
                    else weigh(std::false_type());
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
                    const int n_keys = lost ? min(last + 1 - key0, 64) : 0;
                    const __nv_bfloat16* keys = kPaged ? nullptr : g.k + (long long)(t.k0 + key0) * g.k_ts + t.gk * g.k_hs;
                    auto score = [&](int i) -> float {        // -inf: the row does not see it
                        if constexpr (kPaged) return seen_of(i >> 5) >> (i & 31) & 1u ? paged_dot<D, kCodes>(g.pages, t.seq, t.gk, key0 + i, q_row) * scale_log2 : -INFINITY;
                        else return prompt_dot<D>(q_row, keys + i * g.k_ts) * scale_log2;
                    };
                    float mine = ref;
                    if (over && !lost) mine += ceilf(log2f(l_step));
                    for (int i = 0; i < n_keys; ++i) mine = fmaxf(mine, score(i));
                    // up by a whole number, as above; so far (or from the lowest reference) that what stood before is zero: to the score itself
                    if (lost && mine - ref < 512.f) mine = ref + ceilf(mine - ref);
                    sm.other_ref[team][half][row] = mine;
                    pair_sync();
                    m_new = fmaxf(m_prev, fmaxf(mine, sm.other_ref[team][half ^ 1][row]));
                    // (pages: a reference that did not begin with the other team's may lie a fraction apart)
                    if (kPaged && m_new - ref < 512.f) m_new = ref + ceilf(m_new - ref);
                    const MovedBy f(ref - m_new);
                    l_step = lost ? 0.f : f.of(l_step);
                    l_sum *= fast_exp2(m_ref - m_new);
                    tc::tmem_wait_st();
                    const bool rewrite = !kPaged || __any_sync(0xffffffffu, ref != m_new);   // (pages: a first reference moves nothing)
#pragma unroll 1
                    for (int c = 0; c < (rewrite ? 4 : 0); ++c) {
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
                                    if constexpr (kPaged) p[y] = i < n_keys ? fast_exp2(score(i) - m_new) : 0.f;
                                    else p[y] = i < n_keys ? fast_exp2(fmaf(prompt_dot<D>(q_row, keys + i * g.k_ts), scale_log2, -m_new)) : 0.f;
                                    l_step += p[y];
                                }
                                w[e] = pack_bf16x2(p[0], p[1]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(f.of(__uint_as_float(w[e] << 16)), f.of(__uint_as_float(w[e] & 0xffff0000u)));
                        }
                        __syncwarp();
                        tc::tmem_st_32x8(s_addr + c * 8, w);
                    }
                    if (j > 0 && __any_sync(0xffffffffu, m_new != m_prev && (!kPaged || (valid && m_prev != kPromptLowest)))) {   // (from the lowest: O is zero)
                        // O holds the products of all steps up to the last one, and no later one starts before this step's weights are
                        // reported; half its columns each
                        const MovedBy factor(m_prev - m_new);
                        if (!tc::mbar_wait(&sm.v_empty[(gs - 1) % kVStages], ((gs - 1) / kVStages) & 1, abort_flag)) ok = false;
                        tc::tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < D / 64; ++c) {
                            uint32_t o0[32];
                            const uint32_t at = lane_addr + kOCol + half * (D / 2) + c * 32;
                            tc::tmem_ld_32x32(at, o0);
                            tc::tmem_wait_ld_for(o0);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o0[e] = __float_as_uint(factor.of(__uint_as_float(o0[e])));
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
                    if (half == 0) reinterpret_cast<float2*>(partial + (size_t)kPromptSlots * 256 * D)[part_row] = make_float2(m_ref, l_fin);
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
                        if (kPaged && !mine) continue;
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
                if (kPaged && odd && mine) {                  // rare: values that are no numbers and that this row sees
                    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(srow);
                    for (int j = t.next_masked(0); j < t.n_steps; j = t.next_masked(j + 1))
                        for (int key = t.key_of(j), end = key + min(128, last + 1 - key); key < end; ++key) {
                            if (key < first && key >= g.sinks) continue;
                            for (int c = 0; c < D / 16; ++c) {
                                const uint4 chunk = paged_chunk<D, kCodes>(g.pages, g.pages.v, g.pages.vs, t.seq, t.gk, key, half * (D / 16) + c);
                                const uint32_t w[4] = {chunk.x, chunk.y, chunk.z, chunk.w};
                                for (int e = 0; e < 8; ++e) {
                                    const float x = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
                                    const int d = c * 8 + e;
                                    if (fabsf(x) < INFINITY) continue;
                                    if (part_o != nullptr) part_o[d] += x;
                                    else o[d] = __float2bfloat16(__bfloat162float(o[d]) + x);
                                }
                            }
                        }
                }
                if (!kPaged && odd && mine) {
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
// part is item i.  Pages: grid (runs - 1, ..), CTA (i, y) the tile that begins in run i and is cut by that run's end.
constexpr int kPromptJoinThreads = 256, kPromptJoinRows = 16;

template <int D, bool kPaged>
__global__ void __launch_bounds__(kPromptJoinThreads) prompt_join_kernel(PromptGeom g, int n_pairs, const float* partial, __nv_bfloat16* out, float* lse) {
    constexpr int kLanes = D / 4, kRows = 32 / kLanes;        // threads of a row, rows of a warp
    __shared__ PromptSeq<kPaged> seq;
    __shared__ int part_at[kPaged ? kPromptSlots : 1], n_parts, tile, gk;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp == 0) {
        int n = 0;
        if constexpr (kPaged) {
            PromptLine w;
            bool fine;
            const long long total = w.begin(g, lane, fine);
            const PromptRuns runs(total, n_pairs);
            const long long cut = runs.begin(blockIdx.x + 1);
            if (cut < total && w.seek(g, cut, lane) && w.place < cut && w.place >= runs.begin(blockIdx.x)) {
                const PromptSpan x(g, w.seq, w.tile);
                // a lane a run: of those that the tile lies in, the ones that hold steps of it
                for (int r = blockIdx.x; r < n_pairs && runs.begin(r) < w.place + w.cost; r += 32) {
                    const int run = r + lane, begin = run < n_pairs ? w.steps_before(runs.begin(run), x.n) : 0,
                              end = run < n_pairs ? w.steps_before(runs.begin(run + 1), x.n) : 0;
                    const uint32_t holds = __ballot_sync(0xffffffffu, end > begin);
                    if (end > begin) part_at[n + __popc(holds & ((1u << lane) - 1u))] = 2 * run + (begin > 0 ? 0 : 1);
                    n += __popc(holds);
                }
                if (n == 1) n = 0;                            // whole after all
                if (lane == 0) {
                    seq = w.seq;
                    tile = w.tile;
                    gk = w.gk;
                }
            }
        } else {
            PromptWalk<false> w;
            w.begin(g, true, n_pairs, lane);
            if (w.find(g, blockIdx.x, lane, true) && w.part == 0) {
                n = w.parts;
                if (lane == 0) {
                    seq = w.seq;
                    tile = w.tile;
                    gk = w.gk;
                }
            }
        }
        if (lane == 0) n_parts = n;
    }
    __syncthreads();
    launch_dependents();
    wait_for_previous_kernel();
    const int parts = n_parts;
    if (parts == 0) return;
    auto first_token = [&](int rank) -> int { return (2 * tile + rank) * g.T; };
    const float2* stats = reinterpret_cast<const float2*>(partial + (size_t)kPromptSlots * 256 * D);
    const int d4 = lane % kLanes;
    for (int r = warp * kRows + lane / kLanes; r < kPromptJoinRows; r += kRows * (kPromptJoinThreads / 32)) {
        const int row = blockIdx.y * kPromptJoinRows + r, rank = row >> 7;
        int tok, head;
        g.div_g.divmod(row & 127, tok, head);
        if (tok >= min(max(seq.nq - first_token(rank), 0), g.T)) continue;
        // statistics and outputs of four parts are asked for together; more are joined to what these gave
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p0 = 0; p0 < parts; p0 += 4) {
            float2 s[4];
            float4 o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int p = min(p0 + i, parts - 1);
                const size_t at = (size_t)(kPaged ? part_at[p] : (int)blockIdx.x + p) * 256 + row;
                s[i] = stats[at];
                o[i] = *reinterpret_cast<const float4*>(partial + at * D + 4 * d4);
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p0 + i < parts && s[i].y != 0.f) top = fmaxf(top, s[i].x);      // (0: the row sees none of the part's keys)
            if (p0 > 0) {
                const MovedBy c(l != 0.f ? m - top : -INFINITY);
                l = c.of(l);
                acc = make_float4(c.of(acc.x), c.of(acc.y), c.of(acc.z), c.of(acc.w));
            }
            m = top;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (p0 + i >= parts || s[i].y == 0.f) continue;
                const float d = s[i].x - m, f = fast_exp2(fmaxf(d, -120.f));
                if (d < -120.f) {                             // rare (two factors, as MovedBy; for every part: 0.9 us more)
                    const float b = fast_exp2(d + 120.f);
                    s[i].y *= b;
                    o[i] = make_float4(o[i].x * b, o[i].y * b, o[i].z * b, o[i].w * b);
                }
                l = fmaf(s[i].y, f, l);
                acc.x = fmaf(o[i].x, f, acc.x);
                acc.y = fmaf(o[i].y, f, acc.y);
                acc.z = fmaf(o[i].z, f, acc.z);
                acc.w = fmaf(o[i].w, f, acc.w);
            }
        }
        const float inv = l != 0.f ? 1.f / l : 0.f;
        const long long at = (long long)(seq.q0 + first_token(rank) + tok) * g.Hq + gk * g.G + head;
        *reinterpret_cast<uint2*>(out + at * D + 4 * d4) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        if (d4 == 0 && lse != nullptr) lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    }
}

}  // namespace adaspark
