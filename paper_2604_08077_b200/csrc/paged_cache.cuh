// The paged cache of the text operators: new keys and values written into their pages, as bf16 or as 8-bit floats, and
// read back.
//
// A page holds page_size tokens of one sequence: [kv head][slot][d], so that what an attention step reads of one head is one
// run of memory.  In 8 bits a row x of D values is stored as e4m3 codes c and one byte s, x ~ c * 2^(s - 127): s is the smallest
// for which max|x| <= 448 * 2^(s - 127).  The scale is a power of two because then nothing but the one rounding to e4m3 (off by
// at most 2^-4 of the value, or half of e4m3's smallest step, 2^-10 * 2^(s - 127)) is ever lost: scaling is exact, and
// every stored value is a bf16 number, so reading back rounds nothing and the tensor cores take what the cache holds.  (A scale of
// max|x| / 448 would win at most one binade at the small end and would round again at each of those places.)
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace adaspark {

// A paged cache as the kernels see it.  Offsets are in elements and 64 bits wide: a pool may hold more than 2^31 of them.
struct PageGeom {
    uint8_t *k, *v;                 // pages
    uint8_t *ks, *vs;               // bytes of the powers of two (e4m3), else null
    long long page_stride;          // elements from page to page
    long long scale_stride;         // bytes from page to page
    const int32_t* table;           // [batch][table_width] page numbers
    int table_width, n_pages;
    int page_shift;                 // log2(page_size)
    int Hkv;
};

// Place of token `pos` of sequence `seq` in its page, or -1: no such place (nothing is read or written there then).
__device__ __forceinline__ long long page_of(const PageGeom& p, int seq, int pos) {
    const int col = pos >> p.page_shift;
    if (pos < 0 || col >= p.table_width) return -1;
    const int page = p.table[(size_t)seq * p.table_width + col];
    return page >= 0 && page < p.n_pages ? page : -1;
}

// 2^(s - 127), s in 0 .. 254
__device__ __forceinline__ float pow2_of_byte(uint32_t s) { return __uint_as_float(s == 0 ? 0x00400000u : s << 23); }

// The byte of the power of two for the largest magnitude `top` (bf16 bits without the sign, finite) of a row: 448 = 1.75 * 2^8, and 0x1f
// carries into the exponent from the first mantissa above .75 on.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) { return (uint32_t)max((int)((top + 0x1fu) >> 7) - 8, 0); }

// 8 bf16 -> the larger of each pair's halves' magnitudes, as two bf16 without sign
__device__ __forceinline__ uint32_t chunk_tops(const uint4& x) {
    return __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
}
// The same over the finite ones alone (infinite or no number: exponent bits all ones).
__device__ __forceinline__ uint32_t chunk_finite_tops(const uint4& x) {
    const uint32_t w[4] = {x.x & 0x7fff7fffu, x.y & 0x7fff7fffu, x.z & 0x7fff7fffu, x.w & 0x7fff7fffu};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & __vcmpltu2(w[i], 0x7f807f80u));
    return m;
}
// Largest magnitudes of two rows (their D / 8 lanes hold a and b), in the halves of the result; every lane of the warp takes part.
template <int kLanes>
__device__ __forceinline__ uint32_t row_tops(uint32_t a, uint32_t b) {
    uint32_t t = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
    for (int s = 1; s < kLanes; s <<= 1) t = __vmaxu2(t, __shfl_xor_sync(0xffffffffu, t, s));
    return t;
}
__device__ __forceinline__ bool any_odd(uint32_t tops) { return (tops & 0xffffu) >= 0x7f80u || (tops >> 16) >= 0x7f80u; }
// 8 bf16 times 2^(127 - s) -> 8 codes
__device__ __forceinline__ uint2 chunk_codes(const uint4& x, uint32_t s) {
    const float inv = __uint_as_float((254u - s) << 23);
    const unsigned long long inv2 = pack_f32x2(inv, inv);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), inv2), lo, hi);
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(hi), "f"(lo));
        c[i] = two;
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
// What is infinite becomes NaN: e4m3 has no infinity, and a saturated 448 would pass for a value.
__device__ __forceinline__ uint4 infinities_to_nan(const uint4& x) {
    uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] |= __vcmpgeu2(w[i] & 0x7fff7fffu, 0x7f807f80u) & 0x007f007fu;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// two codes (low 16 bits) -> f16 pair: exact
__device__ __forceinline__ uint32_t codes_to_f16x2(uint32_t two) {
    uint32_t r;
    asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}\n" : "=r"(r) : "r"(two));
    return r;
}
// 8 codes times 2^(s - 127) -> 8 bf16: exact
__device__ __forceinline__ uint4 chunk_values(const uint2& c, uint32_t s) {
    const float f = pow2_of_byte(s);
    const uint32_t h[4] = {codes_to_f16x2(c.x & 0xffffu), codes_to_f16x2(c.x >> 16), codes_to_f16x2(c.y & 0xffffu), codes_to_f16x2(c.y >> 16)};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        r[i] = pack_bf16x2(v.x * f, v.y * f);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

// The sequence that row `at` of the packed tensors belongs to: the last one with cu[seq] <= at, or -1 (rows in front of
// the first sequence or behind the last one).  If cu decreases somewhere, some sequence with cu[seq] <= at < cu[seq + 1], or -1.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int at) {
    if (at < cu[0] || at >= cu[batch]) return -1;
    int lo = 0, hi = batch;                                                   // cu[lo] <= at < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= at) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Are these the first row and the one behind the last of a sequence in tensors of n rows?
__device__ __forceinline__ bool bounds_fit(int begin, int end, int n) { return 0 <= begin && begin <= end && end <= n; }

constexpr int kCacheThreads = 256;

// Places of the CTA's kTokens tokens from t0 on, by its first threads: offsets (elements, scales) of a token's first kv head in the pages;
// first < 0: -1 a row of no sequence, -2 one of a sequence that has no place for it, or whose bounds are none.
template <int kTokens, int D>
__device__ __forceinline__ void find_tokens(const PageGeom& p, const int32_t* cu, const int32_t* kv_len, int batch, int n, int t0, long long (&place)[kTokens],
                                            long long (&scale_place)[kTokens], int32_t* status) {
    for (int i = threadIdx.x; i < kTokens; i += kCacheThreads) {
        const int at = t0 + i;
        long long x = -1, y = 0;
        const int seq = at < n ? sequence_of(cu, batch, at) : -1;
        if (seq >= 0) {
            const int len = kv_len[seq], end = cu[seq + 1];
            const int pos = len > 0 ? len - (end - at) : -1, in = pos & ((1 << p.page_shift) - 1);
            const long long page = bounds_fit(cu[seq], end, n) ? page_of(p, seq, pos) : -1;
            if (page < 0) {
                x = -2;
                if (status != nullptr) atomicExch(status, 1);
            } else {
                x = page * p.page_stride + (long long)in * D;
                y = page * p.scale_stride + in;
            }
        }
        place[i] = x;
        scale_place[i] = y;
    }
}

// A sequence with bad bounds may have no row in the tensors (all of it behind them): the CTAs share the batch out among them and look at every
// sequence's.  (Behind the copies: in front of them it took registers that left room for a CTA less, 157 instead of 146 us for 131072 tokens
// written and read in 8 bits; hence the bound of 4 CTAs on both kernels, too.)
__device__ __forceinline__ void report_bounds(const int32_t* cu, int batch, int n, int32_t* status) {
    if (status == nullptr || blockIdx.y != 0) return;
    for (long long b = blockIdx.x * (long long)kCacheThreads + threadIdx.x; b < batch; b += gridDim.x * (long long)kCacheThreads)
        if (!bounds_fit(cu[b], cu[b + 1], n)) atomicExch(status, 1);
}

// Both kernels: a CTA has kTokens tokens, a thread one 16-byte piece (8 values) of a row of one head of K or V and every
// kCacheThreads / columns-th token: what belongs to the column is worked out once, a token costs an offset from shared memory.  Bound by HBM, every
// value read once and written once.  (With the pieces of 8 tokens dealt to the threads one by one, index arithmetic took the issue slots: 131072 tokens, 4
// heads of 128, 8 bits: 107 us written and 88 read.)  grid (tokens / kTokens, columns / 256).

// k, v [n][Hkv][D] (row and head strides in elements) -> pages.  D / 8 neighbouring threads find a row's largest magnitude by shuffles; the
// first loads of a thread are under way before its CTA has looked up where they go.
template <int D, bool kE4m3, int kTokens>
__global__ void __launch_bounds__(kCacheThreads, 4) paged_write_kernel(
    PageGeom p, const __nv_bfloat16* k, long long k_ts, long long k_hs, const __nv_bfloat16* v, long long v_ts, long long v_hs,
    const int32_t* cu, const int32_t* kv_len, int batch, int n, int32_t* status) {
    constexpr int kLanes = D / 8, kAhead = 4;
    __shared__ long long place[kTokens], scale_place[kTokens];
    const int t0 = blockIdx.x * kTokens, cols = 2 * p.Hkv * kLanes, col0 = blockIdx.y * kCacheThreads, width = min(cols - col0, kCacheThreads);
    const int tokens = kCacheThreads / width, mine = (int)threadIdx.x / width;             // of a pass, of this thread
    const int col = col0 + (int)threadIdx.x - mine * width, row = col / kLanes, part = col % kLanes;
    const bool is_v = row >= p.Hkv;
    const int head = is_v ? row - p.Hkv : row;
    const long long ts = is_v ? v_ts : k_ts;
    const __nv_bfloat16* src = (is_v ? v + head * v_hs : k + head * k_hs) + part * 8 + t0 * ts;
    uint8_t* dst = (is_v ? p.v : p.k) + (((long long)head << p.page_shift) * D + part * 8) * (kE4m3 ? 1 : 2);
    uint8_t* scales = (is_v ? p.vs : p.ks) + ((long long)head << p.page_shift);
    const int count = mine < tokens ? min(kTokens, n - t0) : 0;
    launch_dependents();
    wait_for_previous_kernel();
    bool looked = false;
    for (int pass = 0; pass < kTokens; pass += kAhead * tokens) {   // (as often for every thread: the shuffles and the barrier need all of them)
        const int t = pass + mine;
        uint4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = t + i * tokens < count ? *reinterpret_cast<const uint4*>(src + (t + i * tokens) * ts) : make_uint4(0u, 0u, 0u, 0u);
        if (!looked) {
            find_tokens<kTokens, D>(p, cu, kv_len, batch, n, t0, place, scale_place, status);
            __syncthreads();
            looked = true;
        }
#pragma unroll
        for (int i = 0; i < kAhead; i += 2) {                 // two rows at a time
            uint32_t tops = 0u;
            if (kE4m3) {
                tops = row_tops<kLanes>(chunk_tops(x[i]), chunk_tops(x[i + 1]));
                if (__any_sync(0xffffffffu, any_odd(tops))) { // rare
                    tops = row_tops<kLanes>(chunk_finite_tops(x[i]), chunk_finite_tops(x[i + 1]));
                    x[i] = infinities_to_nan(x[i]);
                    x[i + 1] = infinities_to_nan(x[i + 1]);
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int tt = t + (i + y) * tokens;
                const long long at = tt < count ? place[tt] : -1;
                if (at < 0) continue;
                if (kE4m3) {
                    const uint32_t s = scale_byte(y ? tops >> 16 : tops & 0xffffu);
                    *reinterpret_cast<uint2*>(dst + at) = chunk_codes(x[i + y], s);
                    if (part == 0) scales[scale_place[tt]] = (uint8_t)s;
                } else {
                    *reinterpret_cast<uint4*>(dst + at * 2) = x[i + y];
                }
            }
        }
    }
    report_bounds(cu, batch, n, status);
}

// pages -> k_out, v_out [n][Hkv][D] bf16 (row and head strides in elements).  Rows of no sequence are left as they are; rows of a sequence that
// have no place in its pages read as zeros.
template <int D, bool kE4m3, int kTokens>
__global__ void __launch_bounds__(kCacheThreads, 4) paged_read_kernel(
    PageGeom p, __nv_bfloat16* k_out, long long k_ts, long long k_hs, __nv_bfloat16* v_out, long long v_ts, long long v_hs, const int32_t* cu,
    const int32_t* kv_len, int batch, int n, int32_t* status) {
    constexpr int kLanes = D / 8, kAhead = kE4m3 ? 8 : 4;
    __shared__ long long place[kTokens], scale_place[kTokens];
    const int t0 = blockIdx.x * kTokens, cols = 2 * p.Hkv * kLanes, col0 = blockIdx.y * kCacheThreads, width = min(cols - col0, kCacheThreads);
    const int tokens = kCacheThreads / width, mine = (int)threadIdx.x / width;
    const int col = col0 + (int)threadIdx.x - mine * width, row = col / kLanes, part = col % kLanes;
    const bool is_v = row >= p.Hkv;
    const int head = is_v ? row - p.Hkv : row;
    const long long ts = is_v ? v_ts : k_ts;
    __nv_bfloat16* dst = (is_v ? v_out + head * v_hs : k_out + head * k_hs) + part * 8 + t0 * ts;
    const uint8_t* src = (is_v ? p.v : p.k) + (((long long)head << p.page_shift) * D + part * 8) * (kE4m3 ? 1 : 2);
    const uint8_t* scales = (is_v ? p.vs : p.ks) + ((long long)head << p.page_shift);
    const int count = mine < tokens ? min(kTokens, n - t0) : 0;
    launch_dependents();
    wait_for_previous_kernel();
    find_tokens<kTokens, D>(p, cu, kv_len, batch, n, t0, place, scale_place, status);
    __syncthreads();
    for (int t = mine; t < count; t += kAhead * tokens) {
        uint4 x[kAhead];
        uint32_t s[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tt = t + i * tokens;
            const long long at = tt < count ? place[tt] : -1;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            s[i] = 0u;
            if (at >= 0) {
                if (kE4m3) {
                    const uint2 c = *reinterpret_cast<const uint2*>(src + at);
                    x[i].x = c.x;
                    x[i].y = c.y;
                    s[i] = scales[scale_place[tt]];
                } else {
                    x[i] = *reinterpret_cast<const uint4*>(src + at * 2);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int tt = t + i * tokens;
            if (tt < count && place[tt] != -1) *reinterpret_cast<uint4*>(dst + tt * ts) = kE4m3 ? chunk_values(make_uint2(x[i].x, x[i].y), s[i]) : x[i];
        }
    }
    report_bounds(cu, batch, n, status);
}

}  // namespace adaspark
