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

// The byte of the power of two for the largest magnitude `top` (bf16 bits without the sign, finite) of a row.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int s = (int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);      // 448 = 1.75 * 2^8, 0x60: the .75
    return (uint32_t)max(s, 0);
}

// 8 bf16 -> the largest finite magnitude, as bf16 bits; `odd` is set where one is infinite or no number.
__device__ __forceinline__ uint32_t chunk_top(const uint4& x, bool& odd) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t m = 0;
    odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = w[i] & 0x7fff7fffu;
        m = __vmaxu2(m, a);
    }
    uint32_t top = max(m & 0xffffu, m >> 16);
    if (top >= 0x7f80u) {                                                     // rare
        odd = true;
        top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            for (int e = 0; e < 2; ++e) {
                const uint32_t a = (w[i] >> (16 * e)) & 0x7fffu;
                if (a < 0x7f80u) top = max(top, a);
            }
    }
    return top;
}
// 8 bf16 times 2^(127 - s) -> 8 codes.  What is infinite or no number becomes e4m3's NaN: it has no infinity, and a saturated 448
// would pass for a value.
__device__ __forceinline__ uint2 chunk_codes(const uint4& x, uint32_t s, bool odd) {
    const float inv = __uint_as_float((254u - s) << 23);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo = __uint_as_float(w[i] << 16) * inv, hi = __uint_as_float(w[i] & 0xffff0000u) * inv;
        if (odd) {
            if ((w[i] & 0x7f80u) == 0x7f80u) lo = NAN;
            if ((w[i] & 0x7f800000u) == 0x7f800000u) hi = NAN;
        }
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(hi), "f"(lo));
        c[i] = two;
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
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
// the first sequence or behind the last one).
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

constexpr int kCacheTokens = 8;      // tokens of a CTA
constexpr int kCacheThreads = 256;

// Page and place of the CTA's tokens, by its first threads: page in [0, n_pages) or -1 (not ours), place in the page.
__device__ __forceinline__ void find_tokens(const PageGeom& p, const int32_t* cu, const int32_t* kv_len, int batch, int n, int t0,
                                            int (&page)[kCacheTokens], int (&place)[kCacheTokens], int32_t* status) {
    if (threadIdx.x < kCacheTokens) {
        const int at = t0 + threadIdx.x;
        int pg = -1, pl = 0;
        const int seq = at < n ? sequence_of(cu, batch, at) : -1;
        if (seq >= 0) {
            const int pos = kv_len[seq] - (cu[seq + 1] - at);
            pg = (int)page_of(p, seq, pos);
            pl = pos & ((1 << p.page_shift) - 1);
            if (pg < 0) {
                pg = -2;                                                      // a row of a sequence that has no place for it
                if (status != nullptr) atomicExch(status, 1);
            }
        }
        page[threadIdx.x] = pg;
        place[threadIdx.x] = pl;
    }
}

// k, v [n][Hkv][D] (row and head strides in elements) -> pages.  Bound by HBM: every value read once and written once.  A thread takes
// 16 bytes (8 values) at a time, D / 8 neighbouring threads a row, whose largest magnitude they find by shuffles; the loads of a
// thread are under way before its CTA has looked up where they go.
template <int D, bool kE4m3>
__global__ void __launch_bounds__(kCacheThreads) paged_write_kernel(
    PageGeom p, const __nv_bfloat16* k, long long k_ts, long long k_hs, const __nv_bfloat16* v, long long v_ts, long long v_hs,
    const int32_t* cu, const int32_t* kv_len, int batch, int n, FastDiv div_rows, FastDiv div_heads, int32_t* status) {
    constexpr int kLanes = D / 8, kBatch = 4;
    __shared__ int page[kCacheTokens], place[kCacheTokens];
    const int t0 = blockIdx.x * kCacheTokens;
    launch_dependents();
    wait_for_previous_kernel();
    const int n_chunks = kCacheTokens * 2 * p.Hkv * kLanes;                   // (a multiple of a warp)
    bool looked = false;
    for (int c0 = threadIdx.x; c0 < n_chunks; c0 += kBatch * kCacheThreads) {
        uint4 x[kBatch];
        int tok[kBatch], head[kBatch], is_v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int c = c0 + i * kCacheThreads, row = c / kLanes, d = (c % kLanes) * 8;
            int r, w, h;
            div_rows.divmod(row, r, w);                                       // [token][k, v][head]
            div_heads.divmod(w, w, h);
            tok[i] = r;
            head[i] = h;
            is_v[i] = w;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (c < n_chunks && t0 + r < n) {
                const __nv_bfloat16* src = w ? v + (long long)(t0 + r) * v_ts + h * v_hs : k + (long long)(t0 + r) * k_ts + h * k_hs;
                x[i] = *reinterpret_cast<const uint4*>(src + d);
            }
        }
        if (!looked) {
            find_tokens(p, cu, kv_len, batch, n, t0, page, place, status);
            __syncthreads();
            looked = true;
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int c = c0 + i * kCacheThreads, part = c % kLanes;
            if (c - (int)(threadIdx.x & 31) >= n_chunks) break;               // (the same for the whole warp)
            const int pg = page[tok[i]];
            const long long row = ((long long)head[i] << p.page_shift) + place[tok[i]];
            if (kE4m3) {
                bool odd;
                uint32_t top = chunk_top(x[i], odd);
#pragma unroll
                for (int s = 1; s < kLanes; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
                const uint32_t s = scale_byte(top);
                if (pg >= 0) {
                    uint8_t* dst = (is_v[i] ? p.v : p.k) + (long long)pg * p.page_stride + row * D + part * 8;
                    *reinterpret_cast<uint2*>(dst) = chunk_codes(x[i], s, odd);
                    if (part == 0) (is_v[i] ? p.vs : p.ks)[(long long)pg * p.scale_stride + row] = (uint8_t)s;
                }
            } else if (pg >= 0) {
                uint8_t* dst = (is_v[i] ? p.v : p.k) + ((long long)pg * p.page_stride + row * D + part * 8) * 2;
                *reinterpret_cast<uint4*>(dst) = x[i];
            }
        }
    }
}

// pages -> k_out, v_out [n][Hkv][D] bf16 (row and head strides in elements).  Rows of no sequence are left as they are; rows of a sequence that have no place in
// its pages read as zeros.
template <int D, bool kE4m3>
__global__ void __launch_bounds__(kCacheThreads) paged_read_kernel(
    PageGeom p, __nv_bfloat16* k_out, long long k_ts, long long k_hs, __nv_bfloat16* v_out, long long v_ts, long long v_hs, const int32_t* cu,
    const int32_t* kv_len, int batch, int n, FastDiv div_rows, FastDiv div_heads, int32_t* status) {
    constexpr int kLanes = D / 8, kBatch = 4;
    __shared__ int page[kCacheTokens], place[kCacheTokens];
    const int t0 = blockIdx.x * kCacheTokens;
    launch_dependents();
    wait_for_previous_kernel();
    const int n_chunks = kCacheTokens * 2 * p.Hkv * kLanes;
    find_tokens(p, cu, kv_len, batch, n, t0, page, place, status);
    __syncthreads();
    for (int c0 = threadIdx.x; c0 < n_chunks; c0 += kBatch * kCacheThreads) {
        uint4 x[kBatch];
        uint32_t s[kBatch];
        __nv_bfloat16* dst[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int c = c0 + i * kCacheThreads, row = c / kLanes, part = c % kLanes;
            int r, w, h;
            div_rows.divmod(row, r, w);
            div_heads.divmod(w, w, h);
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            s[i] = 0;
            dst[i] = nullptr;
            if (c < n_chunks && page[r] != -1) {
                const int pg = page[r];
                dst[i] = (w ? v_out + (long long)(t0 + r) * v_ts + h * v_hs : k_out + (long long)(t0 + r) * k_ts + h * k_hs) + part * 8;
                if (pg >= 0) {
                    const long long at = ((long long)h << p.page_shift) + place[r];
                    if (kE4m3) {
                        const uint2 cc = *reinterpret_cast<const uint2*>((w ? p.v : p.k) + (long long)pg * p.page_stride + at * D + part * 8);
                        x[i].x = cc.x;
                        x[i].y = cc.y;
                        s[i] = (w ? p.vs : p.ks)[(long long)pg * p.scale_stride + at];
                    } else {
                        x[i] = *reinterpret_cast<const uint4*>((w ? p.v : p.k) + ((long long)pg * p.page_stride + at * D + part * 8) * 2);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (dst[i] != nullptr) *reinterpret_cast<uint4*>(dst[i]) = kE4m3 ? chunk_values(make_uint2(x[i].x, x[i].y), s[i]) : x[i];
    }
}

}  // namespace adaspark
