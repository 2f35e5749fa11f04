// Attention of one new token per sequence over the pages of its cache: a warp per (sequence, query head).
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"

namespace adaspark {

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

template <int D, bool kE4m3>
__global__ void __launch_bounds__(64) paged_append_kernel(PageGeom p, const __nv_bfloat16* k, long long k_ts, long long k_hs, const __nv_bfloat16* v,
                                                          long long v_ts, long long v_hs, const int32_t* kv_len, int32_t* status) {
    launch_dependents();
    wait_for_previous_kernel();
    const int b = blockIdx.y, h = blockIdx.x, n = kv_len[b], w = threadIdx.x >> 5;
    if (n <= 0) return;
    const int page = (int)page_of(p, b, n - 1);
    if (page < 0) return;
    append_row<D, kE4m3>(p, page, h, (n - 1) & ((1 << p.page_shift) - 1), w, w ? v + b * v_ts + h * v_hs : k + b * k_ts + h * k_hs, threadIdx.x & 31);
}

template <int D, bool kE4m3>
__global__ void __launch_bounds__(32) paged_decode_kernel(PageGeom p, const __nv_bfloat16* q, long long q_ts, long long q_hs, const int32_t* kv_len, int Hq,
                                                          int G, float scale_log2, __nv_bfloat16* out, float* lse, int32_t* status) {
    constexpr int kPer = D / 32;
    launch_dependents();
    wait_for_previous_kernel();
    const int b = blockIdx.y, h = blockIdx.x, gk = h / G, lane = threadIdx.x, n = kv_len[b];
    float qv[kPer], o[kPer], m = -INFINITY, l = 0.f;
    for (int e = 0; e < kPer; ++e) {
        qv[e] = __bfloat162float(q[b * q_ts + h * q_hs + lane * kPer + e]);
        o[e] = 0.f;
    }
    bool bad = n < 0 || n > (p.table_width << p.page_shift);
    for (int j = 0; j < n && !bad; ++j) {
        const int page = (int)page_of(p, b, j);
        if (page < 0) { bad = true; break; }
        const long long row = ((long long)gk << p.page_shift) + (j & ((1 << p.page_shift) - 1));
        float kx[kPer], vx[kPer];
        for (int e = 0; e < kPer; ++e) {
            const long long at = (long long)page * p.page_stride + row * D + lane * kPer + e;
            if (kE4m3) {
                __half_raw a = __half_raw(), c = __half_raw();
                a.x = (unsigned short)codes_to_f16x2(p.k[at]);
                c.x = (unsigned short)codes_to_f16x2(p.v[at]);
                kx[e] = __half2float(__half(a)) * pow2_of_byte(p.ks[(long long)page * p.scale_stride + row]);
                vx[e] = __half2float(__half(c)) * pow2_of_byte(p.vs[(long long)page * p.scale_stride + row]);
            } else {
                kx[e] = __bfloat162float(((const __nv_bfloat16*)p.k)[at]);
                vx[e] = __bfloat162float(((const __nv_bfloat16*)p.v)[at]);
            }
        }
        float s = 0.f;
        for (int e = 0; e < kPer; ++e) s = fmaf(qv[e], kx[e], s);
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale_log2;
        const float m_new = fmaxf(m, s), corr = exp2f(m - m_new), w = exp2f(s - m_new);
        l = l * corr + w;
        for (int e = 0; e < kPer; ++e) o[e] = o[e] * corr + w * vx[e];
        m = m_new;
    }
    if (bad && status != nullptr && lane == 0) atomicExch(status, 1);
    const bool none = bad || n <= 0;
    for (int e = 0; e < kPer; ++e) out[((long long)b * Hq + h) * D + lane * kPer + e] = __float2bfloat16(none ? 0.f : o[e] / l);
    if (lse != nullptr && lane == 0) lse[(long long)b * Hq + h] = none ? -INFINITY : (m + log2f(l)) * 0.69314718056f;
}

}  // namespace adaspark
