// Causal attention of several new tokens per sequence over the pages of its cache, all of it or a window of the last tokens and the first few.
//
//   o_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = 2^(scale_log2 q_i.k_j - m_i),  j <= p_i and (j > p_i - window or j < sinks)
//
// A warp per (token, head), a key at a time.
#pragma once
#include "paged_cache.cuh"

namespace adaspark {

struct ChunkCall {
    const int32_t *cu, *kv_len;
    int batch, n, Hq, G;
    const __nv_bfloat16* q;
    long long q_ts, q_hs;
    float scale_log2;
    int window, sinks;                       // window 0: none
    __nv_bfloat16* out;
    float* lse;
    int32_t* status;
};

constexpr int kChunkWarps = 4;

template <int D, bool kE4m3>
__global__ void __launch_bounds__(kChunkWarps * 32) attn_paged_kernel(PageGeom p, ChunkCall a) {
    constexpr int kPer = D / 32;
    const int lane = threadIdx.x & 31;
    launch_dependents();
    wait_for_previous_kernel();
    const long long item = blockIdx.x * (long long)kChunkWarps + (threadIdx.x >> 5);
    report_bounds(a.cu, a.batch, a.n, a.status);
    if (item >= (long long)a.n * a.Hq) return;
    const int at = (int)(item / a.Hq), head = (int)(item - (long long)at * a.Hq), gk = head / a.G;
    int seq = 0;                             // (one by one: bounds that decrease are those of a sequence left out, not of its neighbours)
    while (seq < a.batch && !(bounds_fit(a.cu[seq], a.cu[seq + 1], a.n) && a.cu[seq] <= at && at < a.cu[seq + 1])) ++seq;
    if (seq == a.batch) return;
    const int len = a.kv_len[seq], pos = len - (a.cu[seq + 1] - at);
    const bool fits = len >= 0 && len <= (p.table_width << p.page_shift);
    bool bad = !fits || pos < 0;
    float q[kPer], o[kPer], m = -INFINITY, l = 0.f;
    for (int i = 0; i < kPer; ++i) {
        q[i] = __bfloat162float(a.q[at * a.q_ts + head * a.q_hs + lane * kPer + i]) * a.scale_log2;
        o[i] = 0.f;
    }
    const int from = a.window > 0 ? max(pos + 1 - a.window, 0) : 0;
    for (int j = a.window > 0 && a.sinks > 0 ? 0 : from; fits && j <= pos; ++j) {
        if (j >= a.sinks && j < from) j = from;
        const long long page = page_of(p, seq, j);
        if (page < 0) bad = true;
        const int in = j & ((1 << p.page_shift) - 1);
        const long long row = ((long long)gk << p.page_shift) + in, x = page * p.page_stride + row * D + lane * kPer;
        float k[kPer], v[kPer], s = 0.f;
        for (int i = 0; i < kPer; ++i) {
            k[i] = v[i] = 0.f;
            if (page >= 0) {
                if (kE4m3) {
                    const long long sx = page * p.scale_stride + row;
                    const uint32_t two = codes_to_f16x2((uint32_t)p.k[x + i] | ((uint32_t)p.v[x + i] << 8));
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&two));
                    k[i] = f.x * pow2_of_byte(p.ks[sx]);
                    v[i] = f.y * pow2_of_byte(p.vs[sx]);
                } else {
                    k[i] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.k)[x + i]);
                    v[i] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p.v)[x + i]);
                }
            }
            s = fmaf(q[i], k[i], s);
        }
        for (int b = 16; b > 0; b >>= 1) s += __shfl_xor_sync(0xffffffffu, s, b);
        const float top = fmaxf(m, s), ref = top == -INFINITY ? 0.f : top;
        const float c = m == -INFINITY ? 0.f : fast_exp2(m - ref), w = fast_exp2(s - ref);
        m = top;
        l = l * c + w;
        for (int i = 0; i < kPer; ++i) o[i] = fmaf(w, v[i], o[i] * c);
    }
    const size_t row = (size_t)at * a.Hq + head;
    for (int i = 0; i < kPer; ++i) a.out[row * D + lane * kPer + i] = __float2bfloat16(l != 0.f ? o[i] / l : 0.f);
    if (lane == 0 && a.lse != nullptr) a.lse[row] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
    if (lane == 0 && bad && a.status != nullptr) atomicExch(a.status, 1);
}

}  // namespace adaspark
