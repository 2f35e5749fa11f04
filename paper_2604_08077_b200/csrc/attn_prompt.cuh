// Causal attention of whole prompts, packed one behind the other: a warp per (row, query head).
#pragma once
#include "common.cuh"

namespace adaspark {

// Row i of a sequence with n_q rows and n_k keys sees the keys 0 .. n_k - n_q + i.
template <int D>
__global__ void __launch_bounds__(128) attn_prompt_kernel(const __nv_bfloat16* q, long long q_ts, long long q_hs, const __nv_bfloat16* k, long long k_ts,
                                                          long long k_hs, const __nv_bfloat16* v, long long v_ts, long long v_hs, const int32_t* cu_q,
                                                          const int32_t* cu_k, int batch, int n_q, int n_k, int Hq, int G, float scale_log2,
                                                          __nv_bfloat16* out, float* lse, int32_t* status) {
    constexpr int kPer = D / 32;
    launch_dependents();
    wait_for_previous_kernel();
    const long long w = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, row = (int)(w / Hq), h = (int)(w % Hq), gk = h / G;
    if (row >= n_q) return;
    int seq = -1;
    for (int i = 0; i < batch; ++i) {
        const bool valid = 0 <= cu_q[i] && cu_q[i] <= cu_q[i + 1] && cu_q[i + 1] <= n_q && 0 <= cu_k[i] && cu_k[i] <= cu_k[i + 1] && cu_k[i + 1] <= n_k;
        if (!valid && status != nullptr) atomicExch(status, 1);
        if (valid && row >= cu_q[i] && row < cu_q[i + 1]) seq = i;
    }
    if (seq < 0) return;
    const int k0 = cu_k[seq], last = (cu_k[seq + 1] - k0) - (cu_q[seq + 1] - cu_q[seq]) + (row - cu_q[seq]);
    float qv[kPer], o[kPer], m = -INFINITY, l = 0.f;
    for (int e = 0; e < kPer; ++e) {
        qv[e] = __bfloat162float(q[row * q_ts + h * q_hs + lane * kPer + e]);
        o[e] = 0.f;
    }
    for (int j = 0; j <= last; ++j) {
        const __nv_bfloat16* kr = k + (long long)(k0 + j) * k_ts + gk * k_hs + lane * kPer;
        const __nv_bfloat16* vr = v + (long long)(k0 + j) * v_ts + gk * v_hs + lane * kPer;
        float s = 0.f;
        for (int e = 0; e < kPer; ++e) s = fmaf(qv[e], __bfloat162float(kr[e]), s);
        for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale_log2;
        const float m_new = fmaxf(m, s), corr = exp2f(m - m_new), p = exp2f(s - m_new);
        l = l * corr + p;
        for (int e = 0; e < kPer; ++e) o[e] = o[e] * corr + p * __bfloat162float(vr[e]);
        m = m_new;
    }
    for (int e = 0; e < kPer; ++e) out[((long long)row * Hq + h) * D + lane * kPer + e] = __float2bfloat16(last >= 0 ? o[e] / l : 0.f);
    if (lse != nullptr && lane == 0) lse[(long long)row * Hq + h] = last >= 0 ? (m + log2f(l)) * 0.69314718056f : -INFINITY;
}

}  // namespace adaspark
