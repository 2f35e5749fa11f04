// Queries and keys between the projection and the attention: each head divided by the root of its mean square (where the model does
// so) and rotated by its token's positions; on request straight into the pages of a cache, with the values beside them.
//
//   y = x / sqrt(mean x^2 + eps) * w;   pair i of a head, (a, b):  (a cos t - b sin t, b cos t + a sin t),  t = position[axis_i] * f_i
//
// Pairs are the values (i, i + pairs) of a head or its neighbours (2 i, 2 i + 1); values behind the 2 * pairs first ones are not rotated.
// Everything is computed in 32 bits and rounded once, keys for 8-bit pages from 32 bits to their codes, too.
//
// Angles are counted in whole turns as 64-bit fixed point: f_i / 2 pi * 2^64 times the position, modulo 2^64, is the angle's place in its turn
// with 2^-33 of a turn at positions of 31 bits, without a division, a reduction or a number of 64 bits in floating point; the signed rest is
// a 32-bit float of half turns, relative to whose size nothing is lost.
//
// Bound by HBM: every row is read once and written once.  A group of D / 16 threads takes a row at a time, 16 values each: the
// chunks of 8 that are rotated into one another.  A group stays with one token: its cosines and sines (worked out once for all heads of a
// token, through shared memory) and the weights of the norms stay in registers.
#pragma once
#include "common.cuh"
#include "paged_cache.cuh"

namespace adaspark {

constexpr int kRotaryPairs = 64;

struct RowsIn {
    const __nv_bfloat16* p;
    long long ts, hs;
};
struct RowsOut {
    __nv_bfloat16* p;
    long long ts, hs;
};

// What one call works on.
struct RotateCall {
    RowsIn q, k, v;                 // v: pages alone
    RowsOut q_out, k_out;           // k_out: without pages
    const __nv_bfloat16 *q_norm, *k_norm;
    const int32_t* positions;       // [axes][n]; null: the place in the sequence (pages alone)
    const int32_t *cu, *kv_len;     // pages alone
    int32_t* status;
    int n, batch, Hq, Hkv;          // Hq, Hkv 0: no such rows
    float eps;
    int pairs, adjacent;
    uint64_t turns[kRotaryPairs];   // of pair i per position: of a whole turn, times 2^64
    uint8_t axis[kRotaryPairs];
};

// Cosine and sine of a place in a turn (64-bit fixed point)
__device__ __forceinline__ float2 turned_by(uint64_t turn) {
    float2 r;
    sincospif((float)(long long)turn * 0x1p-63f, &r.y, &r.x);
    return r;
}

// 8 bf16 -> 8 numbers
__device__ __forceinline__ void unpack_chunk(const uint4& c, float* x) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack_chunk(const float* x) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
// 8 numbers times 2^(127 - s) -> 8 codes
__device__ __forceinline__ uint2 pack_codes(const float* x, uint32_t s) {
    const float inv = __uint_as_float((254u - s) << 23);
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(two) : "f"(x[2 * i + 1] * inv), "f"(x[2 * i] * inv));
        c[i] = two;
    }
    return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

constexpr int kRotateThreads = kCacheThreads;

// kPages: 0 rows out; 1, 2 keys and values into pages of bf16, e4m3.  grid (tokens / kTokens).
template <int D, int kPages, int kTokens>
__global__ void __launch_bounds__(kRotateThreads, 3) rotate_kernel(const __grid_constant__ RotateCall a, const __grid_constant__ PageGeom p) {
    constexpr int kLanes = D / 16, kGroups = kRotateThreads / kLanes / kTokens;     // of a token
    __shared__ float2 turn[kTokens][kRotaryPairs + 2];        // (a row of neighbours' chunks of 64 bytes each starts in another bank)
    __shared__ TokenPlace place[kTokens];
    const int tid = threadIdx.x, t0 = blockIdx.x * kTokens;
    launch_dependents();
    wait_for_previous_kernel();
    if (kPages) {
        if (tid < kTokens) place[tid] = place_of<D>(p, a.cu, a.kv_len, a.batch, a.n, t0 + tid, a.status);
        if (a.positions == nullptr) __syncthreads();
    }
    for (int i = tid; i < kTokens * a.pairs; i += kRotateThreads) {
        const int t = i / a.pairs, x = i - t * a.pairs;
        if (t0 + t >= a.n) break;
        const int pos = kPages && a.positions == nullptr ? place[t].pos : a.positions[(size_t)a.axis[x] * a.n + t0 + t];
        turn[t][x] = turned_by((uint64_t)(long long)pos * a.turns[x]);
    }
    __syncthreads();
    const int group = tid / kLanes, l = tid % kLanes, t = group / kGroups, at = t0 + t;
    // this thread's two chunks of a row, and whether they are rotated
    const int pc = a.pairs / 8;
    const bool halves = !a.adjacent && l < pc;
    const int c0 = a.adjacent ? l : halves ? l : 2 * l, c1 = a.adjacent ? l + kLanes : halves ? l + pc : 2 * l + 1;
    float2 cs[8];                                             // halves: of the pairs 8 l ..; neighbours: of 4 in either chunk
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        cs[i] = make_float2(1.f, 0.f);
        if (a.adjacent) {
            const int x = (i < 4 ? c0 : c1) * 4 + (i & 3);
            if (x < a.pairs) cs[i] = turn[t][x];
        } else if (halves) {
            cs[i] = turn[t][l * 8 + i];
        }
    }
    bool mine = at < a.n, there = true;
    if (kPages && mine) {
        mine = place[t].first != -1;
        there = place[t].first >= 0;
    }
    const int rows = a.Hq + a.Hkv + (kPages ? a.Hkv : 0);
    const uint4 one = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
    uint4 wq[2] = {one, one}, wk[2] = {one, one};
    if (a.q_norm != nullptr) {
        wq[0] = *reinterpret_cast<const uint4*>(a.q_norm + c0 * 8);
        wq[1] = *reinterpret_cast<const uint4*>(a.q_norm + c1 * 8);
    }
    if (a.k_norm != nullptr) {
        wk[0] = *reinterpret_cast<const uint4*>(a.k_norm + c0 * 8);
        wk[1] = *reinterpret_cast<const uint4*>(a.k_norm + c1 * 8);
    }
    constexpr int kAhead = 2;
    // (as often for every thread: the shuffles need all of a warp)
    for (int r0 = 0; r0 < rows; r0 += kGroups * kAhead) {
        uint4 in[kAhead][2];
#pragma unroll
        for (int y = 0; y < kAhead; ++y) {
            const int row = r0 + y * kGroups + group % kGroups;
            in[y][0] = in[y][1] = make_uint4(0u, 0u, 0u, 0u);
            if (row < rows && mine && there) {
                const RowsIn& src = row < a.Hq ? a.q : row < a.Hq + a.Hkv ? a.k : a.v;
                const int head = row < a.Hq ? row : row < a.Hq + a.Hkv ? row - a.Hq : row - a.Hq - a.Hkv;
                const __nv_bfloat16* x = src.p + at * src.ts + head * src.hs;
                in[y][0] = *reinterpret_cast<const uint4*>(x + c0 * 8);
                in[y][1] = *reinterpret_cast<const uint4*>(x + c1 * 8);
            }
        }
#pragma unroll
        for (int y = 0; y < kAhead; ++y) {
            const int row = r0 + y * kGroups + group % kGroups;
            const bool is_q = row < a.Hq, is_v = kPages && row >= a.Hq + a.Hkv;
            const int head = is_q ? row : is_v ? row - a.Hq - a.Hkv : row - a.Hq;
            const bool has_norm = is_q ? a.q_norm != nullptr : !is_v && a.k_norm != nullptr;
            float x[16];
            unpack_chunk(in[y][0], x);
            unpack_chunk(in[y][1], x + 8);
            if (a.q_norm != nullptr || a.k_norm != nullptr) {
                auto sum_of_squares = [&](float f) -> float {
                    float s0 = 0.f, s1 = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = x[i] * f, w = x[8 + i] * f;
                        s0 = fmaf(u, u, s0);
                        s1 = fmaf(w, w, s1);
                    }
                    float s = s0 + s1;
#pragma unroll
                    for (int b = 1; b < kLanes; b <<= 1) s += __shfl_xor_sync(0xffffffffu, s, b);
                    return s;
                };
                float s = sum_of_squares(1.f), f = rsqrtf(s * (1.f / D) + a.eps);
                if (__any_sync(0xffffffffu, !(s < 0x1p126f))) {   // rare: squares that leave 32 bits (eps is nothing beside them)
                    const float s2 = sum_of_squares(0x1p-70f);
                    if (!(s < 0x1p126f)) f = rsqrtf(s2 * (1.f / D)) * 0x1p-70f;
                }
                if (has_norm) {
                    float w[16];
                    unpack_chunk(is_q ? wq[0] : wk[0], w);
                    unpack_chunk(is_q ? wq[1] : wk[1], w + 8);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = x[i] * f * w[i];
                }
            }
            if (!is_v) {
                if (a.adjacent) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = x[2 * i], w = x[2 * i + 1];
                        x[2 * i] = fmaf(u, cs[i].x, -w * cs[i].y);
                        x[2 * i + 1] = fmaf(w, cs[i].x, u * cs[i].y);
                    }
                } else if (halves) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float u = x[i], w = x[8 + i];
                        x[i] = fmaf(u, cs[i].x, -w * cs[i].y);
                        x[8 + i] = fmaf(w, cs[i].x, u * cs[i].y);
                    }
                }
            }
            uint32_t s = 0u;
            if (kPages == 2) {
                // the row's largest magnitude as bits; infinite or no number: over the finite ones alone, and what is infinite becomes NaN
                auto largest = [&](bool finite) -> uint32_t {
                    uint32_t top = 0u;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
                        top = max(top, finite && b >= 0x7f800000u ? 0u : b);
                    }
#pragma unroll
                    for (int b = 1; b < kLanes; b <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, b));
                    return top;
                };
                uint32_t top = largest(false);
                if (__any_sync(0xffffffffu, top >= 0x7f800000u)) {
                    top = largest(true);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if ((__float_as_uint(x[i]) & 0x7fffffffu) >= 0x7f800000u && !is_q) x[i] = __uint_as_float(0x7fffffffu);
                }
                // 448 = 1.75 * 2^8, and 0x1fffff carries into the exponent from the first mantissa above .75 on
                s = (uint32_t)max((int)((top + 0x1fffffu) >> 23) - 8, 0);
            }
            if (row >= rows || !mine) continue;
            if (is_q || !kPages) {
                const RowsOut& dst = is_q ? a.q_out : a.k_out;
                __nv_bfloat16* o = dst.p + at * dst.ts + head * dst.hs;
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                *reinterpret_cast<uint4*>(o + c0 * 8) = there ? pack_chunk(x) : zero;
                *reinterpret_cast<uint4*>(o + c1 * 8) = there ? pack_chunk(x + 8) : zero;
            } else if (there) {
                const long long to = place[t].first + ((long long)head << p.page_shift) * D;
                uint8_t* page = is_v ? p.v : p.k;
                if (kPages == 2) {
                    *reinterpret_cast<uint2*>(page + to + c0 * 8) = pack_codes(x, s);
                    *reinterpret_cast<uint2*>(page + to + c1 * 8) = pack_codes(x + 8, s);
                    if (l == 0) (is_v ? p.vs : p.ks)[place[t].scale + ((long long)head << p.page_shift)] = (uint8_t)s;
                } else {
                    *reinterpret_cast<uint4*>(page + (to + c0 * 8) * 2) = is_v ? in[y][0] : pack_chunk(x);
                    *reinterpret_cast<uint4*>(page + (to + c1 * 8) * 2) = is_v ? in[y][1] : pack_chunk(x + 8);
                }
            }
        }
    }
    if (kPages) report_bounds(a.cu, a.batch, a.n, a.status);
}

}  // namespace adaspark
