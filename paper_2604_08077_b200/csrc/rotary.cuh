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
// a 32-bit float of half turns and what that leaves of it, of first order.
//
// Bound by HBM: every row is read once and written once.  A group of D / 16 threads takes a row at a time, 16 values each: two chunks of
// 8 that are rotated into one another (of neighbours: each in itself).  A group stays with one token, whose cosines and sines are worked out once for
// all heads and kept in registers, as are the weights of the norm, and walks along its heads with a pointer: instructions are what came second
// (312 a row of a warp: 71 us for 16512 tokens of 28 + 4 heads with norms).  Rows come through a ring of shared memory that each thread fills for
// itself, kRotateRing - 1 rows ahead, the first ones before the positions are there.
#pragma once
#include <type_traits>

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
    const float half_turns = (float)(long long)turn, rest = (float)((long long)turn - (long long)half_turns) * (0x1p-63f * 3.14159265f);
    float s, c;
    sincospif(half_turns * 0x1p-63f, &s, &c);
    return make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
}

// Two chunks of 8 bf16 as pairs of numbers.  x[0] and x[1] are rotated into one another: the chunks themselves, or (adjacent) the first
// and the second values of their pairs, those of chunk 0 before those of chunk 1.
__device__ __forceinline__ void unpack_chunks(const uint4& c0, const uint4& c1, bool adjacent, unsigned long long (&x)[2][4]) {
    const uint32_t w[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = __uint_as_float(w[i] << 16);
        hi[i] = __uint_as_float(w[i] & 0xffff0000u);
    }
    if (adjacent) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[0][i] = pack_f32x2(lo[2 * i], lo[2 * i + 1]);
            x[1][i] = pack_f32x2(hi[2 * i], hi[2 * i + 1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[0][i] = pack_f32x2(lo[i], hi[i]);
            x[1][i] = pack_f32x2(lo[4 + i], hi[4 + i]);
        }
    }
}
// The chunks' 16 values in order, from x as above
__device__ __forceinline__ void values_in_order(const unsigned long long (&x)[2][4], bool adjacent, float (&v)[16]) {
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unpack_f32x2(x[0][i], a[2 * i], a[2 * i + 1]);
        unpack_f32x2(x[1][i], b[2 * i], b[2 * i + 1]);
    }
    if (adjacent) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[2 * i] = a[i];
            v[2 * i + 1] = b[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = a[i];
            v[8 + i] = b[i];
        }
    }
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
__device__ __forceinline__ uint4 pack_bf16x8(const float* x) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

constexpr int kRotateThreads = 128;                           // (256: 52 for 49 us of 16512 tokens, 236 for 222 of 65536 into 8-bit pages)
constexpr int kRotateRing = 4;                                // rows of a group under way, and one in work
// (CTAs an SM, ring: 6, 4 take 49.3 us for 16512 tokens rotated and 183.5 for 65536 into pages; 5, 4 51.1 and 201; 7, 4 50.7 and 190; 8, 4 55 and 200;
// 6, 3 51 and 186; 6, 6 51 and 185)

// kPages: 0 rows out; 1, 2 keys and values into pages of bf16, e4m3.  grid (tokens / kTokens).
template <int D, int kPages, int kTokens>
__global__ void __launch_bounds__(kRotateThreads, 6) rotate_kernel(const __grid_constant__ RotateCall a, const __grid_constant__ PageGeom p) {
    constexpr int kLanes = D / 16, kGroups = kRotateThreads / kLanes / kTokens;     // of a token
    __shared__ uint4 ring[kRotateRing][2][kRotateThreads];
    __shared__ float2 turn[kTokens][D / 2 + 2];               // (the tokens of a warp on banks of their own)
    __shared__ TokenPlace place[kTokens];
    const int tid = threadIdx.x, t0 = blockIdx.x * kTokens;
    const int group = tid / kLanes, l = tid % kLanes, t = group / kGroups, at = t0 + t, g = group % kGroups;
    // this thread's two chunks of a row, and whether they are rotated
    const int pc = a.pairs / 8;
    const bool rotated = l < pc, adjacent = a.adjacent != 0;
    const int c0 = rotated ? l : 2 * l, c1 = rotated ? l + pc : 2 * l + 1;
    // The rows ahead: heads g, g + kGroups, ... of q, of k, of v.
    int kind_ahead = -1, left_ahead = 0;                      // (left: heads of the kind from the first group's on)
    const __nv_bfloat16* ahead = nullptr;
    long long step_ahead = 0;
    auto load_row = [&](int slot) {
        while (left_ahead <= 0 && kind_ahead < (kPages ? 2 : 1)) {
            ++kind_ahead;
            const RowsIn& src = kind_ahead == 0 ? a.q : kind_ahead == 1 ? a.k : a.v;
            left_ahead = kind_ahead == 0 ? a.Hq : a.Hkv;
            ahead = src.p + (long long)min(at, a.n - 1) * src.ts + g * src.hs;
            step_ahead = kGroups * src.hs;
        }
        if (g < left_ahead) {                                 // (rows of no sequence, too: they are in the tensors)
            cp_async_16(&ring[slot][0][tid], ahead + c0 * 8);
            cp_async_16(&ring[slot][1][tid], ahead + c1 * 8);
        }
        cp_async_commit();
        ahead += step_ahead;
        left_ahead -= kGroups;
    };
    launch_dependents();
    wait_for_previous_kernel();
#pragma unroll 1
    for (int i = 0; i < kRotateRing - 1; ++i) load_row(i);
    if (kPages) {
        if (tid < 32) {
            const TokenPlace x = place_of_lane<D, kTokens>(p, a.cu, a.kv_len, a.batch, a.n, t0, tid, a.status);
            if (tid < kTokens) place[tid] = x;
        }
        if (a.positions == nullptr) __syncthreads();
    }
    for (int i = tid; i < kTokens * a.pairs; i += kRotateThreads) {
        const int y = i / a.pairs, x = i - y * a.pairs;
        if (t0 + y >= a.n) break;
        const int pos = kPages && a.positions == nullptr ? place[y].pos : a.positions[(size_t)a.axis[x] * a.n + t0 + y];
        turn[y][x] = turned_by((uint64_t)(long long)pos * a.turns[x]);
    }
    __syncthreads();
    bool mine = at < a.n, there = true;
    if (kPages && mine) {
        mine = place[t].first != -1;
        there = place[t].first >= 0;
    }
    // cosines, sines and negative sines beside x[0] and x[1]
    unsigned long long cosine[4], sine[4], minus[4], weight[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int x = adjacent ? (i < 2 ? c0 * 4 + 2 * i : c1 * 4 + 2 * i - 4) : c0 * 8 + 2 * i;
        const float2 u = rotated ? turn[t][x] : make_float2(1.f, 0.f), v = rotated ? turn[t][x + 1] : make_float2(1.f, 0.f);
        cosine[i] = pack_f32x2(u.x, v.x);
        sine[i] = pack_f32x2(u.y, v.y);
        minus[i] = pack_f32x2(-u.y, -v.y);
    }
    int slot = 0;
    // kind: 0 q, 1 k, 2 v.  (As often for every group of a warp: the shuffles need all of it)
    auto rows_of = [&](auto which) {
        constexpr int kKind = which.value;
        constexpr bool kOut = kKind == 0 || kPages == 0;      // rows out, not into pages
        const int heads = kKind == 0 ? a.Hq : a.Hkv;
        const __nv_bfloat16* norm = kKind == 0 ? a.q_norm : kKind == 1 ? a.k_norm : nullptr;
        if (norm != nullptr) unpack_chunks(*reinterpret_cast<const uint4*>(norm + c0 * 8), *reinterpret_cast<const uint4*>(norm + c1 * 8), adjacent, weight);
        const RowsOut& dst = kKind == 0 ? a.q_out : a.k_out;
        // rows out, or a row of the page in bytes; the powers of two
        uint8_t* to = nullptr;
        uint8_t* scale = nullptr;
        long long step;
        constexpr int kBytes = kOut || kPages == 1 ? 2 : 1;
        if (kOut) {
            to = reinterpret_cast<uint8_t*>(dst.p + (long long)at * dst.ts + g * dst.hs);
            step = kGroups * dst.hs * 2;
        } else {
            const TokenPlace x = place[t];
            to = (kKind == 2 ? p.v : p.k) + (x.first + ((long long)g << p.page_shift) * D) * kBytes;
            scale = (kKind == 2 ? p.vs : p.ks) + x.scale + ((long long)g << p.page_shift);
            step = ((long long)kGroups << p.page_shift) * (D * kBytes);
        }
        for (int left = heads; left > 0; left -= kGroups, to += step, scale += kGroups << p.page_shift) {
            cp_async_wait<kRotateRing - 2>();
            const uint4 in0 = ring[slot][0][tid], in1 = ring[slot][1][tid];
            load_row(slot == 0 ? kRotateRing - 1 : slot - 1);
            slot = slot == kRotateRing - 1 ? 0 : slot + 1;
            const bool stores = mine && g < left && (kOut || there);
            if (kKind == 2 && kPages == 1) {                  // as they are
                if (stores) {
                    *reinterpret_cast<uint4*>(to + c0 * 16) = in0;
                    *reinterpret_cast<uint4*>(to + c1 * 16) = in1;
                }
                continue;
            }
            unsigned long long x[2][4];
            unpack_chunks(in0, in1, adjacent, x);
            if (norm != nullptr) {
                auto sum_of_squares = [&]() -> float {
                    unsigned long long s0 = 0ull, s1 = 0ull;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s0 = fma_f32x2(x[0][i], x[0][i], s0);
                        s1 = fma_f32x2(x[1][i], x[1][i], s1);
                    }
                    float lo, hi;
                    unpack_f32x2(add_f32x2(s0, s1), lo, hi);
                    float s = lo + hi;
#pragma unroll
                    for (int b = 1; b < kLanes; b <<= 1) s += __shfl_xor_sync(0xffffffffu, s, b);
                    return s;
                };
                auto root = [](float v) -> float {            // 1 / sqrt(v), and what that leaves to first order
                    const float r = rsqrtf(v);
                    return fmaf(0.5f * r, fmaf(-v * r, r, 1.f), r);
                };
                float v = sum_of_squares() * (1.f / D) + a.eps;
                // rare: squares that leave 32 bits at either end, or an eps that nearly does.  (2^-100 <= v < 2^118 by v's bits, one comparison)
                if (__any_sync(0xffffffffu, __float_as_uint(v) - 0x0d800000u >= 0x7a800000u - 0x0d800000u)) {
                    const float by = v < 0x1p-100f ? 0x1p100f : !(v < 0x1p118f) ? 0x1p-70f : 1.f;
                    auto times = [&](float y) {
                        const unsigned long long y2 = pack_f32x2(y, y);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[0][i] = mul_f32x2(x[0][i], y2);
                            x[1][i] = mul_f32x2(x[1][i], y2);
                        }
                    };
                    times(by);
                    v = sum_of_squares() * (1.f / D) + a.eps * by * by;
                    if (v == INFINITY) {                      // beside an infinity what is finite becomes zeros
                        times(0.f);
                        v = 1.f;
                    }
                }
                const float f = root(v);
                const unsigned long long f2 = pack_f32x2(f, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[0][i] = mul_f32x2(mul_f32x2(x[0][i], f2), weight[0][i]);
                    x[1][i] = mul_f32x2(mul_f32x2(x[1][i], f2), weight[1][i]);
                }
            }
            if (kKind != 2 && rotated) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned long long u = x[0][i], v = x[1][i];
                    x[0][i] = fma_f32x2(v, minus[i], mul_f32x2(u, cosine[i]));
                    x[1][i] = fma_f32x2(u, sine[i], mul_f32x2(v, cosine[i]));
                }
            }
            float v[16];
            values_in_order(x, adjacent, v);
            if (kOut) {
                if (stores) {
                    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4*>(to + c0 * 16) = there ? pack_bf16x8(v) : zero;
                    *reinterpret_cast<uint4*>(to + c1 * 16) = there ? pack_bf16x8(v + 8) : zero;
                }
            } else if (kPages == 1) {
                if (stores) {
                    *reinterpret_cast<uint4*>(to + c0 * 16) = pack_bf16x8(v);
                    *reinterpret_cast<uint4*>(to + c1 * 16) = pack_bf16x8(v + 8);
                }
            } else {
                float top = 0.f, none = 0.f;                  // none: no number if some value is infinite or none
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    top = fmaxf(top, fabsf(v[i]));
                    none = fmaf(v[i], 0.f, none);
                }
                if (__any_sync(0xffffffffu, none != 0.f)) {   // (no number is unequal to anything.)  Rare: over the finite ones alone; what is infinite becomes NaN
                    top = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const bool odd = !(fabsf(v[i]) < INFINITY);
                        top = fmaxf(top, odd ? 0.f : fabsf(v[i]));
                        if (odd) v[i] = __uint_as_float(0x7fffffffu);
                    }
                }
#pragma unroll
                for (int b = 1; b < kLanes; b <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, b));
                // 448 = 1.75 * 2^8, and 0x1fffff carries into the exponent from the first mantissa above .75 on
                const uint32_t s = (uint32_t)max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8, 0);
                if (stores) {
                    *reinterpret_cast<uint2*>(to + c0 * 8) = pack_codes(v, s);
                    *reinterpret_cast<uint2*>(to + c1 * 8) = pack_codes(v + 8, s);
                    if (l == 0) *scale = (uint8_t)s;
                }
            }
        }
    };
    rows_of(std::integral_constant<int, 0>());
    rows_of(std::integral_constant<int, 1>());
    if (kPages) rows_of(std::integral_constant<int, 2>());
    cp_async_wait<0>();
    if (kPages) report_bounds<kRotateThreads>(a.cu, a.batch, a.n, a.status);
}

}  // namespace adaspark
