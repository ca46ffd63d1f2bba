// RMSNorm of each query and key head with the position rotation: what the
// forward and backward kernels (qk_norm_rope.hip) and the backward's fused
// quantisation (qk_quant.hip) share.
//
// A head x of D values: n = x r gamma with r = 1 / sqrt(mean(x^2) + eps), and
// the pairs (a, b) of its first R values turned by the position's angle:
// a' = a c - b s, b' = b c + a s. The pairs are (i, i + R / 2) or, interleaved,
// (2 i, 2 i + 1). Backward: dn = the gradient turned back, dgamma = the sum of
// dn x r over tokens and heads, and with g = dn gamma, h = x r,
// dx = r (g - h mean(g h)).
//
// Layout: L = 1, 2, 4, .. 32 lanes hold a head, eight values each: consecutive
// ones (one 16-byte vector), the pairs' other values exchanged between lanes;
// or, where whole heads that fill their lanes turn by pairs (i, i + D / 2), four
// pairs (two 8-byte pieces D / 2 values apart), so that no value changes lanes
// and no entry of the table is loaded twice. Sums over a head stay within its
// lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"
#include "kernels.h"

namespace puro {

// The value of the lane whose number differs in bit X (X = 1, 2, 4, .. 32):
// lane moves inside the vector ALU where those reach (8 and below), row swaps
// between the 16-lane rows above.
template <int X>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
    if constexpr (X == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);    // quad 1 0 3 2
    else if constexpr (X == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);   // quad 2 3 0 1
    else if constexpr (X == 4) {
        // lane ^ 7 (mirror of 8), then ^ 3 (quad 3 2 1 0)
        const int m = __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);
        return (uint32_t)__builtin_amdgcn_update_dpp(0, m, 0x1B, 0xF, 0xF, true);
    } else if constexpr (X == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true);   // ror 8
    else return (uint32_t)__shfl_xor((int)v, X, 64);
}
template <int X>
__device__ __forceinline__ float lane_xor_f(float v) { return __uint_as_float(lane_xor<X>(__float_as_uint(v))); }

// Sum over the L lanes of a head, in every one of them.
template <int L>
__device__ __forceinline__ float head_sum(float v) {
    if constexpr (L >= 2) v += lane_xor_f<1>(v);
    if constexpr (L >= 4) v += lane_xor_f<2>(v);
    if constexpr (L >= 8) v += lane_xor_f<4>(v);
    if constexpr (L >= 16) v += lane_xor_f<8>(v);
    if constexpr (L >= 32) v += lane_xor_f<16>(v);
    return v;
}

// A token's place: its sequence and its position there.
struct Token {
    int b, s;
};
__device__ __forceinline__ Token token_of(int t, const Divisor& per_seq) {
    const int b = (int)per_seq.quotient((uint32_t)t);
    return {b, t - b * (int)per_seq.d};
}
__device__ __forceinline__ const uint16_t* head_at(const HeadsArg& h, const Token& k) {
    return h.p + k.b * h.bs + k.s * h.rs;
}

// How a lane takes part: its column within the head, whether it holds values
// of the head at all, whether they are rotated, and where their pairs' other
// values are.
struct LaneRole {
    int col;         // first of its eight columns (0 where the lane is past the head)
    bool holds;
    bool turns;
    bool first;      // its values are their pairs' first ones (not interleaved)
    int pair;        // first pair of its values in the table's row
    int partner;     // lane that holds the pairs' other values (not interleaved)
};

template <int L>
__device__ __forceinline__ LaneRole lane_role(int D, int R, int interleaved, int lane) {
    LaneRole r;
    const int c = (lane % L) * 8;
    r.holds = c < D;
    r.col = r.holds ? c : 0;
    r.turns = c < R;                                   // R <= D, R % 16 == 0
    r.first = c < R / 2;
    r.pair = interleaved ? c / 2 : (r.first ? c : c - R / 2);
    if (!r.turns) r.pair = 0;
    r.partner = !r.turns ? lane : (r.first ? lane + R / 16 : lane - R / 16);
    return r;
}

// How a kernel's instance turns heads: not at all; pairs (i, i + D / 2) of
// whole heads that fill their lanes, four pairs a lane; such pairs of any head,
// eight consecutive values a lane; neighbours. (As types: with the table's
// loads in branches the compiler split them into single words.)
enum : int { kTurnNone = 0, kTurnHalf = 1, kTurnPart = 2, kTurnPairs = 3 };
__host__ __device__ inline int turn_kind(const RopeArgs& a, int lanes) {
    return a.dim == 0 ? kTurnNone : a.interleaved ? kTurnPairs : a.dim == lanes * 8 ? kTurnHalf : kTurnPart;
}

// The eight values of a lane, from the start of their head, as 16 bytes.
template <int L, int TURN>
__device__ __forceinline__ uint4 load8(const uint16_t* head, const LaneRole& r) {
    if constexpr (TURN != kTurnHalf) return *reinterpret_cast<const uint4*>(head + r.col);
    const uint2 lo = *reinterpret_cast<const uint2*>(head + r.col / 2);
    const uint2 hi = *reinterpret_cast<const uint2*>(head + L * 4 + r.col / 2);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}
template <int L, int TURN>
__device__ __forceinline__ void store8(uint16_t* head, const LaneRole& r, const uint4 v) {
    if constexpr (TURN != kTurnHalf) {
        *reinterpret_cast<uint4*>(head + r.col) = v;
    } else {
        *reinterpret_cast<uint2*>(head + r.col / 2) = make_uint2(v.x, v.y);
        *reinterpret_cast<uint2*>(head + L * 4 + r.col / 2) = make_uint2(v.z, v.w);
    }
}
// Their columns: e < 4 and e >= 4.
template <int L, int TURN>
__device__ __forceinline__ int column(const LaneRole& r, int e) {
    return TURN == kTurnHalf ? (e < 4 ? r.col / 2 + e : L * 4 + r.col / 2 + e - 4) : r.col + e;
}

// A lane's factors at one position: y_e = n_e c_e + p_e s_e with p_e the pair's
// other value and the sign of the pair's first value in s. With four pairs a
// lane: the pairs' c and s, as they are. back: turned the other way. A position
// outside the table has no angle: NaN.
struct Turn {
    float c[8], s[8];
};
template <int TURN>
__device__ __forceinline__ Turn load_turn(const RopeArgs& a, const LaneRole& r, int pos, bool back) {
    Turn t{};
    if constexpr (TURN == kTurnNone) return t;
    const bool in = (unsigned)pos < (unsigned)a.len;
    const float2* const row = a.table + (int64_t)(in ? pos : 0) * (a.dim / 2);
    const float4* const v = reinterpret_cast<const float4*>(row + (TURN == kTurnHalf ? r.col / 2 : r.pair));
    constexpr int N = TURN == kTurnPart ? 8 : 4;       // pairs that the lane needs
    float4 u[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) u[i] = v[i];
    const uint32_t sign = r.first != back ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float c = i & 1 ? u[i / 2].z : u[i / 2].x, s = i & 1 ? u[i / 2].w : u[i / 2].y;
        if constexpr (TURN == kTurnPairs) {
            t.c[2 * i] = t.c[2 * i + 1] = c;
            t.s[2 * i] = back ? s : -s;
            t.s[2 * i + 1] = back ? -s : s;
        } else {
            t.c[i] = c;
            t.s[i] = TURN == kTurnHalf ? s : __uint_as_float(__float_as_uint(s) ^ sign);
        }
    }
    if (__builtin_amdgcn_ballot_w64(!in)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.c[i] = in ? t.c[i] : __builtin_nanf("");
            t.s[i] = in ? t.s[i] : __builtin_nanf("");
        }
    }
    return t;
}

// Four pairs (v_e, v_4+e) turned by (c_e, s_e), or back.
__device__ __forceinline__ void turn_pairs4(float v[8], const float c[4], const float s[4], bool back) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float a = v[e], b = v[4 + e];
        v[e] = fmaf(b, back ? s[e] : -s[e], a * c[e]);
        v[4 + e] = fmaf(a, back ? -s[e] : s[e], b * c[e]);
    }
}

// The eight values turned. (Lanes past the rotated values keep theirs, not by
// c = 1, s = 0: an infinity times 0 would be a NaN. Where all of a head turns,
// lanes that hold none of it turn their zeros.)
template <int TURN>
__device__ __forceinline__ void turn8(float v[8], const Turn& t, const LaneRole& r, const RopeArgs& a, int D, bool back) {
    if constexpr (TURN == kTurnNone) return;
    if constexpr (TURN == kTurnHalf) {
        turn_pairs4(v, t.c, t.s, back);
        return;
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float p = TURN == kTurnPairs ? v[i ^ 1] : __shfl(v[i], r.partner, 64);
        y[i] = fmaf(p, t.s[i], v[i] * t.c[i]);
    }
    const bool all = a.dim == D;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = all || r.turns ? y[i] : v[i];
}

__device__ __forceinline__ void unpack8(const uint4 w, float v[8]) {
    v[0] = bf16lo(w.x); v[1] = bf16hi(w.x); v[2] = bf16lo(w.y); v[3] = bf16hi(w.y);
    v[4] = bf16lo(w.z); v[5] = bf16hi(w.z); v[6] = bf16lo(w.w); v[7] = bf16hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float v[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7]));
}

// 1 / sqrt(mean(x^2) + eps) of the head whose eight values the lane holds
// (zeros where it holds none), by the reciprocal-root instruction (1 ulp, which
// flushes numbers below the normal range). Where mean and eps are so small that
// squares have lost bits or vanished (a binary32 square below 2^-126; from
// 2^-100 on what is lost is less than 2^-40 of the mean), the head is scaled:
// x becomes x s and the result r / s with s = 2^96, otherwise s = 1; x r stays.
// An eps of 2^-100 rules that out for a whole call: instances without SMALL do
// not look (the look, which parts the heads that a wave has in flight, is 43.0 ->
// 44.1 us of the backward at 8192 tokens of 16 + 8 heads of 128, 55.5 -> 57.0 of
// the one quantised in groups).
constexpr float kLeastMean = 0x1p-100f;
template <int L, bool SMALL>
__device__ __forceinline__ float head_rstd(float x[8], float inv_d, float eps, float& s) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    float m = fmaf(head_sum<L>(ss), inv_d, eps);
    s = 1.0f;
    if constexpr (SMALL) {
        const bool tiny = m < kLeastMean;
        s = tiny ? 0x1p96f : 1.0f;
        if (__builtin_amdgcn_ballot_w64(tiny)) {
            ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= s;
                ss = fmaf(x[i], x[i], ss);
            }
            m = fmaf(head_sum<L>(ss), inv_d, eps * s * s);
        }
    }
    return __builtin_amdgcn_rsqf(m);
}

// The backward of the norm: d (the gradient of n, turned back) becomes dx, and
// what the lane's columns add to dgamma is returned in w. (x: zeros where the
// lane holds none; d is zero there too.)
template <int L, bool SMALL>
__device__ __forceinline__ void norm_bwd8(float d[8], float x[8], const float g[8], float inv_d, float eps,
                                          float w[8]) {
    float s;
    const float r = head_rstd<L, SMALL>(x, inv_d, eps, s);
    float m = 0.0f, h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        h[i] = x[i] * r;
        w[i] = d[i] * h[i];
        d[i] *= g[i];
        m = fmaf(d[i], h[i], m);
    }
    m = head_sum<L>(m) * inv_d;
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] = r * fmaf(-h[i], m, d[i]) * (SMALL ? s : 1.0f);
}

}  // namespace puro
