// RMSNorm of each query and key head with the position rotation: what the
// forward and backward kernels (qk_norm_rope.hip) and the backward's fused
// quantisation (quant.hip) share.
//
// A head x of D values: n = x r gamma with r = 1 / sqrt(mean(x^2) + eps), and
// the pairs (a, b) of its first R values turned by the position's angle:
// a' = a c - b s, b' = b c + a s. The pairs are (i, i + R / 2) or, interleaved,
// (2 i, 2 i + 1). Backward: dn = the gradient turned back, dgamma = the sum of
// dn x r over tokens and heads, and with g = dn gamma, h = x r,
// dx = r (g - h mean(g h)).
//
// Layout: L = 1, 2, 4, .. 32 lanes hold a head, eight consecutive values (one
// 16-byte vector) each; sums over a head and the exchange of the pairs stay
// within those lanes.
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

// A lane's part of the rotation at one position: y_e = n_e c_e + p_e s_e with
// p_e the pair's other value and the sign of the pair's first value in s.
// Lanes past the rotated values keep theirs (not by c = 1, s = 0: an infinity
// times 0 would be a NaN).
struct Turn {
    float c[8], s[8];
};

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

// The table's row of a position, for this lane; back: turned the other way.
// A position outside the table has no angle: NaN.
__device__ __forceinline__ Turn load_turn(const RopeArgs& a, const LaneRole& r, int pos, bool back) {
    Turn t;
    const bool in = (unsigned)pos < (unsigned)a.len;
    const float2* row = a.table + (int64_t)(in ? pos : 0) * (a.dim / 2) + r.pair;
    const float4* v = reinterpret_cast<const float4*>(row);
    const float nan = __builtin_nanf("");
    if (a.interleaved) {
        const float4 u[2] = {v[0], v[1]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float c = in ? (i & 1 ? u[i / 2].z : u[i / 2].x) : nan;
            const float s = in ? (i & 1 ? u[i / 2].w : u[i / 2].y) : nan;
            t.c[2 * i] = t.c[2 * i + 1] = c;
            t.s[2 * i] = back ? s : -s;
            t.s[2 * i + 1] = back ? -s : s;
        }
    } else {
        const float4 u[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = i & 1 ? u[i / 2].z : u[i / 2].x, s = i & 1 ? u[i / 2].w : u[i / 2].y;
            t.c[i] = in ? c : nan;
            t.s[i] = in ? (r.first != back ? -s : s) : nan;
        }
    }
    return t;
}

// The eight values turned. HALF: the pairs' other values are L / 2 lanes away
// (the whole head is rotated), else wherever LaneRole says.
template <int L>
__device__ __forceinline__ void turn8(float v[8], const Turn& t, const LaneRole& r, int interleaved, bool half) {
    float p[8];
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = v[i ^ 1];
    } else if (L >= 2 && half) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = lane_xor_f<(L >= 2 ? L / 2 : 1)>(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = __shfl(v[i], r.partner, 64);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = r.turns ? fmaf(p[i], t.s[i], v[i] * t.c[i]) : v[i];
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
// (zeros where it holds none).
template <int L>
__device__ __forceinline__ float head_rstd(const float x[8], float inv_d, float eps) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    return 1.0f / sqrtf(fmaf(head_sum<L>(ss), inv_d, eps));
}

// The backward of the norm: d (the gradient of n, turned back) becomes dx, and
// what the lane's columns add to dgamma is returned in w. (x: zeros where the
// lane holds none; d is zero there too.)
template <int L>
__device__ __forceinline__ void norm_bwd8(float d[8], const float x[8], const float g[8], float inv_d, float eps,
                                          float w[8]) {
    const float r = head_rstd<L>(x, inv_d, eps);
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
    for (int i = 0; i < 8; ++i) d[i] = r * fmaf(-h[i], m, d[i]);
}

}  // namespace puro
