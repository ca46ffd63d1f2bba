// RMSNorm of the query and key heads and their position rotation, forward and
// backward (gfx950). The mathematics and the lane layout: qk_norm_rope.h.
//
// Both passes read every value once and write it once; about ten operations a
// byte leave them bound by memory. A wave takes one token and walks its heads
// (64 / L at a time, L lanes a head), so that the position's cosines and sines
// are loaded once per token instead of once per head: as binary32 they are
// four times the size of a head's own BF16 values. 8192 tokens of 16 + 8 heads
// of 128: forward 18 to 19 us for 103 MB (5.4 TB/s; a large copy reaches 5.15),
// backward 34 us for 187 MB (5.4) and 4 for the sum of dgamma; one token 2.5 us.

#include <algorithm>

#include "qk_norm_rope.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Heads that a lane has in flight: their loads are issued together.
// (backward, which loads two vectors a head: two heads take 64 to 95 registers and
// five waves or more fit a SIMD; four took 126, 52.7 against 41.9 us at 8192
// tokens of 16 + 8 heads of 128)
constexpr int kUnroll = 4, kUnrollBwd = 2;

// Table of cosines and sines: the angle in double precision (at position 10^6
// a binary32 angle is off by 0.03), reduced and evaluated there.
__global__ __launch_bounds__(kThreads) void rope_table_kernel(float2* __restrict__ table, int64_t len, int dim,
                                                              double theta) {
    const int half = dim / 2;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= len * half) return;
    const int64_t p = i / half;
    const int e = (int)(i - p * half);
    double s, c;
    sincos((double)p * pow(theta, -2.0 * e / dim), &s, &c);
    table[i] = make_float2((float)c, (float)s);
}

// Heads of one kind: block row y takes the query heads (0), the key heads (1)
// or (backward) the value heads (2), so that a wave holds one kind's pointers
// and strides in scalar registers, which are too few for all of them.

// Forward: wave w takes steps [part * per, part * per + per) of 64 / L heads
// of token w / parts. Few tokens are split over more waves.
template <int L, int TURN, bool SMALL>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_fwd_kernel(QkArgs a, Divisor per_seq, int per) {
    constexpr int GPW = 64 / L;
    const bool key = blockIdx.y != 0;
    const HeadsArg in = key ? a.k : a.q, out = key ? a.ok : a.oq;
    const uint16_t* const gamma = key ? a.gk : a.gq;
    const int heads = key ? a.hk : a.hq;
    const int steps = (heads + GPW - 1) / GPW, parts = (steps + per - 1) / per;
    if (parts == 0) return;
    const int w = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6));
    const int t = w / parts, part = w - t * parts;
    if (t >= a.tokens) return;
    const int lane = threadIdx.x & 63, grp = lane / L;
    const LaneRole role = lane_role<L>(a.D, a.rope.dim, a.rope.interleaved, lane);
    const Token tok = token_of(t, per_seq);
    const uint16_t* const x = head_at(in, tok);
    uint16_t* const y = const_cast<uint16_t*>(head_at(out, tok));
    const Turn turn = load_turn<TURN>(a.rope, role, TURN && a.rope.pos ? a.rope.pos[t] : tok.s, false);
    uint4 gw{};
    if (gamma) gw = load8<L, TURN>(gamma, role);
    const float inv_d = 1.0f / (float)a.D;
    const int i1 = min(steps, part * per + per);
    for (int i = part * per; i < i1; i += kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)     // (lanes past the last head read it again and store nothing)
            raw[u] = load8<L, TURN>(x + min((i + u) * GPW + grp, heads - 1) * in.hs, role);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (i + u >= i1) break;
            const int h = (i + u) * GPW + grp;
            float v[8], g[8];
            unpack8(raw[u], v);
            if (!role.holds) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.0f;
            }
            if (gamma) {
                float s;
                const float r = head_rstd<L, SMALL>(v, inv_d, a.eps, s);
                unpack8(gw, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = v[e] * r * g[e];
            }
            turn8<TURN>(v, turn, role, a.rope, a.D, false);
            if (role.holds && h < heads) store8<L, TURN>(y + h * out.hs, role, pack8(v));
        }
    }
}

// Sums of dgamma: a binary32 sum of n terms of one sign is off by up to n / 2
// units in the last place (2^20 tokens of 16 heads of 128 are 1366 a lane), so
// after kDeep additions it moves to a binary64 one, rounded once at the end.
// (Fewer terms never leave binary32; 8192 tokens of 16 + 8 heads: 6 a lane.)
constexpr int kDeep = 64;

// Backward: wave w takes tokens w, w + waves, ..; every lane keeps the sums of
// dgamma of its eight columns in binary32 (the long ones' binary64 parts in
// LDS, each lane its own), the block adds them up in a fixed order and writes
// part[kind][block][D].
template <int L, int TURN, bool SMALL>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_bwd_kernel(QkArgs a, Divisor per_seq) {
    constexpr int GPW = 64 / L;
    __shared__ float red[kWaves][L * 8];
    __shared__ double deep[8][kThreads];
    const int kind = blockIdx.y;
    const HeadsArg grad = kind == 0 ? a.dq : (kind == 1 ? a.dk : a.dv);
    const HeadsArg out = kind == 0 ? a.oq : (kind == 1 ? a.ok : a.ov);
    const uint16_t* const gamma = kind == 0 ? a.gq : (kind == 1 ? a.gk : nullptr);
    // (heads that are not normalised are not read: the gradient stands in)
    const HeadsArg in = !gamma ? grad : (kind == 0 ? a.q : a.k);
    const int heads = kind == 0 ? a.hq : a.hk;
    const int wave = threadIdx.x >> 6;
    const int lane = threadIdx.x & 63, grp = lane / L;
    const int w = __builtin_amdgcn_readfirstlane((int)blockIdx.x * kWaves + wave);
    const int waves = (int)gridDim.x * kWaves;
    const LaneRole role = lane_role<L>(a.D, a.rope.dim, a.rope.interleaved, lane);
    const bool turned = TURN != kTurnNone && kind < 2;
    float sum[8];
    uint4 gw{};
    if (gamma) gw = load8<L, TURN>(gamma, role);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    const float inv_d = 1.0f / (float)a.D;
    int adds = 0;
    bool folded = false;
    for (int64_t t64 = w; heads > 0 && t64 < a.tokens; t64 += waves) {
        const int t = (int)t64;
        const Token tok = token_of(t, per_seq);
        const uint16_t* const d = head_at(grad, tok);
        const uint16_t* const x = head_at(in, tok);
        uint16_t* const y = const_cast<uint16_t*>(head_at(out, tok));
        Turn turn{};
        if (turned) turn = load_turn<TURN>(a.rope, role, a.rope.pos ? a.rope.pos[t] : tok.s, true);
        for (int i = 0; i * GPW < heads; i += kUnrollBwd) {
            uint4 rd[kUnrollBwd], rx[kUnrollBwd];
#pragma unroll
            for (int u = 0; u < kUnrollBwd; ++u) {
                const int h = min((i + u) * GPW + grp, heads - 1);
                rd[u] = load8<L, TURN>(d + h * grad.hs, role);
                if (gamma) rx[u] = load8<L, TURN>(x + h * in.hs, role);
                else rx[u] = rd[u];
            }
#pragma unroll
            for (int u = 0; u < kUnrollBwd; ++u) {
                if ((i + u) * GPW >= heads) break;
                const int h = (i + u) * GPW + grp;
                const bool live = role.holds && h < heads;
                float v[8], n[8], wg[8];
                unpack8(rd[u], v);
                unpack8(rx[u], n);
                if (!role.holds) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = n[e] = 0.0f;
                }
                if (turned) turn8<TURN>(v, turn, role, a.rope, a.D, true);
                if (gamma) {
                    // (unpacked anew for each head: kept, it would hold eight registers)
                    float g[8];
                    asm volatile("" : "+v"(gw.x), "+v"(gw.y), "+v"(gw.z), "+v"(gw.w));
                    unpack8(gw, g);
                    norm_bwd8<L, SMALL>(v, n, g, inv_d, a.eps, wg);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += live ? wg[e] : 0.0f;
                }
                // (an untouched head as its bits are: a signalling NaN is not made quiet)
                if (live) store8<L, TURN>(y + h * out.hs, role, turned || gamma ? pack8(v) : rd[u]);
            }
            adds += kUnrollBwd;
            if (adds >= kDeep) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    deep[e][threadIdx.x] = (folded ? deep[e][threadIdx.x] : 0.0) + (double)sum[e];
                    sum[e] = 0.0f;
                }
                adds = 0;
                folded = true;
            }
        }
    }
    if (!a.part || kind == 2) return;
    if (folded) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = (float)(deep[e][threadIdx.x] + (double)sum[e]);
    }
    // the groups of a wave, then the block's waves
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float s = sum[e];
#pragma unroll
        for (int o = L; o < 64; o *= 2) s += __shfl_xor(s, o, 64);
        if (grp == 0 && role.holds) red[wave][column<L, TURN>(role, e)] = s;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.D; c += kThreads)
        a.part[((int64_t)kind * gridDim.x + blockIdx.x) * a.D + c] = (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
}

// dgamma of 8 columns per block: two lanes a row of partial sums (16 bytes
// each), 128 rows at a time, four loads in flight per lane; then across the
// wave and the four waves. LONG: every kDeep rounds the lane's sums move to
// binary64 ones, as above; kLongRows rows (2^18 tokens of 16 heads quantised)
// are the most that never would.
constexpr int64_t kLongRows = 512 * kDeep;
template <bool LONG>
__global__ __launch_bounds__(kThreads) void dgamma_sum_kernel(const float* __restrict__ pq, int64_t nq,
                                                              float* __restrict__ dgq, const float* __restrict__ pk,
                                                              int64_t nk, float* __restrict__ dgk, int64_t ldp) {
    __shared__ float4 red[kWaves][2];
    const float* const p = (blockIdx.y ? pk : pq) + blockIdx.x * 8 + (threadIdx.x & 1) * 4;
    float* const out = blockIdx.y ? dgk : dgq;
    const int64_t n = blockIdx.y ? nk : nq;
    if (!out) return;
    double deep[4] = {};
    float t[4];
    for (int64_t i0 = threadIdx.x >> 1;; i0 += kLongRows) {
        float4 s[4] = {};
        const int64_t end = LONG ? min(n, i0 + kLongRows) : n;
        for (int64_t i = i0; i < end; i += 512) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + 128 * u < n) {
                    const float4 v = *reinterpret_cast<const float4*>(p + (i + 128 * u) * ldp);
                    s[u].x += v.x; s[u].y += v.y; s[u].z += v.z; s[u].w += v.w;
                }
        }
        t[0] = (s[0].x + s[1].x) + (s[2].x + s[3].x);
        t[1] = (s[0].y + s[1].y) + (s[2].y + s[3].y);
        t[2] = (s[0].z + s[1].z) + (s[2].z + s[3].z);
        t[3] = (s[0].w + s[1].w) + (s[2].w + s[3].w);
        if constexpr (!LONG) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            deep[e] += (double)t[e];
            t[e] = (float)deep[e];
        }
        if (i0 + kLongRows >= n) break;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        t[e] += lane_xor_f<2>(t[e]);
        t[e] += lane_xor_f<4>(t[e]);
        t[e] += lane_xor_f<8>(t[e]);
        t[e] += lane_xor_f<16>(t[e]);
        t[e] += lane_xor_f<32>(t[e]);
    }
    if ((threadIdx.x & 63) < 2) red[threadIdx.x >> 6][threadIdx.x & 1] = make_float4(t[0], t[1], t[2], t[3]);
    __syncthreads();
    if (threadIdx.x < 2) {
        const float4 a = red[0][threadIdx.x], b = red[1][threadIdx.x], c = red[2][threadIdx.x], d = red[3][threadIdx.x];
        float* const o = out + blockIdx.x * 8 + threadIdx.x * 4;
        o[0] = (a.x + b.x) + (c.x + d.x); o[1] = (a.y + b.y) + (c.y + d.y);
        o[2] = (a.z + b.z) + (c.z + d.z); o[3] = (a.w + b.w) + (c.w + d.w);
    }
}

// Blocks of the backward per kind of heads: enough to fill the chip, each wave
// with a token or more, and few partial sums (8192 tokens as above: 512 blocks
// 41.8 us, 768 41.1, 1024 41.2).
int64_t bwd_blocks(int64_t tokens) {
    return std::max<int64_t>(1, std::min<int64_t>((tokens + kWaves - 1) / kWaves, 768));
}

// f(lanes of a head, how it turns, whether heads may be too small for their
// squares), as types.
template <class F>
void by_lanes(const QkArgs& a, F&& f) {
    const int D = a.D;
    auto small = [&](auto lanes, auto turn) {
        if ((a.gq || a.gk) && a.eps < kLeastMean) f(lanes, turn, std::integral_constant<bool, true>{});
        else f(lanes, turn, std::integral_constant<bool, false>{});
    };
    auto turns = [&](auto lanes) {
        switch (turn_kind(a.rope, decltype(lanes)::value)) {
        case kTurnNone: small(lanes, std::integral_constant<int, kTurnNone>{}); break;
        case kTurnHalf: small(lanes, std::integral_constant<int, kTurnHalf>{}); break;
        case kTurnPart: small(lanes, std::integral_constant<int, kTurnPart>{}); break;
        default: small(lanes, std::integral_constant<int, kTurnPairs>{});
        }
    };
    if (D <= 8) turns(std::integral_constant<int, 1>{});
    else if (D <= 16) turns(std::integral_constant<int, 2>{});
    else if (D <= 32) turns(std::integral_constant<int, 4>{});
    else if (D <= 64) turns(std::integral_constant<int, 8>{});
    else if (D <= 128) turns(std::integral_constant<int, 16>{});
    else turns(std::integral_constant<int, 32>{});
}

}  // namespace

void launch_rope_table(float2* table, int64_t len, int dim, double theta, hipStream_t stream) {
    const int64_t n = len * (dim / 2);
    if (n == 0) return;
    rope_table_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, stream>>>(table, len, dim, theta);
}

void launch_qk_norm_rope_fwd(const QkArgs& a, hipStream_t stream) {
    const int heads = std::max(a.hq, a.hk);
    if (a.tokens == 0 || heads == 0) return;
    by_lanes(a, [&](auto lanes, auto turn, auto small) {
        constexpr int L = decltype(lanes)::value, GPW = 64 / L;
        const int steps = (heads + GPW - 1) / GPW;
        // a wave a step up to 2048 of them, and a wave a token beyond (us, split
        // and whole; 16 + 8 heads of 128, four steps: 1 token 2.33 and 2.74, 256
        // 2.89 and 3.32, 512 3.67 and 3.52, 1024 5.29 and 4.13, 4096 13.3 and 10.1;
        // 16 + 4 of 256, eight steps: 256 tokens 3.59 and 4.86, 512 5.01 and 5.20,
        // 1024 7.60 and 7.22): the split's waves load the position's row anew
        const int per = a.tokens * steps <= 2048 ? 1 : steps;
        const int64_t waves = a.tokens * ((steps + per - 1) / per);
        qk_norm_rope_fwd_kernel<L, decltype(turn)::value, decltype(small)::value>
            <<<dim3((unsigned)((waves + kWaves - 1) / kWaves), a.hk > 0 ? 2 : 1), kThreads, 0, stream>>>(a, Divisor::of((uint32_t)a.seq), per);
    });
}

void launch_dgamma_sum(const float* part_q, int64_t nq, float* dgq, const float* part_k, int64_t nk, float* dgk,
                       int64_t ldp, int D, hipStream_t stream) {
    const dim3 grid((unsigned)(D / 8), 2);
    if (std::max(nq, nk) > kLongRows) dgamma_sum_kernel<true><<<grid, kThreads, 0, stream>>>(part_q, nq, dgq, part_k, nk, dgk, ldp);
    else dgamma_sum_kernel<false><<<grid, kThreads, 0, stream>>>(part_q, nq, dgq, part_k, nk, dgk, ldp);
}

size_t qk_bwd_ws_bytes(int64_t tokens, int D) {
    return (size_t)bwd_blocks(tokens) * 2 * D * sizeof(float);
}

void launch_qk_norm_rope_bwd(QkArgs a, void* ws, hipStream_t stream) {
    const bool sums = a.dgq || a.dgk;
    const int64_t blocks = bwd_blocks(a.tokens);
    a.part = sums ? reinterpret_cast<float*>(ws) : nullptr;
    if (a.tokens > 0)
        by_lanes(a, [&](auto lanes, auto turn, auto small) {
            qk_norm_rope_bwd_kernel<decltype(lanes)::value, decltype(turn)::value, decltype(small)::value>
                <<<dim3((unsigned)blocks, a.dv.p ? 3 : 2), kThreads, 0, stream>>>(a, Divisor::of((uint32_t)a.seq));
        });
    if (sums) {
        const int64_t n = a.tokens > 0 ? blocks : 0;
        launch_dgamma_sum(a.part, n, a.dgq, a.part + blocks * a.D, n, a.dgk, a.D, a.D, stream);
    }
}

}  // namespace puro
