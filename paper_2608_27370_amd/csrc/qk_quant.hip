// The backward of the query / key norm with rotation, quantised as it is formed
// (gfx950): the gradient of the QKV projection's output is the dY of that
// projection's Dgrad and Wgrad (Section 3.2 quantises it right before them),
// so its BF16 values never go to memory.
//
// A block takes a 128 x 128 tile, as the quantisers do: a head of 128 values,
// or two of 64, is a tile's width, and the 16 (8) lanes that hold a head's row
// exchange its pairs and its sums by lane moves. Bound by memory: 4 bytes read
// and 1 byte a copy written per query and key value, 2 and 1 per value head's.
// 8192 tokens of 16 + 8 heads of 128, E4M3 rows and columns: 50 us for 187 MB
// (3.7 TB/s; the BF16 backward and the quantiser one after the other move 321 MB).
// 163 to 166 registers (heads of 128, the usual case below) let three blocks
// share a CU, 171 to 174 (heads of 64) two, 101 to 128 (any other case) four,
// and each of them loads, computes and stores its one tile in that order: 2048
// tiles are 2.7 rounds of three a CU. With the sum of dgamma, us at 8192 tokens,
// in groups and per tensor: 16 + 8 heads of 128 turned by halves 54 to 56 and 76,
// by neighbours 59 and 82, 48 of their values 58 and 82, query heads alone
// normalised 56 and 80; 32 + 8 of 64 51 and 70, half turned by neighbours 48 and 67.

#include "qk_norm_rope.h"
#include "quant_tile.h"

namespace puro {

namespace {

// The heads of one kind, 0 query, 1 key, 2 value, as a tile takes them: the
// first one's number, where the gradient and the head before the norm are
// (heads that are not normalised are not read: the gradient stands in).
struct Kind {
    const uint16_t *g, *x, *gamma;
    int64_t gbs, grs, ghs, xbs, xrs, xhs;
    int64_t first;
};
struct Kinds {
    Kind of[3];
};

Kinds kinds_of(const QkArgs& k) {
    Kinds r;
    const HeadsArg g[3] = {k.dq, k.dk, k.dv}, x[3] = {k.gq ? k.q : k.dq, k.gk ? k.k : k.dk, k.dv};
    const uint16_t* const gamma[3] = {k.gq, k.gk, nullptr};
    const int64_t first[3] = {0, k.hq, (int64_t)k.hq + k.hk};
    for (int i = 0; i < 3; ++i)
        r.of[i] = Kind{g[i].p, x[i].p, gamma[i], g[i].bs, g[i].rs, g[i].hs, x[i].bs, x[i].rs, x[i].hs, first[i]};
    return r;
}

// What a thread takes of the head of L lanes that it belongs to; head0: the
// tile's first head (one of 128 values, or two of 64). A head's kind is read
// from the kernel's arguments (their first) by its number.
struct HeadOf {
    int kind;
    bool none;                    // past the last head: the last one again, and zeros
    int64_t gbs, grs, xbs, xrs;   // strides of the gradient and of the head
    const uint16_t *gp, *xp;      // the head at token 0
    const uint16_t* gamma;
};
template <int L>
__device__ __forceinline__ HeadOf head_of(const QkArgs& k, int head0) {
    typedef const __attribute__((address_space(4))) Kinds* kinds_ptr;
    const kinds_ptr kinds = (kinds_ptr)__builtin_amdgcn_kernarg_segment_ptr();
    const int hqk = k.hq + k.hk;
    auto one = [&](int head) __attribute__((always_inline)) {
        HeadOf h;
        h.none = head >= hqk + k.hk;
        head = min(head, hqk + k.hk - 1);
        h.kind = (head >= k.hq ? 1 : 0) + (head >= hqk ? 1 : 0);
        const auto& c = kinds->of[h.kind];
        const int64_t at = head - c.first;
        h.gbs = c.gbs; h.grs = c.grs; h.xbs = c.xbs; h.xrs = c.xrs;
        h.gp = c.g + at * c.ghs;
        h.xp = c.x + at * c.xhs;
        h.gamma = c.gamma;
        return h;
    };
    HeadOf h = one(head0);
    if constexpr (L == 8) {
        const bool second = (threadIdx.x & 8) != 0;
        const HeadOf b = one(head0 + 1);
        // (into vector registers one field after the other: there are too few scalar ones)
        auto pick = [&](auto x, auto y) __attribute__((always_inline)) {
            auto v = second ? y : x;
            asm volatile("" : "+v"(v));
            return v;
        };
        h.kind = pick(h.kind, b.kind);
        h.none = second ? b.none : h.none;
        h.gp = pick(h.gp, b.gp); h.gbs = pick(h.gbs, b.gbs); h.grs = pick(h.grs, b.grs);
        h.xp = pick(h.xp, b.xp); h.xbs = pick(h.xbs, b.xbs); h.xrs = pick(h.xrs, b.xrs);
        h.gamma = pick(h.gamma, b.gamma);
    }
    return h;
}

// (The sums are pinned after each row: the compiler moves their additions to
// where the sums are used, behind a branch, and keeps 64 terms until then.)

// Any case, two rows at a time.
template <int L, bool SMALL>
__device__ __forceinline__ void load_qk_bwd_any(const QkArgs& k, const Divisor& per_seq, const Tile& t, int head0,
                                                uint32_t w[8][4], float sum[8], int col[2]) {
    const LaneRole role = lane_role<L>(k.D, k.rope.dim, k.rope.interleaved, threadIdx.x & 63);
    HeadOf h = head_of<L>(k, head0);
    h.gp += role.col;
    h.xp += role.col;
    const int kind = h.kind;
    col[0] = t.cc * 8;
    col[1] = t.cc * 8 + 4;
    const bool norm = h.gamma != nullptr;
    const float inv_d = 1.0f / (float)k.D;
    uint4 gw{};
    if (norm) gw = *reinterpret_cast<const uint4*>(h.gamma + role.col);
    const int turn_as = turn_kind(k.rope, L);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
#pragma unroll
    for (int i0 = 0; i0 < 8; i0 += 2) {
        uint4 rd[2], rx[2];
        int pos[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // rows past the last one are the last one again, and zeros below
            const int row = (int)min(t.row0 + i0 + u, k.tokens - 1);
            const Token tok = token_of(row, per_seq);
            rd[u] = *reinterpret_cast<const uint4*>(h.gp + tok.b * h.gbs + tok.s * h.grs);
            rx[u] = *reinterpret_cast<const uint4*>(h.xp + tok.b * h.xbs + tok.s * h.xrs);
            pos[u] = turn_as != kTurnNone && k.rope.pos ? k.rope.pos[row] : tok.s;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = i0 + u;
            const bool live = t.row0 + i < k.tokens && !h.none;
            float d[8], n[8], x8[8], gm[8], wg[8];
            unpack8(rd[u], d);
            auto turned = [&](auto as) __attribute__((always_inline)) {
                constexpr int TURN = decltype(as)::value;
                turn8<TURN>(d, load_turn<TURN>(k.rope, role, pos[u], true), role, k.rope, k.D, true);
            };
            if (turn_as == kTurnPart || turn_as == kTurnHalf) turned(std::integral_constant<int, kTurnPart>{});
            else if (turn_as == kTurnPairs) turned(std::integral_constant<int, kTurnPairs>{});
            unpack8(rx[u], x8);
            unpack8(gw, gm);
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] = d[e];
            norm_bwd8<L, SMALL>(n, x8, gm, inv_d, k.eps, wg);
            uint4 o = rd[u];
            if (kind != 2) o = pack8(norm ? n : d);
            w[i][0] = live ? o.x : 0u; w[i][1] = live ? o.y : 0u;
            w[i][2] = live ? o.z : 0u; w[i][3] = live ? o.w : 0u;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum[e] += live && norm ? wg[e] : 0.0f;
                asm volatile("" : "+v"(sum[e]));
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The usual case: both kinds of heads normalised with an eps that stands over
// the smallest heads, whole heads turned by pairs (i, i + D / 2), sequences of
// whole groups of 8 tokens, so that a thread's rows are one sequence's and all
// or none of them exist. Here lane l of a head holds
// the pairs 4 l .. 4 l + 3, two 8-byte pieces D / 2 values apart: no value changes
// lanes, and the lanes' cosines and sines are one run of the table (with eight
// consecutive values a lane, every entry is loaded by two lanes and each of
// four 16-byte loads touches all of the row's lines, which held up the loads: 70
// against 54 us at 8192 tokens of 16 + 8 heads of 128). The results change to the
// quantiser's columns through LDS, a row of a wave at a time. The tile's loads
// are all issued before the first is waited for, a row's cosines and sines one
// row ahead. (A wave with a position outside the table takes the way above.)
template <int L>
__device__ __forceinline__ void load_qk_bwd_usual(const QkArgs& k, const Divisor& per_seq, const Tile& t,
                                                  int head0, uint8_t (*stage)[1024], uint32_t w[8][4], float sum[8],
                                                  int col[2]) {
    constexpr int D = L * 8;
    const HeadOf h = head_of<L>(k, head0);
    const int kind = h.kind;
    const bool live = t.row0 < k.tokens && !h.none;
    const int row0 = (int)min(t.row0, k.tokens - 8);
    const Token tok = token_of(row0, per_seq);
    const int lane = threadIdx.x & 63, l = lane % L;
    col[0] = t.cc / L * D + 4 * l;
    col[1] = col[0] + D / 2;
    const uint16_t* const gp = h.gp + tok.b * h.gbs + tok.s * h.grs;
    const uint16_t* const xp = h.xp + tok.b * h.xbs + tok.s * h.xrs + 4 * l;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    if (wave_none(kind != 2)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(gp + i * h.grs + 8 * l);
            w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
        }
    } else {
        int pos[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) pos[i] = tok.s + i;
        if (k.rope.pos) {
            bool out = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                pos[i] = k.rope.pos[row0 + i];
                out = out || (unsigned)pos[i] >= (unsigned)k.rope.len;
            }
            if (!wave_none(out)) {
                load_qk_bwd_any<L, false>(k, per_seq, t, head0, w, sum, col);
                return;
            }
        }
        auto turn_row = [&](int p, float4 u[2]) __attribute__((always_inline)) {
            const float4* const v = reinterpret_cast<const float4*>(k.rope.table + (int64_t)p * (D / 2) + 4 * l);
            u[0] = v[0];
            u[1] = v[1];
        };
        uint2 rd[8][2], rx[8][2];
        float4 next[2];
        turn_row(pos[0], next);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint16_t* const g = gp + i * h.grs + 4 * l;
            rd[i][0] = *reinterpret_cast<const uint2*>(g);
            rd[i][1] = *reinterpret_cast<const uint2*>(g + D / 2);
            rx[i][0] = *reinterpret_cast<const uint2*>(xp + i * h.xrs);
            rx[i][1] = *reinterpret_cast<const uint2*>(xp + i * h.xrs + D / 2);
        }
        uint2 gw[2] = {};
        if (L == 16 || h.gamma) {
            gw[0] = *reinterpret_cast<const uint2*>(h.gamma + 4 * l);
            gw[1] = *reinterpret_cast<const uint2*>(h.gamma + D / 2 + 4 * l);
        }
        __builtin_amdgcn_sched_barrier(0);
        // a wave's four rows of 256 bytes, odd ones with their halves swapped
        // (so that two rows' 8-byte pieces do not meet in a bank)
        const int r = lane >> 4, swap = (r & 1) << 7, at = (lane & 15) / L * (D * 2) + 8 * l;
        uint8_t* const mine = stage[threadIdx.x >> 6] + r * 256;
        constexpr float inv_d = 1.0f / (float)D;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 u[2] = {next[0], next[1]};
            if (i < 7) turn_row(pos[i + 1], next);
            float d[8], x8[8], wg[8], gm[8];
            unpack8(make_uint4(rd[i][0].x, rd[i][0].y, rd[i][1].x, rd[i][1].y), d);
            unpack8(make_uint4(rx[i][0].x, rx[i][0].y, rx[i][1].x, rx[i][1].y), x8);
            asm volatile("" : "+v"(gw[0].x), "+v"(gw[0].y), "+v"(gw[1].x), "+v"(gw[1].y));
            unpack8(make_uint4(gw[0].x, gw[0].y, gw[1].x, gw[1].y), gm);
            const float c[4] = {u[0].x, u[0].z, u[1].x, u[1].z}, sn[4] = {u[0].y, u[0].w, u[1].y, u[1].w};
            turn_pairs4(d, c, sn, true);
            norm_bwd8<L, false>(d, x8, gm, inv_d, k.eps, wg);
            const uint4 n = pack8(d);
            uint2 lo = make_uint2(n.x, n.y), hi = make_uint2(n.z, n.w);
            if constexpr (L == 8) {
                lo.x = kind != 2 ? lo.x : rd[i][0].x; lo.y = kind != 2 ? lo.y : rd[i][0].y;
                hi.x = kind != 2 ? hi.x : rd[i][1].x; hi.y = kind != 2 ? hi.y : rd[i][1].y;
            }
            __builtin_amdgcn_wave_barrier();
            *reinterpret_cast<uint2*>(mine + (at ^ swap)) = lo;
            *reinterpret_cast<uint2*>(mine + ((at + D) ^ swap)) = hi;
            __builtin_amdgcn_wave_barrier();
            const uint4 o = *reinterpret_cast<const uint4*>(mine + (((lane & 15) * 16) ^ swap));
            w[i][0] = o.x; w[i][1] = o.y; w[i][2] = o.z; w[i][3] = o.w;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum[e] += wg[e];
                asm volatile("" : "+v"(sum[e]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = live ? sum[e] : 0.0f;
    }
    if (!wave_none(!live)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i][j] = live ? w[i][j] : 0u;
    }
}

enum : int { kQkAmax = 0, kQkTensor = 1, kQkRow = 2, kQkRowCol = 3, kQkCol = 4 };

// One tile per block. The block's sums for dgamma go to
// k.part[tile row][head][D] (query and key heads), in the one pass that the
// grouped modes take and in the amax pass of the per-tensor mode.
template <int FMT, int MODE, int L, bool USUAL, bool FLOOR = false>
__global__ __launch_bounds__(kThreads) void qk_bwd_quant_kernel(Kinds kinds, QuantArgs a, QkArgs k, Divisor per_seq,
                                                                uint32_t* partial) {
    constexpr bool GROUPS = MODE >= kQkRow;
    constexpr bool ROWS = MODE == kQkRow || MODE == kQkRowCol, COLS = MODE == kQkRowCol || MODE == kQkCol;
    (void)kinds;      // (read where they lie, by number)
    __shared__ uint32_t red[4];
    __shared__ uint32_t colmax[COLS ? 4 : 1][kTile / 2];
    __shared__ float sums[MODE == kQkTensor ? 1 : 4][kTile];
    __shared__ __attribute__((aligned(16))) uint8_t stage[USUAL ? 4 : 1][1024];
    __shared__ __attribute__((aligned(16))) uint8_t tq[COLS || MODE == kQkTensor ? kTile * kTile : 16];
    const int bx = blockIdx.x;
    const int64_t by = blockIdx.y;
    const Tile t = tile_coords(a.cols, bx, by);
    const int head0 = L == 16 ? bx : bx * 2;
    PartialShare ps;
    if constexpr (MODE == kQkTensor) ps = load_partials(a);
    uint32_t w[8][4];
    float sum[8];
    int col[2];
    if constexpr (USUAL) load_qk_bwd_usual<L>(k, per_seq, t, head0, stage, w, sum, col);
    // (twice: one that always looks for tiny heads takes 137 to 140 registers in
    // groups, 56 -> 64 us where query heads alone are normalised)
    else if (k.eps < kLeastMean) load_qk_bwd_any<L, true>(k, per_seq, t, head0, w, sum, col);
    else load_qk_bwd_any<L, false>(k, per_seq, t, head0, w, sum, col);
    if constexpr (MODE != kQkTensor) {
        if (k.part && head0 < k.hq + k.hk) {
            // the wave's four row groups (16 lanes apart), then the four waves
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = sum[e];
                s += __shfl_xor(s, 16, 64);
                s += __shfl_xor(s, 32, 64);
                if ((threadIdx.x & 63) < 16) sums[threadIdx.x >> 6][col[e / 4] + e % 4] = s;
            }
            __syncthreads();
            if (threadIdx.x < kTile) {
                const int c = threadIdx.x, h = L == 16 ? bx : bx * 2 + (c >> 6), d = L == 16 ? c : c & 63;
                if (h < k.hq + k.hk) {
                    const float s = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
                    // all tile rows' query heads, then all tile rows' key heads
                    const int64_t at = h < k.hq ? by * k.hq + h
                                                : (int64_t)gridDim.y * k.hq + by * k.hk + (h - k.hq);
                    k.part[at * k.D + d] = s;
                }
            }
        }
    }
    if constexpr (MODE == kQkAmax) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, absmax_bits8(w[i]));
        m = block_max(m, red);
        if (threadIdx.x == 0) partial[by * gridDim.x + bx] = m;
    } else if constexpr (GROUPS) {
        quant_groups_tile<FMT, ROWS, COLS, FLOOR>(a, t, bx, by, w, colmax, tq);
    } else {
        const TensorScale sc = tensor_scale<FMT>(a, tensor_amax(a, ps, red));
        if (bx == 0 && by == 0 && threadIdx.x == 0 && a.scale) a.scale[0] = sc.s;
        store_tensor_codes<FMT>(a, t, sc, by * kTile, (int64_t)bx * kTile, w, tq);
    }
}

template <int FMT, int L, bool USUAL>
void launch_fmt(int mode, QuantArgs a, const QkArgs& k, void* ws, hipStream_t stream) {
    const dim3 grid((unsigned)tiles_x(a.cols), (unsigned)tiles_y(a.rows));
    const Divisor per_seq = Divisor::of((uint32_t)k.seq);
    const Kinds kinds = kinds_of(k);
    uint32_t* partial = reinterpret_cast<uint32_t*>(ws);
    switch (mode) {
    case kQTensor:
        qk_bwd_quant_kernel<kE4M3, kQkAmax, L, USUAL><<<grid, kThreads, 0, stream>>>(kinds, a, k, per_seq, partial);
        amax_source(a, (int)(grid.x * grid.y), ws, stream);
        qk_bwd_quant_kernel<FMT, kQkTensor, L, USUAL><<<grid, kThreads, 0, stream>>>(kinds, a, k, per_seq, partial);
        break;
    case kQRow:
        by_rule(a, [&](auto floor) {
            constexpr bool FLOOR = decltype(floor)::value;
            if (a.qT) qk_bwd_quant_kernel<FMT, kQkRowCol, L, USUAL, FLOOR><<<grid, kThreads, 0, stream>>>(kinds, a, k, per_seq, partial);
            else qk_bwd_quant_kernel<FMT, kQkRow, L, USUAL, FLOOR><<<grid, kThreads, 0, stream>>>(kinds, a, k, per_seq, partial);
        });
        break;
    case kQCol:
        by_rule(a, [&](auto floor) {
            qk_bwd_quant_kernel<FMT, kQkCol, L, USUAL, decltype(floor)::value><<<grid, kThreads, 0, stream>>>(kinds, a, k, per_seq, partial);
        });
        break;
    }
}

// The tiles' maxima and the reduced one, then the partial sums of dgamma.
size_t sums_at(int64_t tokens, int hq, int hk, int D) {
    const int64_t tiles = tiles_x((int64_t)(hq + 2 * hk) * D) * tiles_y(tokens);
    return (((size_t)tiles * sizeof(uint32_t) + 255) / 256 * 256 + sizeof(float) + 255) / 256 * 256;
}

}  // namespace

size_t qk_bwd_quantize_ws_bytes(int64_t tokens, int hq, int hk, int D) {
    return sums_at(tokens, hq, hk, D) + (size_t)(tiles_y(tokens) * (hq + hk)) * D * sizeof(float);
}

void launch_qk_norm_rope_bwd_quantize(int fmt, int mode, QuantArgs a, QkArgs k, void* ws, hipStream_t stream) {
    const bool sums = k.dgq || k.dgk;
    const int64_t gy = tiles_y(a.rows);
    k.part = sums ? reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ws) + sums_at(k.tokens, k.hq, k.hk, k.D)) : nullptr;
    if (a.rows == 0 || a.cols == 0) {
        // the scale of an empty tensor, sums of nothing
        if (mode == kQTensor) {
            amax_source(a, 0, ws, stream);
            launch_quantize(fmt, kQTensor, a, stream);
        }
        if (sums) launch_dgamma_sum(k.part, 0, k.dgq, k.part, 0, k.dgk, k.D, k.D, stream);
        return;
    }
    auto run = [&](auto fmt_c) {
        constexpr int FMT = decltype(fmt_c)::value;
        const bool usual = k.gq && k.gk && k.eps >= kLeastMean && turn_kind(k.rope, k.D / 8) == kTurnHalf && k.seq % 8 == 0;
        if (k.D == 128) {
            if (usual) launch_fmt<FMT, 16, true>(mode, a, k, ws, stream);
            else launch_fmt<FMT, 16, false>(mode, a, k, ws, stream);
        } else {
            if (usual) launch_fmt<FMT, 8, true>(mode, a, k, ws, stream);
            else launch_fmt<FMT, 8, false>(mode, a, k, ws, stream);
        }
    };
    if (fmt == kE4M3) run(std::integral_constant<int, kE4M3>{});
    else run(std::integral_constant<int, kE5M2>{});
    if (sums)
        launch_dgamma_sum(k.part, gy * k.hq, k.dgq, k.part + gy * k.hq * k.D, gy * k.hk, k.dgk, k.D, k.D, stream);
}

}  // namespace puro
