// The backward of the query / key norm with rotation, quantised as it is formed
// (gfx950): the gradient of the QKV projection's output is the dY of that
// projection's Dgrad and Wgrad (Section 3.2 quantises it right before them),
// so its BF16 values never go to memory.
//
// A block takes a 128 x 128 tile, as the quantisers do: a head of 128 values,
// or two of 64, is a tile's width, and the 16 (8) lanes that hold a head's row
// exchange its pairs and its sums by lane moves. Bound by memory: 4 bytes read
// and 1 byte a copy written per query and key value, 2 and 1 per value head's.

#include "qk_norm_rope.h"
#include "quant_tile.h"

namespace puro {

namespace {

// The thread's 8x8 block of [dq | dk | dv] (BF16 bits), and what its columns
// add to dgamma, from the head of L lanes it belongs to; kind: 0 a query head,
// 1 a key head, 2 a value head or none.
template <int L>
__device__ __forceinline__ void load_qk_bwd_8x8(const QkArgs& k, const Divisor& per_seq, const Tile& t, int head,
                                                uint32_t w[8][4], float sum[8], int& kind) {
    const int hqk = k.hq + k.hk;
    const bool none = head >= hqk + k.hk;      // the last head again, and zeros
    head = min(head, hqk + k.hk - 1);
    kind = head < k.hq ? 0 : (head < hqk ? 1 : 2);
    const LaneRole role = lane_role<L>(k.D, k.rope.dim, k.rope.interleaved, threadIdx.x & 63);
    const HeadsArg g = kind == 0 ? k.dq : (kind == 1 ? k.dk : k.dv);
    const int first = kind == 0 ? 0 : (kind == 1 ? k.hq : hqk);
    const uint16_t* gamma = kind == 0 ? k.gq : (kind == 1 ? k.gk : nullptr);
    const bool norm = gamma != nullptr;
    // (heads that are not normalised are not read: the gradient stands in)
    const HeadsArg x = norm ? (kind == 0 ? k.q : k.k) : g;
    const int64_t hc = head - first;
    const uint16_t* const gp = g.p + hc * g.hs + role.col;
    const uint16_t* const xp = x.p + hc * x.hs + role.col;
    const int rows = (int)max((int64_t)0, min((int64_t)8, k.tokens - t.row0));   // of the thread's eight
    uint4 rd[8], rx[8];
    int pos[8];
    const bool turned = k.rope.dim > 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // rows past the last are the last one again, and zeros below
        const int row = (int)min(t.row0 + i, k.tokens - 1);
        const Token tok = token_of(row, per_seq);
        rd[i] = *reinterpret_cast<const uint4*>(gp + tok.b * g.bs + tok.s * g.rs);
        rx[i] = *reinterpret_cast<const uint4*>(xp + tok.b * x.bs + tok.s * x.rs);
        pos[i] = tok.s;
        if (turned && k.rope.pos) pos[i] = k.rope.pos[row];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    if (wave_none(kind != 2)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool live = i < rows && !none;
            w[i][0] = live ? rd[i].x : 0u; w[i][1] = live ? rd[i].y : 0u;
            w[i][2] = live ? rd[i].z : 0u; w[i][3] = live ? rd[i].w : 0u;
        }
        return;
    }
    float gm[8];
    uint4 gw{};
    if (norm) gw = *reinterpret_cast<const uint4*>(gamma + role.col);
    unpack8(gw, gm);
    const float inv_d = 1.0f / (float)k.D;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float d[8], n[8], x8[8], wg[8];
        unpack8(rd[i], d);
        if (turned) {
            const Turn turn = load_turn(k.rope, role, pos[i], true);
            turn8<L>(d, turn, role, k.rope.interleaved, k.rope.dim == L * 8);
        }
        unpack8(rx[i], x8);
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = d[e];
        norm_bwd8<L>(n, x8, gm, inv_d, k.eps, wg);
        const bool live = i < rows && !none;
        uint4 o = rd[i];
        if (kind != 2) o = pack8(norm ? n : d);
        w[i][0] = live ? o.x : 0u; w[i][1] = live ? o.y : 0u;
        w[i][2] = live ? o.z : 0u; w[i][3] = live ? o.w : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += live && norm ? wg[e] : 0.0f;
    }
}

enum : int { kQkAmax = 0, kQkTensor = 1, kQkRow = 2, kQkRowCol = 3, kQkCol = 4 };

// One tile per block. The block's sums for dgamma go to
// k.part[tile row][head][D] (query and key heads), in the one pass that the
// grouped modes take and in the amax pass of the per-tensor mode.
template <int FMT, int MODE, int L, bool FLOOR = false>
__global__ __launch_bounds__(kThreads) void qk_bwd_quant_kernel(QuantArgs a, QkArgs k, Divisor per_seq,
                                                                uint32_t* partial) {
    constexpr bool GROUPS = MODE >= kQkRow;
    constexpr bool ROWS = MODE == kQkRow || MODE == kQkRowCol, COLS = MODE == kQkRowCol || MODE == kQkCol;
    __shared__ uint32_t red[4];
    __shared__ uint32_t colmax[COLS ? 4 : 1][kTile / 2];
    __shared__ float sums[MODE == kQkTensor ? 1 : 4][kTile];
    __shared__ __attribute__((aligned(16))) uint8_t tq[COLS || MODE == kQkTensor ? kTile * kTile : 16];
    const int bx = blockIdx.x;
    const int64_t by = blockIdx.y;
    const Tile t = tile_coords(a.cols, bx, by);
    const int head = L == 16 ? bx : bx * 2 + (t.cc >> 3);
    PartialShare ps;
    if constexpr (MODE == kQkTensor) ps = load_partials(a);
    uint32_t w[8][4];
    float sum[8];
    int kind;
    load_qk_bwd_8x8<L>(k, per_seq, t, head, w, sum, kind);
    if constexpr (MODE != kQkTensor) {
        if (k.part && __builtin_amdgcn_readfirstlane(L == 16 ? head : bx * 2) < k.hq + k.hk) {
            // the wave's four row groups (16 lanes apart), then the four waves
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float s = sum[e];
                s += __shfl_xor(s, 16, 64);
                s += __shfl_xor(s, 32, 64);
                if ((threadIdx.x & 63) < 16) sums[threadIdx.x >> 6][t.cc * 8 + e] = s;
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

template <int FMT, int L>
void launch_fmt(int mode, QuantArgs a, const QkArgs& k, void* ws, hipStream_t stream) {
    const dim3 grid((unsigned)tiles_x(a.cols), (unsigned)tiles_y(a.rows));
    const Divisor per_seq = Divisor::of((uint32_t)k.seq);
    uint32_t* partial = reinterpret_cast<uint32_t*>(ws);
    switch (mode) {
    case kQTensor:
        qk_bwd_quant_kernel<kE4M3, kQkAmax, L><<<grid, kThreads, 0, stream>>>(a, k, per_seq, partial);
        amax_source(a, (int)(grid.x * grid.y), ws, stream);
        qk_bwd_quant_kernel<FMT, kQkTensor, L><<<grid, kThreads, 0, stream>>>(a, k, per_seq, partial);
        break;
    case kQRow:
        by_rule(a, [&](auto floor) {
            constexpr bool FLOOR = decltype(floor)::value;
            if (a.qT) qk_bwd_quant_kernel<FMT, kQkRowCol, L, FLOOR><<<grid, kThreads, 0, stream>>>(a, k, per_seq, partial);
            else qk_bwd_quant_kernel<FMT, kQkRow, L, FLOOR><<<grid, kThreads, 0, stream>>>(a, k, per_seq, partial);
        });
        break;
    case kQCol:
        by_rule(a, [&](auto floor) {
            qk_bwd_quant_kernel<FMT, kQkCol, L, decltype(floor)::value><<<grid, kThreads, 0, stream>>>(a, k, per_seq, partial);
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
        if (k.D == 128) launch_fmt<FMT, 16>(mode, a, k, ws, stream);
        else launch_fmt<FMT, 8>(mode, a, k, ws, stream);
    };
    if (fmt == kE4M3) run(std::integral_constant<int, kE4M3>{});
    else run(std::integral_constant<int, kE5M2>{});
    if (sums)
        launch_dgamma_sum(k.part, gy * k.hq, k.dgq, k.part + gy * k.hq * k.D, gy * k.hk, k.dgk, k.D, k.D, stream);
}

}  // namespace puro
