// A 128x128 tile of a quantisation: which values a thread holds, the scales and
// the stores of the codes and their transposed copy. Shared by the quantisers
// (quant.hip, qk_quant.hip), which differ in where a tile's values come from.
#pragma once

#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;
typedef int v4i __attribute__((ext_vector_type(4)));
// Above this many partial maxima a one-block kernel reduces them once,
// rather than every block of the quantise pass reading them all.
constexpr int kMaxInlinePartials = 2048;

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}

// Whether no (active) lane of the wave has `c`.
__device__ __forceinline__ bool wave_none(bool c) { return __builtin_amdgcn_ballot_w64(c) == 0; }

// Maxima across lanes without LDS: over a row of 16 lanes by rotations within
// it (every lane gets it), and of the lanes 16 or 32 apart by row swaps.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));   // row_ror:8
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));   // row_ror:4
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));   // row_ror:2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));   // row_ror:1
}
__device__ __forceinline__ uint32_t pk_max_rows(uint32_t v) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = pk_max_u16(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return pk_max_u16(b[0], b[1]);
}

// Block-wide max of a per-thread value (256 threads); result in every thread.
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
    v = wave_max(v);
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}

struct Tile {
    int cc, rg;       // column chunk (8 columns) and row group (8 rows) of this thread
    int64_t row0;     // first of the thread's 8 rows
    int64_t col;      // first of the thread's 8 columns
    bool col_ok;
};

// The thread's 8x8 block in tile (bx, by) (tile column, tile row).
__device__ __forceinline__ Tile tile_coords(int64_t cols, int64_t bx, int64_t by) {
    Tile t;
    t.cc = threadIdx.x & 15;
    t.rg = threadIdx.x >> 4;
    t.row0 = by * kTile + t.rg * 8;
    t.col = bx * kTile + t.cc * 8;
    t.col_ok = t.col < cols;
    return t;
}
__device__ __forceinline__ Tile tile_coords(int64_t cols) { return tile_coords(cols, blockIdx.x, blockIdx.y); }

// Buffer descriptor over `bytes` bytes from `base` (32-bit raw data): loads
// at offsets at or beyond `bytes` return zeros and touch no memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_rsrc(const void* base, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
constexpr uint32_t kOOB = 0x80000000u;   // an offset beyond every descriptor's range (ld < 2^23)

__device__ __forceinline__ void store_rows(const QuantArgs& a, const Tile& t, const uint2 c[8]) {
    if (!t.col_ok) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = t.row0 + i;
        if (r < a.rows) *reinterpret_cast<uint2*>(a.q + r * a.cols + t.col) = c[i];
    }
}

// qT [cols, rows] of the tile whose first element is (row0, col0), from the
// codes c of every thread's 8x8 block. Column j of a thread's block becomes
// 8 bytes of LDS row col + j (LDS row r = qT row col0 + r, 128 bytes = the
// tile's rows); then each lane stores 16 bytes, eight lanes one whole
// 128-byte run of a qT row. The 16-byte chunk h of LDS row r sits at
// position h ^ ((r >> 3) & 7): the 8-byte writes of a wave (rows 8 apart
// across lanes) then spread over the banks, and a wave's 16-byte reads of 8
// consecutive rows cover all 64 banks four times (the minimum). rows % 16 ==
// 0, so a 16-byte run never crosses the end of a qT row. Ends with a barrier,
// after which the LDS buffer may be reused. qT not 16-byte aligned: 8-byte
// stores straight from registers.
__device__ __forceinline__ void store_transposed_ct(const QuantArgs& a, const Tile& t, int64_t row0, int64_t col0,
                                                    const uint2 ct[8], uint8_t* lds) {
    if ((reinterpret_cast<uintptr_t>(a.qT) & 15) != 0) {
        if (!t.col_ok || t.row0 >= a.rows) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *reinterpret_cast<uint2*>(a.qT + (t.col + j) * a.rows + t.row0) = ct[j];
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = t.cc * 8 + j;
        const int pos = (((t.rg >> 1) ^ (r >> 3 & 7)) << 4) + ((t.rg & 1) << 3);
        *reinterpret_cast<uint2*>(lds + r * kTile + pos) = ct[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTile * kTile / 16 / kThreads; ++i) {
        const int q = i * kThreads + threadIdx.x;
        const int r = q >> 3, h = q & 7;
        const uint4 v = *reinterpret_cast<const uint4*>(lds + r * kTile + ((h ^ (r >> 3 & 7)) << 4));
        const int64_t col = col0 + r, row = row0 + h * 16;
        if (col < a.cols && row < a.rows) *reinterpret_cast<uint4*>(a.qT + col * a.rows + row) = v;
    }
    __syncthreads();
}

// The same from the codes of the thread's 8x8 block in row order.
__device__ __forceinline__ void store_transposed(const QuantArgs& a, const Tile& t, int64_t row0, int64_t col0,
                                                 const uint2 c[8], uint8_t* lds) {
    uint2 ct[8];
    transpose8x8(c, ct);
    store_transposed_ct(a, t, row0, col0, ct, lds);
}

// Scale of a per-tensor quantisation: s (stored) and the multiplier r, and
// whether encoding must take the saturating path (the amax was supplied and
// values beyond it saturate, the floor rule clips the top values, or the
// amax or r is not finite).
struct TensorScale {
    float s, r;
    bool safe;
};

template <int FMT>
__device__ __forceinline__ TensorScale tensor_scale(const QuantArgs& a, float amax) {
    float s, r;
    bool saturate = a.supplied != 0;
    constexpr float fm = Fp8Traits<FMT>::kMax;
    if (a.pow2) {
        if (amax != amax) {
            s = r = __uint_as_float(0x7FC00000u);
        } else {
            // |amax| as a BF16-or-wider magnitude: reuse the exponent rule on its top bits
            const uint32_t bits = __float_as_uint(fabsf(amax));
            int e;
            if (bits == 0) e = 0;
            else if (bits >= 0x7F800000u) e = 127;
            else if ((bits >> 23) == 0) e = -127;
            else {
                const bool above = (bits & 0x7FFFFFu) > 0x600000u;   // significand > 1.75
                e = (int)(bits >> 23) - 127 - Fp8Traits<FMT>::kEmax + (a.pow2 != 2 && above ? 1 : 0);
                e = e < -127 ? -127 : (e > 127 ? 127 : e);
                // the floor rule (pow2 == 2) saturates the top values of such a tensor
                saturate = saturate || (a.pow2 == 2 && above);
            }
            s = exp2i(e);
            r = exp2i(-e);
        }
    } else if (amax == 0.0f) {
        s = r = 1.0f;
    } else {
        s = amax / fm;
        r = fm / amax;
    }
    return {s, r, saturate || !(fabsf(amax) <= 3.4028235e38f) || !(fabsf(r) <= 3.4028235e38f)};
}

// Partial maxima of a tensor's amax pass as this thread reads them (its
// share of at most kMaxInlinePartials), issued before the tile loads so
// that they return first and the reduction overlaps the tile's arrival.
struct PartialShare {
    uint32_t v[kMaxInlinePartials / kThreads];
};

// Buffer loads: entries past the partials (all of them when the amax is a
// device scalar) read as zeros, which leave the maximum unchanged.
__device__ __forceinline__ PartialShare load_partials(const QuantArgs& a, bool active = true) {
    PartialShare p;
    const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(a.partial, (!active || a.amax) ? 0u : (uint32_t)a.npartial * 4u);
#pragma unroll
    for (int u = 0; u < kMaxInlinePartials / kThreads; ++u)
        p.v[u] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, (u * kThreads + threadIdx.x) * 4u, 0, 0);
    return p;
}

// The tensor's amax: the supplied or finalised device scalar, or the block's
// reduction of the partial maxima (every thread gets it).
__device__ __forceinline__ float tensor_amax(const QuantArgs& a, const PartialShare& p, uint32_t* red) {
    if (a.amax) return *a.amax;
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < kMaxInlinePartials / kThreads; ++u) m = max(m, p.v[u]);
    m = block_max(m, red);
    return __uint_as_float(m << 16);
}

// The codes of a per-tensor quantisation's tile at (row0, col0), q and qT.
template <int FMT>
__device__ __forceinline__ void store_tensor_codes(const QuantArgs& a, const Tile& t, const TensorScale& sc, int64_t row0,
                                                   int64_t col0, const uint32_t w[8][4], uint8_t* tq) {
    uint2 c[8];
    if (sc.safe) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = encode8<FMT, true>(w[i], sc.r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = encode8<FMT, false>(w[i], sc.r);
    }
    if (a.q) store_rows(a, t, c);
    if (a.qT) store_transposed(a, t, row0, col0, c, tq);
}

// 1x128 row groups (q, scale) and/or 128x1 column groups (qT, scaleT) of the
// tile in tile column bx and tile row by, from the BF16 values w of every
// thread's 8x8 block. colmax: packed pairs of column maxima per wave; tq: the
// transposed copy's staging; FLOOR: the floor rule's scales.
template <int FMT, bool ROWS, bool COLS, bool FLOOR>
__device__ __forceinline__ void quant_groups_tile(const QuantArgs& a, const Tile& t, int64_t bx, int64_t by,
                                                  const uint32_t w[8][4], uint32_t (*colmax)[kTile / 2], uint8_t* tq) {
    // (asked at run time in the other rules' instance too: with the careful
    // path's test folded away the compiler orders the common path's code
    // otherwise, 2 to 5% slower: [16384, 1536], rows and columns, 20.0 -> 21.0 us)
    const bool floor_rule = FLOOR || a.pow2 == 2;

    if constexpr (ROWS) {
        uint2 c[8];
        float srow[8];
        uint32_t m[8];
        int e[8];
        PlainExponents<FMT> plain;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = row16_max(absmax_bits8(w[i]));
            e[i] = plain.exponent(m[i], floor_rule);
        }
        if (wave_none(plain.any(floor_rule))) {
            // straight-line for all eight rows
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                srow[i] = exp2i(e[i]);
                c[i] = encode8_pow2<FMT>(w[i], srow[i]);
            }
        } else if (FLOOR && wave_none(plain.outside())) {
            // the floor rule with groups to clip, straight-line too (the
            // groups that need no clipping get the same codes): a branch per
            // group cost the SwiGLU backward's blocks, which take two tiles
            // one after the other, 22.3 against 17.5 us at dH [256, 1024]
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                srow[i] = exp2i(e[i]);
                c[i] = encode8<FMT, true>(w[i], exp2i(-e[i]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (m[i] <= 0x7F7Fu) {                      // finite group
                    const int ei = pow2_exponent_bf16<FMT>(m[i], floor_rule);
                    srow[i] = exp2i(ei);
                    if (floor_rule && floor_rule_saturates(m[i])) c[i] = encode8<FMT, true>(w[i], exp2i(-ei));
                    else if (ei > -127) c[i] = encode8_pow2<FMT>(w[i], srow[i]);
                    else c[i] = encode8<FMT, false>(w[i], exp2i(-ei));
                } else if (m[i] == 0x7F80u) {               // an infinity: largest scale, saturate
                    srow[i] = exp2i(127);
                    c[i] = encode8<FMT, true>(w[i], exp2i(-127));
                } else {                                    // a NaN: NaN scale, NaN codes
                    srow[i] = __uint_as_float(0x7FC00000u);
                    c[i] = encode8<FMT, true>(w[i], srow[i]);
                }
            }
        }
        store_rows(a, t, c);
        if (t.cc == 0) {
            const int64_t ng = a.cols / kTile;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t r = t.row0 + i;
                if (r < a.rows) a.scale[a.kmajor ? bx * a.rows + r : r * ng + bx] = srow[i];
            }
        }
    }
    if constexpr (COLS) {
        // column maxima over the tile's 128 rows, two columns per word (the
        // two magnitude patterns of a word in its halves): 8 rows in-thread,
        // 4 row groups per wave (lanes 16 apart), 4 waves through LDS
        uint32_t cm[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = mag2(w[0][j]);
#pragma unroll
            for (int i = 1; i < 8; ++i) m = pk_max_u16(m, mag2(w[i][j]));
            cm[j] = pk_max_rows(m);
        }
        const int wv = threadIdx.x >> 6;
        if ((threadIdx.x & 63) < 16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) colmax[wv][t.cc * 4 + j] = cm[j];
        }
        __syncthreads();
        uint32_t cw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = t.cc * 4 + j;
            cw[j] = pk_max_u16(pk_max_u16(colmax[0][k], colmax[1][k]), pk_max_u16(colmax[2][k], colmax[3][k]));
        }
        float scol[8];
        int e[8];
        PlainExponents<FMT> plain;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t m = (j & 1) ? (cw[j >> 1] >> 16) : (cw[j >> 1] & 0xFFFFu);
            e[j] = plain.exponent(m, floor_rule);
            scol[j] = exp2i(e[j]);
        }
        uint2 ct[8];
        if (wave_none(plain.any(floor_rule))) {
            // transpose the BF16 block first: each column then shares one
            // scale, and its codes come out in the transposed copy's order
            uint32_t wt[8][4];
            transpose8x8_b16(w, wt);
#pragma unroll
            for (int j = 0; j < 8; ++j) ct[j] = encode8_pow2<FMT>(wt[j], scol[j]);
        } else if (FLOOR && wave_none(plain.outside())) {
            uint32_t wt[8][4];
            transpose8x8_b16(w, wt);
#pragma unroll
            for (int j = 0; j < 8; ++j) ct[j] = encode8<FMT, true>(wt[j], exp2i(-e[j]));
        } else {
            float rcol[8];
            bool finite = true;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t m = (j & 1) ? (cw[j >> 1] >> 16) : (cw[j >> 1] & 0xFFFFu);
                if (m <= 0x7F7Fu) {
                    const int e = pow2_exponent_bf16<FMT>(m, floor_rule);
                    scol[j] = exp2i(e);
                    rcol[j] = exp2i(-e);
                    if (floor_rule && floor_rule_saturates(m)) finite = false;   // take the saturating path
                } else if (m == 0x7F80u) {
                    scol[j] = exp2i(127);
                    rcol[j] = exp2i(-127);
                    finite = false;
                } else {
                    scol[j] = rcol[j] = __uint_as_float(0x7FC00000u);
                    finite = false;
                }
            }
            uint2 c[8];
            if (finite) {
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i] = encode8_cols<FMT, false>(w[i], rcol);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i] = encode8_cols<FMT, true>(w[i], rcol);
            }
            transpose8x8(c, ct);
        }
        store_transposed_ct(a, t, by * kTile, bx * kTile, ct, tq);
        if (t.rg == 0 && t.col_ok) {
            const int64_t ng = a.rows / kTile;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                a.scaleT[a.kmajor ? by * a.cols + t.col + j : (t.col + j) * ng + by] = scol[j];
        }
    }
}

// f(floor) with the floor rule as a type: a kernel instance of its own, since
// its clipping path in the other rules' instances cost their small calls 3 to
// 4% (SwiGLU backward, dH [256, 1024]: 11.6 against 12.1 us).
template <class F>
void by_rule(const QuantArgs& a, F&& f) {
    if (a.pow2 == 2) f(std::true_type{});
    else f(std::false_type{});
}

// Amax source of a per-tensor quantisation whose partial maxima are in ws:
// reduced by every quantise block (few partials) or once by a one-block
// kernel into the amax slot of ws.
void amax_source(QuantArgs& a, int P, void* ws, hipStream_t stream) {
    uint32_t* partial = reinterpret_cast<uint32_t*>(ws);
    a.supplied = 0;
    if (P > kMaxInlinePartials) {
        float* amax = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ws) + ((size_t)P * 4 + 255) / 256 * 256);
        launch_amax_finalize(partial, P, amax, stream);
        a.amax = amax;
    } else {
        // an empty tensor (P = 0) reduces to amax 0: scale 1
        a.amax = nullptr;
        a.partial = partial;
        a.npartial = P;
    }
}

int64_t tiles_x(int64_t cols) { const int64_t g = (cols + kTile - 1) / kTile; return g > 0 ? g : 1; }
int64_t tiles_y(int64_t rows) { const int64_t g = (rows + kTile - 1) / kTile; return g > 0 ? g : 1; }

}  // namespace

}  // namespace puro
