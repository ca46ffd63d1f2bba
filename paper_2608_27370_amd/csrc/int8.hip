// 8-bit integer linear layers for gfx950: the quantisation of rows (tokens, output
// channels) and of columns (transposed copies) to int8, and the product of int8
// codes with a scale for each row of either operand.

#include "gemm_common.h"
#include "quant_tile.h"

namespace puro {

using gemm_detail::add_epilogue1;
using gemm_detail::add_epilogue4;
using gemm_detail::scaled_sum;

namespace {

// ---------------------------------------------------------------- encoding ---
// code = the integer nearest to x r, ties to even: one fused multiply-add with
// 1.5 2^23, where binary32's last place is 1, rounds the exact product once; the
// low byte of the sum's pattern is the code (two's complement). A product that is
// NaN (r = 0 times an infinity, NaN) gives a quiet NaN, whose low byte is 0.
constexpr float kRound = 12582912.0f;
__device__ __forceinline__ uint32_t code_bits(float x, float r) { return __float_as_uint(__builtin_fmaf(x, r, kRound)); }
__device__ __forceinline__ uint32_t pack_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), cd = __builtin_amdgcn_perm(d, c, 0x0C0C0400u);
    return __builtin_amdgcn_perm(cd, ab, 0x05040100u);
}

// Scale s, factor r and (rows below 2^-100, where 127 / amax would overflow) the
// power of two that the values are multiplied by first, from the bits of amax.
struct Int8Scale {
    float s, r, pre;
};
__device__ __forceinline__ Int8Scale int8_scale(uint32_t amax_bits) {
    if (amax_bits >= 0x7F800000u) return {__uint_as_float(0x7FC00000u), 0.0f, 1.0f};
    if (amax_bits == 0u) return {1.0f, 1.0f, 1.0f};
    const float a = __uint_as_float(amax_bits);
    const float pre = a < 0x1p-100f ? 0x1p64f : 1.0f;
    return {a / 127.0f, 127.0f / (a * pre), pre};
}
__device__ __forceinline__ uint2 encode_int8(const float v[8], const Int8Scale& s) {
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = code_bits(v[i] * s.pre, s.r);
    return make_uint2(pack_codes(c[0], c[1], c[2], c[3]), pack_codes(c[4], c[5], c[6], c[7]));
}

// ---------------------------------------------------------------- rows ---
// TPR threads (16, a wave or the block) per row, whose NC chunks of 8 values a thread
// are loaded once, all together, and stay in registers between the row's largest
// magnitude and its codes. Bound by memory: a row is read once and its codes
// written (8192x8960: 38 us, 5.8 TB/s; SwiGLU 75 us, 4.9; RMSNorm 41 us; a short tensor
// is a launch and its latency, 1x1536 2.4 us).
// Rows of a norm whose mean square and eps together are below 2^-100, where binary32
// squares lose bits or vanish, are multiplied by 2^96 first; an eps of 2^-100 rules that
// out for a whole call (then what is lost is less than 2^-40 of the sum), and kRowNorm's
// instances do not look (8192x1536 with eps 0 10.6 us, else 9.9).
enum : int { kRowBf16 = 0, kRowNorm = 1, kRowSwiglu = 2, kRowNormSmall = 3 };
constexpr bool is_norm(int src) { return src == kRowNorm || src == kRowNormSmall; }
constexpr float kLeastMean = 0x1p-100f, kRowUp = 0x1p96f;

__device__ __forceinline__ void words(const uint4& v, uint32_t w[4]) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
__device__ __forceinline__ void floats(const uint32_t w[4], float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(w[i]); v[2 * i + 1] = bf16hi(w[i]); }
}
__device__ __forceinline__ uint32_t max_bits(const float v[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
// over the N lanes of a row
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = N / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <int N>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int o = N / 2; o >= 1; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
    return v;
}
// (up: 1, or what the row is multiplied by first)
__device__ __forceinline__ float sum_squares(const uint32_t w[4], float ss, float up = 1.0f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = bf16lo(w[i]) * up, hi = bf16hi(w[i]) * up;
        ss = fmaf(lo, lo, ss);
        ss = fmaf(hi, hi, ss);
    }
    return ss;
}
struct RowNorm {
    float rstd, up;
};
// The row's norm from a pass over its values, total(up) = the sum of (x up)^2 over the
// row in every thread of it.
template <int SRC, typename F>
__device__ __forceinline__ RowNorm row_norm(const QuantInt8Args& a, F&& total) {
    const float mean = total(1.0f) / (float)a.cols + a.eps;
    if constexpr (SRC == kRowNormSmall) {
        const float up = mean < kLeastMean ? kRowUp : 1.0f;
        return {1.0f / sqrtf(total(up) / (float)a.cols + a.eps * up * up), up};
    }
    return {1.0f / sqrtf(mean), 1.0f};
}
__device__ __forceinline__ void norm_values(const uint32_t x[4], const RowNorm& n, const uint32_t g[4], float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16lo(x[i]) * n.up * n.rstd * bf16lo(g[i]);
        v[2 * i + 1] = bf16hi(x[i]) * n.up * n.rstd * bf16hi(g[i]);
    }
}
__device__ __forceinline__ void swiglu_values(const uint32_t g[4], const uint32_t u[4], float v[8]) {
    auto all = [&](auto near_c) __attribute__((always_inline)) {
        constexpr bool NEAR = decltype(near_c)::value;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = swiglu1<NEAR>(bf16lo(g[i]), bf16lo(u[i]));
            v[2 * i + 1] = swiglu1<NEAR>(bf16hi(g[i]), bf16hi(u[i]));
        }
    };
    if (wave_none(absmax_bits8(g) > kNearGateBits)) all(std::true_type{});
    else all(std::false_type{});
}

template <int SRC, int TPR, int NC>
__device__ __forceinline__ void quant_rows(const QuantInt8Args& a, int64_t block, uint32_t* red, float* sums) {
    constexpr bool WAVE = TPR <= 64;
    const int t = threadIdx.x % TPR;
    const int64_t row = block * (kThreads / TPR) + threadIdx.x / TPR;
    if (WAVE && row >= a.rows) return;          // (all of a row's lanes; the block meets at no barrier)
    const int cpr = (int)(a.cols / 8);
    const uint16_t* xr = a.x + row * a.ld;
    constexpr int SECOND = SRC == kRowBf16 ? 0 : NC;
    uint4 x[NC], y[SECOND > 0 ? SECOND : 1];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = t + i * TPR;
        x[i] = make_uint4(0, 0, 0, 0);
        if constexpr (SECOND > 0) y[i] = x[i];
        if (c < cpr) {
            x[i] = *reinterpret_cast<const uint4*>(xr + c * 8);
            if constexpr (is_norm(SRC)) y[i] = *reinterpret_cast<const uint4*>(a.gamma + c * 8);
            if constexpr (SRC == kRowSwiglu) y[i] = *reinterpret_cast<const uint4*>(xr + a.cols + c * 8);
        }
    }
    RowNorm norm{1.0f, 1.0f};
    if constexpr (is_norm(SRC)) {
        norm = row_norm<SRC>(a, [&](float up) __attribute__((always_inline)) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                uint32_t w[4];
                words(x[i], w);
                ss = sum_squares(w, ss, up);
            }
            ss = lanes_sum<WAVE ? TPR : 64>(ss);
            if constexpr (!WAVE) {
                if constexpr (SRC == kRowNormSmall) __syncthreads();       // (the sums of the pass before have been read)
                if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
                __syncthreads();
                ss = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            }
            return ss;
        });
        if (a.rstd && t == 0) a.rstd[row] = norm.rstd * norm.up;
    }
    // the row's values: as they are loaded, formed twice (two products a value), or
    // formed once and kept
    float h[SRC == kRowSwiglu ? NC : 1][8];
    auto values = [&](int i, float v[8]) __attribute__((always_inline)) {
        uint32_t w[4], z[4];
        words(x[i], w);
        if constexpr (SRC == kRowBf16) floats(w, v);
        if constexpr (is_norm(SRC)) { words(y[i], z); norm_values(w, norm, z, v); }
        if constexpr (SRC == kRowSwiglu) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = h[i][e];
        }
    };
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        if constexpr (SRC == kRowBf16) {
            uint32_t w[4];
            words(x[i], w);
            m = max(m, absmax_bits8(w) << 16);
        } else {
            float v[8];
            if constexpr (SRC == kRowSwiglu) {
                uint32_t w[4], z[4];
                words(x[i], w);
                words(y[i], z);
                swiglu_values(w, z, h[i]);
            }
            values(i, v);
            m = max_bits(v, m);
        }
    }
    m = WAVE ? lanes_max<TPR>(m) : block_max(m, red);
    const Int8Scale s = int8_scale(m);
    if (t == 0) a.scale[row] = s.s;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = t + i * TPR;
        float v[8];
        values(i, v);
        if (c < cpr) *reinterpret_cast<uint2*>(a.q + row * a.cols + c * 8) = encode_int8(v, s);
    }
}

template <int SRC, int TPR, int NC>
__global__ __launch_bounds__(kThreads) void quant_rows_int8_kernel(QuantInt8Args a) {
    __shared__ uint32_t red[4];
    __shared__ float sums[4];
    quant_rows<SRC, TPR, NC>(a, blockIdx.x, red, sums);
}

// The rows of two tensors of one width, `b`'s blocks behind `a`'s.
template <int TPR, int NC>
__global__ __launch_bounds__(kThreads) void quant_two_rows_int8_kernel(QuantInt8Args a, QuantInt8Args b, int blocks) {
    __shared__ uint32_t red[4];
    const int i = (int)blockIdx.x;
    quant_rows<kRowBf16, TPR, NC>(i < blocks ? a : b, i < blocks ? i : i - blocks, red, nullptr);
}

// Rows longer than the registers hold: one block per row, the values formed twice
// (the second time from the caches).
template <int SRC>
__device__ __forceinline__ void row_values(const QuantInt8Args& a, const uint16_t* xr, int64_t c, const RowNorm& norm, float v[8]) {
    uint32_t w[4], z[4];
    words(*reinterpret_cast<const uint4*>(xr + c * 8), w);
    if constexpr (SRC == kRowBf16) floats(w, v);
    if constexpr (is_norm(SRC)) {
        words(*reinterpret_cast<const uint4*>(a.gamma + c * 8), z);
        norm_values(w, norm, z, v);
    }
    if constexpr (SRC == kRowSwiglu) {
        words(*reinterpret_cast<const uint4*>(xr + a.cols + c * 8), z);
        swiglu_values(w, z, v);
    }
}

template <int SRC>
__global__ __launch_bounds__(kThreads) void quant_long_rows_int8_kernel(QuantInt8Args a) {
    __shared__ uint32_t red[4];
    __shared__ float sums[4];
    const int64_t row = blockIdx.x, cpr = a.cols / 8;
    const uint16_t* xr = a.x + row * a.ld;
    RowNorm norm{1.0f, 1.0f};
    if constexpr (is_norm(SRC)) {
        norm = row_norm<SRC>(a, [&](float up) __attribute__((always_inline)) {
            float ss = 0.0f;
            for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
                uint32_t w[4];
                words(*reinterpret_cast<const uint4*>(xr + c * 8), w);
                ss = sum_squares(w, ss, up);
            }
            ss = lanes_sum<64>(ss);
            __syncthreads();                             // (the sums of a pass before have been read)
            if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
            __syncthreads();
            return (sums[0] + sums[1]) + (sums[2] + sums[3]);
        });
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = norm.rstd * norm.up;
    }
    uint32_t m = 0;
    for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
        float v[8];
        row_values<SRC>(a, xr, c, norm, v);
        m = max_bits(v, m);
    }
    const Int8Scale s = int8_scale(block_max(m, red));
    if (threadIdx.x == 0) a.scale[row] = s.s;
    for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
        float v[8];
        row_values<SRC>(a, xr, c, norm, v);
        *reinterpret_cast<uint2*>(a.q + row * a.cols + c * 8) = encode_int8(v, s);
    }
}

// ---------------------------------------------------------------- columns ---
// Largest magnitude patterns of the columns over P ranges of rows: part [P][cols].
// A block has 512 columns (a lane 8 of them), its four waves take the range's rows
// in turn, eight rows' loads in flight each. Bound by memory: a column's scale needs all
// of its rows, so that a transposed copy reads its tensor twice (8192x8960: 74 us for
// 367 MB, 5.0 TB/s).
constexpr int kColBlock = 512;
constexpr int64_t kFarElements = (int64_t)1 << 25;
struct ColMax {
    const uint16_t* x;
    int64_t rows, cols, ld;
    int P;
    uint16_t* part;
};
__device__ __forceinline__ void col_max(const ColMax& a, int bx, int by, uint4* red) {
    const uint16_t* const x = a.x;
    const int64_t rows = a.rows, cols = a.cols, ld = a.ld;
    const int P = a.P;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)bx * kColBlock + lane * 8;
    const int64_t r0 = rows * by / P, r1 = rows * (by + 1) / P;
    uint4 m = make_uint4(0, 0, 0, 0);
    if (col < cols) {
        constexpr int U = 8;
        for (int64_t r = r0 + wave; r < r1; r += 4 * U) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (past the range: the row that is there anyway)
                const int64_t ru = r + 4 * u < r1 ? r + 4 * u : r;
                v[u] = *reinterpret_cast<const uint4*>(x + ru * ld + col);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                m.x = pk_max_u16(m.x, mag2(v[u].x)); m.y = pk_max_u16(m.y, mag2(v[u].y));
                m.z = pk_max_u16(m.z, mag2(v[u].z)); m.w = pk_max_u16(m.w, mag2(v[u].w));
            }
        }
    }
    red[threadIdx.x] = m;
    __syncthreads();
    if (wave == 0 && col < cols) {
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const uint4 v = red[w * 64 + lane];
            m.x = pk_max_u16(m.x, v.x); m.y = pk_max_u16(m.y, v.y); m.z = pk_max_u16(m.z, v.z); m.w = pk_max_u16(m.w, v.w);
        }
        *reinterpret_cast<uint4*>(a.part + (int64_t)by * cols + col) = m;
    }
}

__global__ __launch_bounds__(kThreads) void col_max_kernel(ColMax a, int blocks_x) {
    __shared__ uint4 red[kThreads];
    col_max(a, (int)blockIdx.x % blocks_x, (int)blockIdx.x / blocks_x, red);
}

// Both in one launch: neither waits for the other, and a launch of its own costs a
// short tensor as much as the work. Of every `group` blocks the first are one range of
// rows' for the columns: of a large tensor both walk through the rows together, and the
// second finds them in the last-level cache (both copies of 8192x8960: 105 us with
// the columns' blocks first, 92 so; 16384x1536 33.6 and 36.6).
template <int TPR, int NC>
__global__ __launch_bounds__(kThreads) void rows_and_col_max_kernel(QuantInt8Args a, ColMax c, int blocks_x, Divisor group) {
    __shared__ uint4 red[kThreads];
    const int b = (int)blockIdx.x, g = (int)group.quotient((uint32_t)b), i = b - g * (int)group.d;
    if (g < c.P && i < blocks_x) col_max(c, i, g, red);
    else quant_rows<kRowBf16, TPR, NC>(a, b - min(c.P, g + 1) * blocks_x, reinterpret_cast<uint32_t*>(red), nullptr);
}

// The transposed copy by 128x128 tiles, each thread an 8x8 block. `a`: x, its rows
// rounded up to 16 (which are written; the rows behind `rows` read as zeros), ld, qT,
// scaleT.
struct ColScratch {
    __attribute__((aligned(16))) uint8_t lds[kTile * kTile];
    __attribute__((aligned(16))) float factor[kTile], before[kTile];
};
__device__ __forceinline__ void load_cols(const QuantArgs& a, int64_t rows, int64_t tr0, const Tile& t, v4i w[8]) {
    const int64_t vr = max((int64_t)0, min((int64_t)kTile, rows - tr0));
    const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(vr == 0 ? a.x : a.x + tr0 * a.ld, vr == 0 ? 0u : (uint32_t)(((vr - 1) * a.ld + a.cols) * 2));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, t.col_ok ? (uint32_t)(((t.rg * 8 + i) * a.ld + t.col) * 2) : kOOB, 0, 0);
}
// The scales of the tile's columns from 16 threads' maxima of each chunk of 8; 64
// threads make those of two columns each.
__device__ __forceinline__ void col_factors(const QuantArgs& a, const Tile& t, uint4 m, int64_t col0, bool write, ColScratch& s) {
    uint32_t* const maxima = reinterpret_cast<uint32_t*>(s.lds);      // [16 groups][64 words of two columns]
    *reinterpret_cast<uint4*>(maxima + t.rg * 64 + t.cc * 4) = m;
    __syncthreads();
    if (threadIdx.x < 64) {
        uint32_t v = maxima[threadIdx.x];
#pragma unroll
        for (int g = 1; g < 16; ++g) v = pk_max_u16(v, maxima[g * 64 + threadIdx.x]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j = 2 * threadIdx.x + e;
            const Int8Scale sc = int8_scale((e ? v >> 16 : v & 0xFFFFu) << 16);
            s.factor[j] = sc.r;
            s.before[j] = sc.pre;
            if (write && col0 + j < a.cols) a.scaleT[col0 + j] = sc.s;
        }
    }
    __syncthreads();
}
__device__ __forceinline__ void store_cols(const QuantArgs& a, const Tile& t, const v4i w[8], int64_t tr0, int64_t col0, int64_t ld_qT, ColScratch& s) {
    float r[8], pre[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { r[j] = s.factor[t.cc * 8 + j]; pre[j] = s.before[t.cc * 8 + j]; }
    uint2 c[8], ct[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x[4] = {(uint32_t)w[i].x, (uint32_t)w[i].y, (uint32_t)w[i].z, (uint32_t)w[i].w};
        float v[8];
        floats(x, v);
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = code_bits(v[j] * pre[j], r[j]);
        c[i] = make_uint2(pack_codes(b[0], b[1], b[2], b[3]), pack_codes(b[4], b[5], b[6], b[7]));
    }
    transpose8x8(c, ct);
    // LDS row r = column r of the tile, its 16-byte chunk h (rows 16 h ..) at h ^ ((r >> 3) & 7)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r8 = t.cc * 8 + j;
        *reinterpret_cast<uint2*>(s.lds + r8 * kTile + (((t.rg >> 1) ^ (r8 >> 3 & 7)) << 4) + ((t.rg & 1) << 3)) = ct[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTile * kTile / 16 / kThreads; ++i) {
        const int q = i * kThreads + threadIdx.x;
        const int r8 = q >> 3, h = q & 7;
        const uint4 v = *reinterpret_cast<const uint4*>(s.lds + r8 * kTile + ((h ^ (r8 >> 3 & 7)) << 4));
        const int64_t col = col0 + r8, row = tr0 + h * 16;
        if (col < a.cols && row < a.rows) *reinterpret_cast<uint4*>(a.qT + col * ld_qT + row) = v;
    }
}
__device__ __forceinline__ void max_mag(uint4& m, const uint4& v) {
    m.x = pk_max_u16(m.x, v.x); m.y = pk_max_u16(m.y, v.y); m.z = pk_max_u16(m.z, v.z); m.w = pk_max_u16(m.w, v.w);
}

// The second pass of a long tensor: a tile's values are on their way while the partial
// maxima of its columns are read. Bound by memory and its stores: 8187x1536 8.7 us,
// 8192x2048 10.1 (50 MB, 5.0 TB/s).
__global__ __launch_bounds__(kThreads) void quant_cols_int8_kernel(QuantArgs a, int64_t rows, int64_t ld_qT,
                                                                   const uint16_t* part, int P) {
    __shared__ ColScratch s;
    const Tile t = tile_coords(a.cols);
    const int64_t tr0 = (int64_t)(gridDim.y - 1 - blockIdx.y) * kTile;     // (the last rows first: the pass before has just read them)
    const int64_t col0 = (int64_t)blockIdx.x * kTile;
    v4i w[8];
    load_cols(a, rows, tr0, t, w);
    uint4 m = make_uint4(0, 0, 0, 0);
    if (t.col_ok) {
#pragma unroll 4
        for (int p = t.rg; p < P; p += 16) max_mag(m, *reinterpret_cast<const uint4*>(part + (int64_t)p * a.cols + t.col));
    }
    col_factors(a, t, m, col0, blockIdx.y == 0, s);
    store_cols(a, t, w, tr0, col0, ld_qT, s);
}

// A tensor of few rows: every block reads all of its columns' rows, the others' tiles
// for the maxima alone, and one launch makes both copies, the rows' blocks behind the
// columns'. Latency: 128x2048 4.1 us, by two launches 6.0; 333x2048 5.9 and 7.4.
__device__ __forceinline__ void quant_short_cols(const QuantArgs& a, int64_t rows, int64_t ld_qT, int64_t bx, int by, int tiles, ColScratch& s) {
    const Tile t = tile_coords(a.cols, bx, by);
    constexpr int U = 3;
    v4i own[8], w[U][8];
    load_cols(a, rows, (int64_t)by * kTile, t, own);
    uint4 m = make_uint4(0, 0, 0, 0);
    auto take = [&](const v4i v[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            max_mag(m, make_uint4(mag2((uint32_t)v[i].x), mag2((uint32_t)v[i].y), mag2((uint32_t)v[i].z), mag2((uint32_t)v[i].w)));
    };
    for (int k = 1; k < tiles; k += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (by, and on from there; past the last one: none)
            const int other = k + u >= tiles ? tiles : by + k + u - (by + k + u >= tiles ? tiles : 0);
            load_cols(a, rows, (int64_t)other * kTile, t, w[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) take(w[u]);
    }
    take(own);
    col_factors(a, t, m, bx * kTile, by == 0, s);
    store_cols(a, t, own, (int64_t)by * kTile, bx * kTile, ld_qT, s);
}
__global__ __launch_bounds__(kThreads) void quant_short_cols_int8_kernel(QuantArgs a, int64_t rows, int64_t ld_qT, int tiles) {
    __shared__ ColScratch s;
    quant_short_cols(a, rows, ld_qT, blockIdx.x / tiles, (int)blockIdx.x % tiles, tiles, s);
}
template <int TPR, int NC>
__global__ __launch_bounds__(kThreads) void quant_short_both_int8_kernel(QuantInt8Args a, QuantArgs t, int64_t ld_qT, int tiles, int col_blocks) {
    __shared__ ColScratch s;
    const int b = (int)blockIdx.x;
    if (b < col_blocks) quant_short_cols(t, a.rows, ld_qT, b / tiles, b % tiles, tiles, s);
    else quant_rows<kRowBf16, TPR, NC>(a, b - col_blocks, reinterpret_cast<uint32_t*>(s.lds), nullptr);
}

// Whether a tensor's columns are of few rows: the tiles are read as often as there are
// tiles of rows, a few at a time (700x2048, 576 reads: 7.5 us, by two launches 8.5; 333x
// 17920, 1260: 12.4 and 14.2; 512x17920, 2240: 18.6 and 18.0; 1000x2048, eight tiles of
// rows: 9.9 and 9.3).
bool short_cols(int64_t tiles_x, int64_t tiles_y) { return tiles_y <= 6 && tiles_x * tiles_y * tiles_y <= 1280; }

// Ranges of rows: their blocks fill the chip, and every tile of the second pass reads all
// of their maxima (both copies of 8192x2048: 64 ranges 25.9 us, 128 27.9), of which one
// block's columns have few (100000x64: 64 ranges 39.9 us, 256 32.5).
int col_ranges(int64_t rows, int64_t cols) {
    return (int)std::min<int64_t>(cols <= kColBlock ? 256 : 64, (rows + 31) / 32);
}

// ---------------------------------------------------------------- product of few rows ---
// Up to 64 rows of A: the time is that of reading B once (1x17920x1536 8.3 us, 3.3 TB/s;
// a small B is a launch and the latency of its loads, 1x2048x1536 3.8). A block has 16 columns
// and eight waves that take steps of 128 values of k in turn, straight from memory
// into registers (a lane 32 bytes of its row, four lanes a whole cache line), two
// steps' loads in flight; nothing but the rows of A that exist is read of A, from
// the caches. (16 columns, 8 waves, 2 steps: 1x2048x1536 3.9 us, 5x151936x1536 52.0;
// 32 columns 4.6 and 56.1, 4 waves 3.9 and 52.6, 4 steps 4.3 and 73.9, 16 waves with
// one step 4.1 and 68.7.) Per step and 16 x 16 tile two v_mfma_i32_16x16x64_i8 with B's rows as
// the first operand, so that lane l holds columns 4 (l >> 4) + 0..3 of row l & 15
// (A and B split k alike). The waves' integer sums meet in LDS.
typedef int v4i32 __attribute__((ext_vector_type(4)));

// Outputs [m, n .. n + 3]: the scaled sums, bias, residual, one rounding.
__device__ __forceinline__ void store_int8_outputs(const Int8Problem& p, int64_t m, int64_t n, v4i32 acc, float sa, const float sb[4]) {
    float4 v = make_float4(scaled_sum(acc.x, sa, sb[0]), scaled_sum(acc.y, sa, sb[1]), scaled_sum(acc.z, sa, sb[2]), scaled_sum(acc.w, sa, sb[3]));
    if (m >= p.M || n >= p.N) return;
    if (p.N % 4 == 0) {
        if (!p.f32) {
            if (p.bias || p.residual) add_epilogue4(v, p.bias, p.residual, p.ldr, m, n, 1.0f);
            *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p.D) + m * p.ldd + n) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
            return;
        }
        float4* d = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.D) + m * p.ldd + n);
        if (p.accumulate) {
            const float4 o = *d;
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        *d = v;
        return;
    }
    const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (n + e >= p.N) continue;
        if (p.f32) {
            float* d = reinterpret_cast<float*>(p.D) + m * p.ldd + n + e;
            *d = p.accumulate ? *d + w[e] : w[e];
        } else {
            reinterpret_cast<uint16_t*>(p.D)[m * p.ldd + n + e] = to_bf16(add_epilogue1(w[e], p.bias, p.residual, p.ldr, m, n + e, 1.0f));
        }
    }
}

constexpr int kRowsWaves = 8, kRowsSteps = 2;
template <int MT>
__global__ __launch_bounds__(kRowsWaves * 64) void int8_rows_kernel(Int8Problem p) {
    constexpr int WK = kRowsWaves, U = kRowsSteps;
    __shared__ v4i32 sums[WK * MT * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int K = (int)p.K;
    const int rows_n = (int)min((int64_t)16, p.N - n0);
    const __amdgpu_buffer_rsrc_t rb = buffer_rsrc(p.B + n0 * p.ldb, (uint32_t)((rows_n - 1) * p.ldb + K));
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(p.A, (uint32_t)((p.M - 1) * p.lda + K));
    const uint32_t ob = r < rows_n ? (uint32_t)(r * p.ldb) : kOOB;
    uint32_t oa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) oa[i] = i * 16 + r < p.M ? (uint32_t)((i * 16 + r) * p.lda) : kOOB;
    v4i32 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4i32{0, 0, 0, 0};
    for (int k0 = wave * 128; k0 < K; k0 += WK * 128 * U) {
        v4i32 b[U][2], a[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + u * (WK * 128) + q * 32 + h * 16;
                // (past the reduction's end, and of rows that are not there: zeros)
                const bool in = k < K;
                b[u][h] = __builtin_amdgcn_raw_buffer_load_b128(rb, in ? ob + k : kOOB, 0, 0);
#pragma unroll
                for (int i = 0; i < MT; ++i) a[u][i][h] = __builtin_amdgcn_raw_buffer_load_b128(ra, in ? oa[i] + k : kOOB, 0, 0);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[u][h], a[u][i][h], acc[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[(i * WK + wave) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += WK) {
        const int64_t m = i * 16 + r, n = n0 + q * 4;
        float sb[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sb[e] = n + e < p.N ? p.sb[n + e] : 0.0f;
        const float sa = m < p.M ? p.sa[m] : 0.0f;
        v4i32 v = sums[i * WK * 64 + lane];
#pragma unroll
        for (int w = 1; w < WK; ++w) v += sums[(i * WK + w) * 64 + lane];
        store_int8_outputs(p, m, n, v, sa, sb);
    }
}

// The same for at most 16 rows and a reduction of at most 2048, N % 4 == 0: A's
// values stay in registers (a wave has two steps of k at most) and a block goes
// through many groups of 16 columns, the next one's loads (and scales) in flight
// while one is summed. Two LDS buffers and one barrier a group; the waves take
// turns in storing. Bound by memory: 5x151936x1536 43.4 us, 5.4 TB/s of B.
constexpr int kStreamWaves = 8, kStreamK = kStreamWaves * 2 * 128;
__global__ __launch_bounds__(kStreamWaves * 64, 4) void int8_stream_kernel(Int8Problem p) {
    __shared__ v4i32 sums[2][kStreamWaves * 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, q = lane >> 4;
    const int K = (int)p.K;
    const int groups = (int)((p.N + 15) / 16);
    struct Set {
        v4i32 b[4];
        float4 s;
    };
    // the lane's places in a row of the operands (past the reduction's end: none)
    uint32_t ok[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int k = wave * 128 + (e >> 1) * (kStreamWaves * 128) + q * 32 + (e & 1) * 16;
        ok[e] = k < K ? (uint32_t)k : kOOB;
    }
    v4i32 a[4];
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(p.A, (uint32_t)((p.M - 1) * p.lda + K));
#pragma unroll
    for (int e = 0; e < 4; ++e)
        a[e] = __builtin_amdgcn_raw_buffer_load_b128(ra, r < p.M && ok[e] != kOOB ? (uint32_t)(r * p.lda) + ok[e] : kOOB, 0, 0);
    const float sa = r < p.M ? p.sa[r] : 0.0f;
    const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(p.sb, (uint32_t)(p.N * 4));
    auto load = [&](Set& t, int g) __attribute__((always_inline)) {
        const int64_t n0 = (int64_t)g * 16;
        const int rows = g < groups ? (int)min((int64_t)16, p.N - n0) : 0;
        const __amdgpu_buffer_rsrc_t rb = buffer_rsrc(rows > 0 ? p.B + n0 * p.ldb : p.B, rows > 0 ? (uint32_t)((rows - 1) * p.ldb + K) : 0u);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t.b[e] = __builtin_amdgcn_raw_buffer_load_b128(rb, r < rows && ok[e] != kOOB ? (uint32_t)(r * p.ldb) + ok[e] : kOOB, 0, 0);
        t.s = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(rs, g < groups ? (uint32_t)((g * 16 + q * 4) * 4) : kOOB, 0, 0));
    };
    auto take = [&](const Set& t, int g, int turn) __attribute__((always_inline)) {
        v4i32 acc = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.b[e], a[e], acc, 0, 0, 0);
        v4i32* const buf = sums[turn & 1];
        buf[wave * 64 + lane] = acc;
        __syncthreads();
        if (wave != (turn & (kStreamWaves - 1))) return;
        v4i32 v = buf[lane];
#pragma unroll
        for (int w = 1; w < kStreamWaves; ++w) v += buf[w * 64 + lane];
        const float sb[4] = {t.s.x, t.s.y, t.s.z, t.s.w};
        store_int8_outputs(p, r, (int64_t)g * 16 + q * 4, v, sa, sb);
    };
    Set t0, t1;
    int g = blockIdx.x;
    const int step = gridDim.x;
    load(t0, g);
    for (int turn = 0; g < groups; turn += 2) {
        load(t1, g + step);
        take(t0, g, turn);
        g += step;
        if (g >= groups) break;
        load(t0, g + step);
        take(t1, g, turn + 1);
        g += step;
    }
}

// f(Int<threads per row>, Int<chunks a thread>) for rows of `cols` values: a wave per
// row where there are rows enough to fill the chip with four a block (short rows 16
// lanes: 100000x64 21.7 -> 7.7 us), else a block; in as few chunks a thread as hold the
// row. False: the row is too long.
template <int N> using Int = std::integral_constant<int, N>;
int64_t row_blocks(int64_t rows, int tpr) { return (rows + kThreads / tpr - 1) / (kThreads / tpr); }
template <typename F>
bool fit_rows(int64_t rows, int64_t cols, F&& f) {
    const int64_t cpr = cols / 8;
    auto fit = [&](auto tpr, auto... nc) {
        bool done = false;
        auto one = [&](auto n) {
            if (!done && cpr <= decltype(tpr)::value * decltype(n)::value) {
                f(tpr, n);
                done = true;
            }
        };
        (one(nc), ...);
        return done;
    };
    return (rows >= 4096 && fit(Int<16>{}, Int<1>{})) || (rows >= 1024 && fit(Int<64>{}, Int<1>{}, Int<2>{}, Int<4>{})) ||
           fit(Int<256>{}, Int<1>{}, Int<2>{}, Int<3>{}, Int<5>{}, Int<8>{}, Int<12>{});
}

template <int SRC>
void launch_rows(const QuantInt8Args& a, hipStream_t stream) {
    const bool fits = fit_rows(a.rows, a.cols, [&](auto tpr, auto nc) {
        constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
        quant_rows_int8_kernel<SRC, TPR, NC><<<(unsigned)row_blocks(a.rows, TPR), kThreads, 0, stream>>>(a);
    });
    if (!fits) quant_long_rows_int8_kernel<SRC><<<(unsigned)a.rows, kThreads, 0, stream>>>(a);
}

}  // namespace

void launch_quantize_int8(const QuantInt8Args& a, hipStream_t stream) {
    if (a.swiglu) launch_rows<kRowSwiglu>(a, stream);
    else if (a.gamma && a.eps < kLeastMean) launch_rows<kRowNormSmall>(a, stream);
    else if (a.gamma) launch_rows<kRowNorm>(a, stream);
    else launch_rows<kRowBf16>(a, stream);
}

void launch_quantize_int8_two(const QuantInt8Args& a, const QuantInt8Args& b, hipStream_t stream) {
    const bool together = fit_rows(a.rows + b.rows, a.cols, [&](auto tpr, auto nc) {
        constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
        const int64_t blocks = row_blocks(a.rows, TPR);
        quant_two_rows_int8_kernel<TPR, NC><<<(unsigned)(blocks + row_blocks(b.rows, TPR)), kThreads, 0, stream>>>(a, b, (int)blocks);
    });
    if (together) return;
    launch_quantize_int8(a, stream);
    launch_quantize_int8(b, stream);
}

size_t quant_int8_ws_bytes(int64_t rows, int64_t cols) { return (size_t)col_ranges(rows, cols) * cols * 2; }

void launch_quantize_int8_both(const QuantInt8Args& a, int8_t* qT, int64_t ld_qT, float* scaleT, void* ws, hipStream_t stream) {
    QuantArgs t{};
    t.x = a.x; t.rows = (a.rows + 15) / 16 * 16; t.cols = a.cols; t.ld = a.ld;
    t.qT = reinterpret_cast<uint8_t*>(qT); t.scaleT = scaleT;
    const int64_t tiles_x = (a.cols + kTile - 1) / kTile, tiles_y = (a.rows + kTile - 1) / kTile;
    if (short_cols(tiles_x, tiles_y)) {
        const int tiles = (int)tiles_y, col_blocks = (int)(tiles_x * tiles_y);
        const bool together = a.q && fit_rows(a.rows, a.cols, [&](auto tpr, auto nc) {
            constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
            const unsigned grid = (unsigned)(col_blocks + row_blocks(a.rows, TPR));
            quant_short_both_int8_kernel<TPR, NC><<<grid, kThreads, 0, stream>>>(a, t, ld_qT, tiles, col_blocks);
        });
        if (together) return;
        if (a.q) launch_quantize_int8(a, stream);
        quant_short_cols_int8_kernel<<<(unsigned)col_blocks, kThreads, 0, stream>>>(t, a.rows, ld_qT, tiles);
        return;
    }
    const ColMax c{a.x, a.rows, a.cols, a.ld, col_ranges(a.rows, a.cols), reinterpret_cast<uint16_t*>(ws)};
    const int blocks_x = (int)((a.cols + kColBlock - 1) / kColBlock), col_blocks = blocks_x * c.P;
    const bool together = a.q && fit_rows(a.rows, a.cols, [&](auto tpr, auto nc) {
        constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
        const unsigned grid = (unsigned)(col_blocks + row_blocks(a.rows, TPR));
        // (of a small tensor the columns' blocks first, as the longer ones)
        const unsigned group = a.rows * a.cols < kFarElements ? (unsigned)blocks_x : grid / (unsigned)c.P;
        rows_and_col_max_kernel<TPR, NC><<<grid, kThreads, 0, stream>>>(a, c, blocks_x, Divisor::of(group));
    });
    if (!together) {
        if (a.q) launch_quantize_int8(a, stream);
        col_max_kernel<<<(unsigned)col_blocks, kThreads, 0, stream>>>(c, blocks_x);
    }
    const dim3 grid((unsigned)tiles_x, (unsigned)tiles_y);
    quant_cols_int8_kernel<<<grid, kThreads, 0, stream>>>(t, a.rows, ld_qT, c.part, c.P);
}

// Whether a product takes the kernels of few rows: those read A's fragments from
// the caches for every 16 columns, which from 17 rows on costs more than the tiled
// kernel's LDS unless the whole product is small (in a graph, weights not in a
// cache: 1x2048x1536 3.8 us against 6.9 tiled, 1x1536x8960 8.3 against 11.0, 5x151936x
// 1536 48.1 against 60.4; 20x2048x1536 4.7 against 6.7, 64x2048x1536 6.7 against 7.1,
// but 20x17920x1536 13.3 against 12.4 and 64x151936x1536 164 against 65).
static bool few_rows(int64_t M, int64_t N, int64_t K) { return M <= 16 || (M <= 64 && N * K <= (int64_t)1 << 22); }

// Blocks of the streaming kernel: two a CU, as many as its registers allow (5x151936x
// 1536: 512 blocks 48.1 us, 768 49.2, 1536 50.1; the other kernel 52.0). Where a
// block would have few groups, the other kernel's many blocks are faster (1x17920x1536
// 8.3 us against 8.6).
constexpr int kStreamBlocks = 512;
constexpr int64_t kStreamColumns = 32768;

template <int MT>
static void launch_few(const Int8Problem& p, hipStream_t stream) {
    int8_rows_kernel<MT><<<(unsigned)((p.N + 15) / 16), kRowsWaves * 64, 0, stream>>>(p);
}

size_t int8_gemm_ws_bytes(int64_t M, int64_t N, int64_t K) {
    return few_rows(M, N, K) ? 0 : gemm_int8_workspace_bytes(M, N, K);
}

void launch_int8_gemm(const Int8Problem& p, void* ws, hipStream_t stream) {
    if (few_rows(p.M, p.N, p.K)) {
        if (p.M <= 16 && p.K <= kStreamK && p.N % 4 == 0 && p.N >= kStreamColumns)
            int8_stream_kernel<<<kStreamBlocks, kStreamWaves * 64, 0, stream>>>(p);
        else if (p.M <= 16) launch_few<1>(p, stream);
        else if (p.M <= 32) launch_few<2>(p, stream);
        else launch_few<4>(p, stream);
        return;
    }
    GemmProblem g{};
    g.M = p.M; g.N = p.N; g.K = p.K;
    g.A = reinterpret_cast<const uint8_t*>(p.A); g.lda = p.lda; g.fa = kInt8; g.sa_mode = kSNone; g.sa = p.sa;
    g.B = reinterpret_cast<const uint8_t*>(p.B); g.ldb = p.ldb; g.fb = kInt8; g.sb_mode = kSNone; g.sb = p.sb;
    g.D = p.D; g.ldd = p.ldd; g.accumulate = p.accumulate;
    g.out = p.f32 ? kOutF32 : p.bias || p.residual ? kOutBF16Epi : kOutBF16;
    g.bias = p.bias; g.residual = p.residual; g.ldr = p.ldr;
    g.nt_f32 = 1;       // (as the FP8 product: a dW or logits, next read by another kernel)
    launch_gemm(g, ws, stream);
}

}  // namespace puro
