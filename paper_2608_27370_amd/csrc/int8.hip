// 8-bit integer linear layers for gfx950: the quantisation of rows (tokens, output
// channels) and of columns (transposed copies) to int8, and the product of int8
// codes with a scale for each row of either operand.

#include "quant_tile.h"

namespace puro {

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
// One block per row: the row's values are formed twice, for its largest
// magnitude and for the codes.
enum : int { kRowBf16 = 0, kRowNorm = 1, kRowSwiglu = 2 };

__device__ __forceinline__ void words(const uint4& v, uint32_t w[4]) { w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }

template <int SRC>
__device__ __forceinline__ void row_values(const QuantInt8Args& a, const uint16_t* xr, int64_t c, float rstd, float v[8]) {
    uint32_t w[4];
    words(*reinterpret_cast<const uint4*>(xr + c * 8), w);
    if constexpr (SRC == kRowBf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(w[i]); v[2 * i + 1] = bf16hi(w[i]); }
    } else if constexpr (SRC == kRowNorm) {
        uint32_t g[4];
        words(*reinterpret_cast<const uint4*>(a.gamma + c * 8), g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = bf16lo(w[i]) * rstd * bf16lo(g[i]);
            v[2 * i + 1] = bf16hi(w[i]) * rstd * bf16hi(g[i]);
        }
    } else {
        uint32_t u[4];
        words(*reinterpret_cast<const uint4*>(xr + a.cols + c * 8), u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = swiglu1<false>(bf16lo(w[i]), bf16lo(u[i]));
            v[2 * i + 1] = swiglu1<false>(bf16hi(w[i]), bf16hi(u[i]));
        }
    }
}

template <int SRC>
__global__ __launch_bounds__(kThreads) void quant_rows_int8_kernel(QuantInt8Args a) {
    __shared__ uint32_t red[4];
    __shared__ float sums[4];
    const int64_t row = blockIdx.x, cpr = a.cols / 8;
    const uint16_t* xr = a.x + row * a.ld;
    float rstd = 1.0f;
    if constexpr (SRC == kRowNorm) {
        float ss = 0.0f;
        for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
            uint32_t w[4];
            words(*reinterpret_cast<const uint4*>(xr + c * 8), w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ss = fmaf(bf16lo(w[i]), bf16lo(w[i]), ss);
                ss = fmaf(bf16hi(w[i]), bf16hi(w[i]), ss);
            }
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
        __syncthreads();
        rstd = 1.0f / sqrtf(((sums[0] + sums[1]) + (sums[2] + sums[3])) / (float)a.cols + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    }
    uint32_t m = 0;
    for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
        float v[8];
        row_values<SRC>(a, xr, c, rstd, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    const Int8Scale s = int8_scale(block_max(m, red));
    if (threadIdx.x == 0) a.scale[row] = s.s;
    for (int64_t c = threadIdx.x; c < cpr; c += kThreads) {
        float v[8];
        row_values<SRC>(a, xr, c, rstd, v);
        *reinterpret_cast<uint2*>(a.q + row * a.cols + c * 8) = encode_int8(v, s);
    }
}

// ---------------------------------------------------------------- columns ---
// Largest magnitude patterns of the columns over P ranges of rows: part [P][cols].
__global__ __launch_bounds__(kThreads) void col_max_kernel(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, int P,
                                                           uint16_t* part) {
    const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (c >= cols / 8) return;
    const int64_t r0 = rows * blockIdx.y / P, r1 = rows * (blockIdx.y + 1) / P;
    uint32_t m[4] = {0u, 0u, 0u, 0u};
    for (int64_t r = r0; r < r1; ++r) {
        uint32_t w[4];
        words(*reinterpret_cast<const uint4*>(x + r * ld + c * 8), w);
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = pk_max_u16(m[i], mag2(w[i]));
    }
    *reinterpret_cast<uint4*>(part + (int64_t)blockIdx.y * cols + c * 8) = make_uint4(m[0], m[1], m[2], m[3]);
}

// The transposed copy by 128x128 tiles: each thread an 8x8 block, the columns'
// scales from the partial maxima. `a`: x, its rows rounded up to 16 (which are
// written; the rows behind `rows` read as zeros), ld, qT, scaleT.
__global__ __launch_bounds__(kThreads) void quant_cols_int8_kernel(QuantArgs a, int64_t rows, int64_t ld_qT,
                                                                   const uint16_t* part, int P) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kTile * kTile];
    const Tile t = tile_coords(a.cols);
    const int64_t tr0 = (int64_t)blockIdx.y * kTile;
    const int64_t vr = max((int64_t)0, min((int64_t)kTile, rows - tr0));
    const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(vr == 0 ? a.x : a.x + tr0 * a.ld, vr == 0 ? 0u : (uint32_t)(((vr - 1) * a.ld + a.cols) * 2));
    v4i w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, t.col_ok ? (uint32_t)(((t.rg * 8 + i) * a.ld + t.col) * 2) : kOOB, 0, 0);
    uint32_t m[4] = {0u, 0u, 0u, 0u};
    if (t.col_ok)
        for (int p = 0; p < P; ++p) {
            uint32_t v[4];
            words(*reinterpret_cast<const uint4*>(part + (int64_t)p * a.cols + t.col), v);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = pk_max_u16(m[i], v[i]);
        }
    Int8Scale s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s[j] = int8_scale((j & 1 ? m[j / 2] >> 16 : m[j / 2] & 0xFFFFu) << 16);
        if (t.rg == 0 && blockIdx.y == 0 && t.col_ok) a.scaleT[t.col + j] = s[j].s;
    }
    uint2 c[8], ct[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t x[4] = {(uint32_t)w[i].x, (uint32_t)w[i].y, (uint32_t)w[i].z, (uint32_t)w[i].w};
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = code_bits((j & 1 ? bf16hi(x[j / 2]) : bf16lo(x[j / 2])) * s[j].pre, s[j].r);
        c[i] = make_uint2(pack_codes(b[0], b[1], b[2], b[3]), pack_codes(b[4], b[5], b[6], b[7]));
    }
    transpose8x8(c, ct);
    // LDS row r = column r of the tile, its 16-byte chunk h (rows 16 h ..) at h ^ ((r >> 3) & 7)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = t.cc * 8 + j;
        *reinterpret_cast<uint2*>(lds + r * kTile + (((t.rg >> 1) ^ (r >> 3 & 7)) << 4) + ((t.rg & 1) << 3)) = ct[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTile * kTile / 16 / kThreads; ++i) {
        const int q = i * kThreads + threadIdx.x;
        const int r = q >> 3, h = q & 7;
        const uint4 v = *reinterpret_cast<const uint4*>(lds + r * kTile + ((h ^ (r >> 3 & 7)) << 4));
        const int64_t col = (int64_t)blockIdx.x * kTile + r, row = tr0 + h * 16;
        if (col < a.cols && row < a.rows) *reinterpret_cast<uint4*>(a.qT + col * ld_qT + row) = v;
    }
}

int col_ranges(int64_t rows) { return (int)std::min<int64_t>(64, (rows + 31) / 32); }

// ---------------------------------------------------------------- product ---
// One wave per 16 x 16 tile of D, operands straight from memory: per 64 values
// of k one v_mfma_i32_16x16x64_i8, B's rows as its first operand, so that lane l
// holds columns 4 (l >> 4) + 0..3 of row l & 15.
typedef int v4i32 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(kThreads) void int8_gemm_kernel(Int8Problem p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tiles_n = (p.N + 15) / 16, tiles = tiles_n * ((p.M + 15) / 16);
    for (int64_t tile = (int64_t)blockIdx.x * 4 + wave; tile < tiles; tile += (int64_t)gridDim.x * 4) {
        const int64_t m0 = tile / tiles_n * 16, n0 = tile % tiles_n * 16;
        const int64_t m = m0 + (lane & 15), nr = n0 + (lane & 15);
        v4i32 acc = {0, 0, 0, 0};
        for (int64_t k = (lane >> 4) * 16; k < (p.K + 63) / 64 * 64; k += 64) {
            v4i32 x = {0, 0, 0, 0}, w = {0, 0, 0, 0};
            if (k < p.K && m < p.M) x = *reinterpret_cast<const v4i32*>(p.A + m * p.lda + k);
            if (k < p.K && nr < p.N) w = *reinterpret_cast<const v4i32*>(p.B + nr * p.ldb + k);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
        }
        if (m >= p.M) continue;
        const float sa = p.sa[m];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t n = n0 + 4 * (lane >> 4) + e;
            if (n >= p.N) continue;
            float v = (float)acc[e] * sa * p.sb[n];
            if (p.bias) v += __uint_as_float((uint32_t)p.bias[n] << 16);
            if (p.residual) v += __uint_as_float((uint32_t)p.residual[m * p.ldr + n] << 16);
            if (p.f32) {
                float* d = reinterpret_cast<float*>(p.D) + m * p.ldd + n;
                *d = p.accumulate ? *d + v : v;
            } else {
                reinterpret_cast<uint16_t*>(p.D)[m * p.ldd + n] = to_bf16(v);
            }
        }
    }
}

}  // namespace

void launch_quantize_int8(const QuantInt8Args& a, hipStream_t stream) {
    const int grid = (int)a.rows;
    if (a.swiglu) quant_rows_int8_kernel<kRowSwiglu><<<grid, kThreads, 0, stream>>>(a);
    else if (a.gamma) quant_rows_int8_kernel<kRowNorm><<<grid, kThreads, 0, stream>>>(a);
    else quant_rows_int8_kernel<kRowBf16><<<grid, kThreads, 0, stream>>>(a);
}

size_t quant_int8_ws_bytes(int64_t rows, int64_t cols) { return (size_t)col_ranges(rows) * cols * 2; }

void launch_quantize_int8_t(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, int8_t* qT, int64_t ld_qT,
                            float* scaleT, void* ws, hipStream_t stream) {
    const int P = col_ranges(rows);
    uint16_t* part = reinterpret_cast<uint16_t*>(ws);
    col_max_kernel<<<dim3((unsigned)((cols / 8 + kThreads - 1) / kThreads), P), kThreads, 0, stream>>>(x, rows, cols, ld, P, part);
    QuantArgs a{};
    a.x = x; a.rows = (rows + 15) / 16 * 16; a.cols = cols; a.ld = ld;
    a.qT = reinterpret_cast<uint8_t*>(qT); a.scaleT = scaleT;
    const dim3 grid((unsigned)((cols + kTile - 1) / kTile), (unsigned)((rows + kTile - 1) / kTile));
    quant_cols_int8_kernel<<<grid, kThreads, 0, stream>>>(a, rows, ld_qT, part, P);
}

size_t int8_gemm_ws_bytes(int64_t M, int64_t N, int64_t K) { return gemm_workspace_bytes(M, N, K, kOutBF16); }

void launch_int8_gemm(const Int8Problem& p, void* ws, hipStream_t stream) {
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
