// The language-model head with the divergence from a teacher's top logits as
// its loss (gfx950), in BF16 as the paper runs this layer (Appendix C).
//
// For hidden states X [M, K], the output embedding W [V, K], a temperature tau
// and, per row, k entries of a teacher (token ids and logits or weights):
//
//   z = X W^T, a = z / tau, lse_m = log sum_v exp a_mv
//   q_m = softmax over the row's entries of t / tau, or the weights given
//   loss_m = sum_j q_mj (log q_mj - a_{m, id_mj} + lse_m)
//   dz_mv = (dloss_m g / tau) (Q_m exp(a_mv - lse_m) - sum_{j: id_mj = v} q_mj),
//   Q_m = sum_j q_mj;  dX = dz W, dW = dz^T X
//
// As with the cross-entropy (lm_head.hip) the logits never reach memory: the
// forward's GEMM reduces them to (max, sum exp) per row and 128 columns, the
// backward recomputes them (by chunks of the vocabulary, where there are very
// many), its GEMM writing the dense part of dz and of its transposed copy (a
// transpose of its own moved the 5 GB of M 8192, V 151936 in 0.97 ms). What
// differs from a one-hot target is sparse: the k logits of a row that the loss
// needs are k dot products, and the gradient at those places is written over
// the dense part's, from the same formula with the entry's q, in one rounding.
// dz is rounded to BF16 because it is an operand of two BF16 products; a row's
// roundings are independent, and dX and dW err by 2^-9 of their size in the mean.
//
// Bound by the matrix products. M 8192, V 151936, K 1536: backward 9.7 ms, of
// which logits and dz 3.9 (3.82 TFLOP and 5 GB of stores), dX 2.78, dW 2.80
// (1.37 PFLOP/s each) and W's transposed copy 0.17; forward at M 4096 1.6 ms, the
// GEMM 1.52 to 1.58 (1.2 PFLOP/s) and the rows 0.11.

#include <math.h>

#include <algorithm>

#include "device_common.h"
#include "kernels.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// (element passes over matrices of any size: a launch holds fewer than 2^32
// threads, so from kMaxBlocks blocks on each takes several pieces)
constexpr int64_t kMaxBlocks = 1 << 20;

__global__ __launch_bounds__(kThreads) void f32_to_bf16_kernel(const float* __restrict__ src, uint16_t* __restrict__ dst,
                                                               int64_t n4) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n4; i += kMaxBlocks * kThreads) {
        const float4 v = reinterpret_cast<const float4*>(src)[i];
        reinterpret_cast<uint2*>(dst)[i] = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
}

__global__ __launch_bounds__(kThreads) void zero_kernel(uint16_t* __restrict__ dst, int64_t n8) {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n8; i += kMaxBlocks * kThreads)
        reinterpret_cast<uint4*>(dst)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// z_top[j] = x . W[id_j] of a row's k entries, 0 for one that does not count,
// by the four waves of a block: kIds entries at a time each, its lanes 16-byte
// pieces of the K values (K % 8 == 0), summed in binary32 and across the wave.
// (64 entries of 4096 rows of 1536: 805 MB of W's rows at 7.7 TB/s, from the
// caches as far as tokens recur; in the GEMM's epilogue each lane would pick
// them from its 64 sums by as many comparisons per entry.)
constexpr int kIds = 4;
__device__ __forceinline__ void top_logits(const uint16_t* __restrict__ x, const uint16_t* __restrict__ W,
                                           const int32_t* __restrict__ ids, int64_t V, int64_t K, int k, float* sz,
                                           float* __restrict__ z_top) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int j0 = wave * kIds; j0 < k; j0 += kIds * 4) {
        const uint16_t* w[kIds];
        float s[kIds];
        bool in[kIds];
#pragma unroll
        for (int u = 0; u < kIds; ++u) {
            const int id = j0 + u < k ? ids[j0 + u] : -1;
            // (an entry that does not count reads row 0 and is dropped below)
            in[u] = (unsigned)id < (uint64_t)V;
            w[u] = W + (in[u] ? id : 0) * K;
            s[u] = 0.0f;
        }
        for (int64_t c = lane * 8; c < K; c += 512) {
            const uint4 xv = *reinterpret_cast<const uint4*>(x + c);
            const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
            for (int u = 0; u < kIds; ++u) {
                const uint4 wv = *reinterpret_cast<const uint4*>(w[u] + c);
                const uint32_t ww[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[u] = fmaf(bf16lo(xw[e]), bf16lo(ww[e]), s[u]);
                    s[u] = fmaf(bf16hi(xw[e]), bf16hi(ww[e]), s[u]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kIds; ++u) {
            const float v = wave_sum(s[u]);
            if (lane == 0 && j0 + u < k) sz[j0 + u] = z_top[j0 + u] = in[u] ? v : 0.0f;
        }
    }
}

// The teacher's weights of a row: q(j) of entry j (0 where it does not count),
// and log q(j) where q(j) > 0. A wave per row.
struct Teacher {
    const int32_t* ids;
    const float* t;
    int64_t V;
    int k, probs;
    float inv_tau;
    float top, log_sum;        // of t / tau over the entries that count; top -inf: none does
    __device__ __forceinline__ bool counts(int j) const { return (unsigned)ids[j] < (uint64_t)V; }
    __device__ __forceinline__ void begin(int lane) {
        if (probs) return;
        top = -kInf;
        for (int j = lane; j < k; j += 64)
            if (counts(j)) top = fmaxf(top, t[j]);
        top = wave_max(top);
        float s = 0.0f;
        if (top > -kInf)
            for (int j = lane; j < k; j += 64)
                if (counts(j)) s += exp_f32((t[j] - top) * inv_tau);
        s = wave_sum(s);
        // (NaN entries: fmaxf leaves them out of top, exp brings them into the sum)
        log_sum = logf(s);
        if (!(top > -kInf)) {
            bool nan = false;
            for (int j = lane; j < k; j += 64) nan = nan || (counts(j) && t[j] != t[j]);
            if (__builtin_amdgcn_ballot_w64(nan)) log_sum = top = __builtin_nanf("");
        }
    }
    __device__ __forceinline__ float log_q(int j) const { return probs ? logf(t[j]) : (t[j] - top) * inv_tau - log_sum; }
    __device__ __forceinline__ float q(int j) const {
        if (!counts(j)) return 0.0f;
        if (probs) return t[j];
        if (top == -kInf) return 0.0f;
        return exp_f32(log_q(j));
    }
};

// lse, z_top and loss of a row, from its blocks' (max, sum exp(a - max)) and
// its entries: a block per row. The pairs are read once, kHold of a thread's stay in
// registers between the maximum and the sum (as many as a vocabulary of 262144
// has; M 4096, V 151936: 13.7 us, a wave per row that read them twice 29.7), their
// loads in flight during the entries' dot products.
constexpr int kHold = 8;
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(const float2* __restrict__ stats, int64_t ld, int nblk,
                                                                const uint16_t* __restrict__ X,
                                                                const uint16_t* __restrict__ W, int64_t K, Teacher tch,
                                                                float* __restrict__ z_top, float* __restrict__ lse,
                                                                float* __restrict__ loss) {
    __shared__ float red[8];
    __shared__ float sz[kDistillMaxTop];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = blockIdx.x;
    const float2* const st = stats + m * ld;
    float2 v[kHold];
    float mx = -kInf;
#pragma unroll
    for (int u = 0; u < kHold; ++u) {
        const int b = (int)threadIdx.x + kThreads * u;
        v[u] = b < nblk ? st[b] : make_float2(-kInf, 0.0f);
    }
    tch.ids += m * tch.k;
    tch.t += m * tch.k;
    top_logits(X + m * K, W, tch.ids, tch.V, K, tch.k, sz, z_top + m * tch.k);
#pragma unroll
    for (int u = 0; u < kHold; ++u) mx = fmaxf(mx, v[u].x);
    for (int b = (int)threadIdx.x + kThreads * kHold; b < nblk; b += kThreads) mx = fmaxf(mx, st[b].x);
    mx = wave_max(mx);
    if (lane == 0) red[wave] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < kHold; ++u)
        if (v[u].y != 0.0f) s += v[u].y * exp_f32(v[u].x - mx);   // NaN sums propagate
    for (int b = (int)threadIdx.x + kThreads * kHold; b < nblk; b += kThreads) {
        const float2 w = st[b];
        if (w.y != 0.0f) s += w.y * exp_f32(w.x - mx);
    }
    s = wave_sum(s);
    if (lane == 0) red[4 + wave] = s;
    __syncthreads();
    if (wave > 0) return;
    const float l = mx + logf((red[4] + red[5]) + (red[6] + red[7]));
    tch.begin(lane);
    float sum = 0.0f;
    for (int j = lane; j < tch.k; j += 64) {
        const float q = tch.q(j);
        if (q != 0.0f) sum += q * (tch.log_q(j) - (sz[j] * tch.inv_tau - l));
    }
    sum = wave_sum(sum);
    if (lane == 0) {
        lse[m] = l;
        loss[m] = sum;
    }
}

// What the backward's chunks need of a row (one wave): coef = dloss g / tau Q,
// the factor of the dense part, and for each entry the whole gradient at its
// place, coef exp(a - lse) - dloss g / tau * (the sum of q over all entries of
// that id): entries of the same id have the same value, whichever is written.
// A row whose coef is 0 (no entries, dloss 0) has no gradient: its hidden state,
// and with it lse, may be anything, and so may the dloss of one without entries.
__global__ __launch_bounds__(64) void distill_coef_kernel(Teacher tch, const float* __restrict__ z_top,
                                                          const float* __restrict__ lse, const float* __restrict__ dloss,
                                                          float g_tau, float* __restrict__ coef, float* __restrict__ val) {
    extern __shared__ float sq[];                       // q[k], then ids[k]
    int32_t* const sid = reinterpret_cast<int32_t*>(sq + tch.k);
    const int lane = threadIdx.x;
    const int64_t m = blockIdx.x;
    tch.ids += m * tch.k;
    tch.t += m * tch.k;
    tch.begin(lane);
    float Q = 0.0f;
    for (int j = lane; j < tch.k; j += 64) {
        const float q = tch.q(j);
        Q += q;
        sq[j] = q;
        sid[j] = tch.ids[j];
    }
    Q = wave_sum(Q);
    __syncthreads();
    const float dl = (dloss ? dloss[m] : 1.0f) * g_tau;
    const float c = Q == 0.0f ? 0.0f : dl * Q, l = lse[m];      // (dl infinite or NaN in a padding token's row)
    if (lane == 0) coef[m] = c;
    for (int j = lane; j < tch.k; j += 64) {
        const int32_t id = sid[j];
        float qs = 0.0f;
        for (int i = 0; i < tch.k; ++i) qs += sid[i] == id ? sq[i] : 0.0f;
        val[m * tch.k + j] = c == 0.0f ? 0.0f : c * exp_f32(z_top[m * tch.k + j] * tch.inv_tau - l) - dl * qs;
    }
}

// The entries of vocabulary columns [c0, c0 + n) into dz [rows][ld] and, where
// there is one, its transposed copy [n][ldt]; and zeros into dz's columns from n
// up to ld (the last chunk's, past the vocabulary).
__global__ __launch_bounds__(kThreads) void distill_entries_kernel(const int32_t* __restrict__ ids, const float* __restrict__ val,
                                                                   int64_t count, int k, int64_t c0, int64_t n,
                                                                   uint16_t* __restrict__ dz, int64_t rows, int64_t ld,
                                                                   uint16_t* __restrict__ dzt, int64_t ldt) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= count) {
        const int64_t j = i - count, width = ld - n;
        if (j < rows * width) dz[j / width * ld + n + j % width] = 0;
        return;
    }
    const int64_t c = (int64_t)ids[i] - c0, m = i / k;
    if (c < 0 || c >= n) return;
    const uint16_t v = to_bf16(val[i]);
    dz[m * ld + c] = v;
    if (dzt) dzt[c * ldt + m] = v;
}

constexpr size_t kAl = 256;
size_t al(size_t v) { return (v + kAl - 1) / kAl * kAl; }
int64_t pad128(int64_t v) { return (v + 127) / 128 * 128; }

// Vocabulary columns per chunk of the backward: as few chunks as keep one copy
// of a chunk's dz within 2.5 GiB (288 GB of memory make a chunk of the whole
// vocabulary the usual case), of even width, a multiple of the 256-wide tiles
// (256 columns of the most rows, 2^21, are 1 GiB).
// Few columns at a time leave the grids of few rows half empty and add every
// chunk's dX to binary32 sums; that a chunk of 8192 columns stays in the
// last-level cache gains less. Backward of V 151936, K 1536 at 8192 columns, at
// 32768 and at all: M 300 1842, 1106, 1029 us; M 2000 3646, 2953, 2823; M 4096
// 6068, 5512, 5308; M 8192 11023, 10438 (30464), 10263.
constexpr int64_t kDzBytes = (int64_t)5 << 29;
int64_t chunk_of(int64_t Mp, int64_t Vp) {
    const int64_t most = kDzBytes / (2 * Mp) / 256 * 256, chunks = (Vp + most - 1) / most;
    return std::min(((Vp + chunks - 1) / chunks + 255) / 256 * 256, Vp);
}

struct Layout {
    size_t stats;                                                  // forward
    size_t coef, val, xt, wt, dz, dzt, dxacc, gemm;                // backward
    size_t total;
};

Layout layout(int64_t M, int64_t V, int64_t K, int64_t k, bool bwd) {
    size_t used = 0;
    auto take = [&](size_t b) { const size_t at = used; used = al(used + b); return at; };
    Layout l{};
    const int64_t Mp = pad128(M), Vp = pad128(V), Vc = chunk_of(Mp, Vp);
    if (!bwd) {
        l.stats = take((size_t)M * (Vp / 128) * sizeof(float2));
    } else {
        l.coef = take((size_t)Mp * sizeof(float));
        l.val = take((size_t)M * k * sizeof(float));
        l.xt = take((size_t)Mp * K * 2);
        l.wt = take((size_t)Vp * K * 2);
        l.dz = take((size_t)Mp * Vc * 2);
        l.dzt = take((size_t)Mp * Vc * 2);
        if (Vc < V) l.dxacc = take((size_t)M * K * 4);
        // the split-K partials of the dX and dW GEMMs, for a full chunk and for the last one
        size_t g = 0;
        const int64_t last = V - (V - 1) / Vc * Vc;
        for (const int64_t n : {std::min(V, Vc), last}) {
            g = std::max(g, gemm_long_k_workspace_bytes(M, K, pad128(n) * 2, kOutF32));
            g = std::max(g, gemm_workspace_bytes(n, K, Mp * 2, kOutF32));
        }
        l.gemm = take(g);
    }
    l.total = used;
    return l;
}

Teacher teacher_of(const DistillArgs& a) {
    Teacher t{};
    t.ids = a.ids; t.t = a.teacher; t.V = a.V; t.k = (int)a.k; t.probs = a.probs; t.inv_tau = 1.0f / a.tau;
    return t;
}

// a = z / tau of vocabulary columns [c0, c0 + n) with an LM-head output kind.
GemmProblem logits(const DistillArgs& a, int64_t c0, int64_t n, int out) {
    GemmProblem g{};
    g.M = a.M; g.N = n; g.K = a.K;
    g.A = reinterpret_cast<const uint8_t*>(a.X); g.lda = a.K; g.fa = kBF16; g.sa_mode = kSNone;
    g.B = reinterpret_cast<const uint8_t*>(a.W + c0 * a.K); g.ldb = a.K; g.fb = kBF16; g.sb_mode = kSNone;
    g.out = out;
    g.col0 = (int)c0;
    g.alpha = 1.0f / a.tau;
    return g;
}

unsigned blocks(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

}  // namespace

size_t lm_distill_ws_bytes(int64_t M, int64_t V, int64_t K, int64_t k, bool bwd) { return layout(M, V, K, k, bwd).total; }

void launch_lm_distill_fwd(const DistillArgs& a, float* lse, float* loss, float* z_top, void* ws, hipStream_t stream) {
    uint8_t* const w8 = reinterpret_cast<uint8_t*>(ws);
    const Layout l = layout(a.M, a.V, a.K, a.k, false);
    GemmProblem g = logits(a, 0, a.V, kOutLseAny);
    g.stats = reinterpret_cast<float2*>(w8 + l.stats);
    g.stats_ld = pad128(a.V) / 128;
    g.ldd = a.V;
    launch_gemm(g, nullptr, stream);
    distill_rows_kernel<<<(unsigned)a.M, kThreads, 0, stream>>>(g.stats, g.stats_ld, (int)g.stats_ld, a.X, a.W, a.K,
                                                              teacher_of(a), z_top, lse, loss);
}

void launch_lm_distill_bwd(const DistillArgs& a, const float* lse, const float* z_top, const float* dloss, float grad_scale,
                           uint16_t* dX, void* dW, bool dw_bf16, int accumulate_dw, void* ws, hipStream_t stream) {
    uint8_t* const w8 = reinterpret_cast<uint8_t*>(ws);
    const int64_t M = a.M, V = a.V, K = a.K, Mp = pad128(M), Vp = pad128(V), Vc = chunk_of(Mp, Vp);
    const Layout l = layout(M, V, K, a.k, true);
    float* const coef = reinterpret_cast<float*>(w8 + l.coef);
    float* const val = reinterpret_cast<float*>(w8 + l.val);
    uint16_t* const xt = reinterpret_cast<uint16_t*>(w8 + l.xt);
    uint16_t* const wt = reinterpret_cast<uint16_t*>(w8 + l.wt);
    uint16_t* const dz = reinterpret_cast<uint16_t*>(w8 + l.dz);
    uint16_t* const dzt = reinterpret_cast<uint16_t*>(w8 + l.dzt);
    float* const dxacc = reinterpret_cast<float*>(w8 + l.dxacc);
    void* const gws = w8 + l.gemm;
    distill_coef_kernel<<<(unsigned)M, 64, (size_t)a.k * 8, stream>>>(teacher_of(a), z_top, lse, dloss, grad_scale / a.tau,
                                                                     coef, val);
    // the operands whose reduction runs down their columns, zeros past the last
    // row and in rows without a gradient (whose X may hold anything)
    if (dW) transpose_bf16(a.X, M, K, K, xt, Mp, stream, 1, 0, 0, Mp, coef);
    if (dX) transpose_bf16(a.W, V, K, K, wt, Vp, stream, 1, 0, 0, Vp);
    for (int64_t c0 = 0; c0 < V; c0 += Vc) {
        const int64_t n = std::min(V - c0, Vc), np = pad128(n);
        GemmProblem g = logits(a, c0, n, kOutSoftmaxGradT);
        g.M = Mp; g.N = np;
        g.rows_a = M; g.rows_b = n;
        g.lse = lse;
        g.row_scale = coef;
        g.D = dz; g.ldd = np;
        if (dW) { g.dzt = dzt; g.ld_dzt = Mp; }
        launch_gemm(g, nullptr, stream);
        distill_entries_kernel<<<blocks(M * a.k + Mp * (np - n)), kThreads, 0, stream>>>(
            a.ids, val, M * a.k, (int)a.k, c0, n, dz, Mp, np, dW ? dzt : nullptr, Mp);
        if (dX) {
            GemmProblem gx{};
            gx.M = M; gx.N = K; gx.K = np; gx.ldd = K; gx.long_k = 1;
            if (Vc < V) { gx.out = kOutF32; gx.D = dxacc; gx.accumulate = c0 > 0; }
            else { gx.out = kOutBF16; gx.D = dX; }
            gx.A = reinterpret_cast<const uint8_t*>(dz); gx.lda = np; gx.fa = kBF16; gx.sa_mode = kSNone;
            gx.B = reinterpret_cast<const uint8_t*>(wt + c0); gx.ldb = Vp; gx.fb = kBF16; gx.sb_mode = kSNone;
            launch_gemm(gx, gws, stream);
        }
        if (dW) {
            GemmProblem gw{};
            gw.M = n; gw.N = K; gw.K = Mp; gw.out = dw_bf16 ? kOutBF16 : kOutF32; gw.ldd = K; gw.accumulate = accumulate_dw;
            gw.D = reinterpret_cast<uint8_t*>(dW) + c0 * K * (dw_bf16 ? 2 : 4);
            gw.A = reinterpret_cast<const uint8_t*>(dzt); gw.lda = Mp; gw.fa = kBF16; gw.sa_mode = kSNone;
            gw.B = reinterpret_cast<const uint8_t*>(xt); gw.ldb = Mp; gw.fb = kBF16; gw.sb_mode = kSNone;
            launch_gemm(gw, gws, stream);
        }
    }
    if (dX && Vc < V) {
        const int64_t n4 = M * K / 4;
        f32_to_bf16_kernel<<<(unsigned)std::min((n4 + kThreads - 1) / kThreads, kMaxBlocks), kThreads, 0, stream>>>(dxacc, dX, n4);
    }
}

void launch_zero(void* dst, int64_t bytes, hipStream_t stream) {
    const int64_t n8 = bytes / 16;
    if (n8 > 0) zero_kernel<<<(unsigned)std::min((n8 + kThreads - 1) / kThreads, kMaxBlocks), kThreads, 0, stream>>>(
        reinterpret_cast<uint16_t*>(dst), n8);
}

}  // namespace puro
