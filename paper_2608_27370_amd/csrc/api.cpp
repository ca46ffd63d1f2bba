// C ABI of libpuro: argument validation, workspace layout and kernel launches.
// Declarations and their documentation: include/puro.h.

#include "puro.h"

#include <hip/hip_runtime.h>

#include "kernels.h"

using namespace puro;

namespace {

constexpr int64_t kGroup = 128;
constexpr size_t kAlign = 256;
// largest FP8 operand row pitch of the GEMM (bytes): buffer offsets over a
// 256-row tile stay below 2^31
constexpr int64_t kMaxPitch = (int64_t)1 << 22;

inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool fmt_ok(puro_fp8_format f) { return f == PURO_E4M3 || f == PURO_E5M2; }

puro_status launched() {
    return hipGetLastError() == hipSuccess ? PURO_OK : PURO_ERR_HIP;
}

// Byte offsets of named regions carved from a caller workspace.
struct Carver {
    size_t used = 0;
    size_t take(size_t bytes) {
        const size_t at = used;
        used = align_up(used + bytes);
        return at;
    }
};

size_t amax_ws(int64_t rows, int64_t cols) {
    return (size_t)amax_num_partials(rows, cols) * sizeof(uint32_t);
}

puro_status check_bf16_matrix(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld) {
    if (rows < 0 || cols < 0 || ld < cols) return PURO_ERR_SHAPE;
    if (rows > 0 && cols > 0 && !x) return PURO_ERR_NULL;
    if ((cols % 8) != 0 || (ld % 8) != 0 || !aligned16(x)) return PURO_ERR_ALIGN;
    if (rows > (int64_t)65535 * kGroup || cols > ((int64_t)1 << 31)) return PURO_ERR_SHAPE;
    return PURO_OK;
}

}  // namespace

extern "C" {

const char* puro_status_string(puro_status s) {
    switch (s) {
    case PURO_OK: return "ok";
    case PURO_ERR_NULL: return "a required pointer is NULL";
    case PURO_ERR_SHAPE: return "invalid or mismatched sizes";
    case PURO_ERR_UNSUPPORTED: return "unsupported format, scale mode or rounding combination";
    case PURO_ERR_ALIGN: return "size or pointer alignment not supported";
    case PURO_ERR_WORKSPACE: return "workspace too small";
    case PURO_ERR_HIP: return "HIP kernel launch failed";
    }
    return "unknown status";
}

// ------------------------------------------------------------------- amax
size_t puro_amax_workspace_size(int64_t rows, int64_t cols) {
    return amax_ws(rows, cols);
}

puro_status puro_amax(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, float* amax,
                      void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_bf16_matrix(x, rows, cols, ld);
    if (st != PURO_OK) return st;
    if (!amax) return PURO_ERR_NULL;
    const int P = amax_num_partials(rows, cols);
    if (P > 0 && !ws) return PURO_ERR_NULL;
    if (ws_bytes < (size_t)P * sizeof(uint32_t)) return PURO_ERR_WORKSPACE;
    uint32_t* partial = reinterpret_cast<uint32_t*>(ws);
    if (P > 0) launch_amax_partials(x, rows, cols, ld, partial, P, stream);
    launch_amax_finalize(partial, P, amax, stream);
    return launched();
}

// --------------------------------------------------------------- quantise
size_t puro_quantize_workspace_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return 0;
    return quant_tensor_ws_bytes(rows, cols);
}

}  // extern "C"

namespace {

// puro_quantize_fp8 and the fused quantise calls (the mode may carry the
// k-block-major layout flag). The values a quantisation encodes: the BF16 tensor x itself; the SwiGLU
// H = BF16(silu(gate) * up) [rows, cols] of a fused gate/up output x [rows,
// 2 cols]; or the RMSNorm y = BF16(x * rstd * gamma) of x [rows, cols], whose
// per-row rstd is written too.
struct Source {
    enum Kind { kBf16, kSwiglu, kRmsnorm, kSwigluBwd, kQkBwd } kind = kBf16;
    const uint16_t* gamma = nullptr;
    float* rstd = nullptr;
    float eps = 0.0f;
    // the SwiGLU backward's saved gate/up output (x is then dH)
    const uint16_t* gu = nullptr;
    int64_t ld_gu = 0;
    // the query / key norm's backward (x is then any of its gradients, checked already)
    const QkArgs* qk = nullptr;
};

puro_status quantize_impl(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, puro_fp8_format fmt,
                          puro_scale_mode mode_arg, puro_scale_rounding rnd, const float* amax_in, uint8_t* q,
                          float* scale, uint8_t* qT, float* scaleT, void* ws, size_t ws_bytes,
                          hipStream_t stream, Source src = Source(), bool static_ws = false) {
    // the scale-layout flag of the grouped modes
    const int kmajor = ((int)mode_arg & PURO_SCALE_KMAJOR) != 0;
    const puro_scale_mode mode = (puro_scale_mode)((int)mode_arg & ~(int)PURO_SCALE_KMAJOR);
    if (kmajor && mode == PURO_SCALE_TENSOR) return PURO_ERR_UNSUPPORTED;
    const bool swiglu = src.kind == Source::kSwiglu, rms = src.kind == Source::kRmsnorm;
    const bool bwd = src.kind == Source::kSwigluBwd;
    if (cols < 0) return PURO_ERR_SHAPE;
    // x's columns: 2 cols for the SwiGLU's gate/up input, cols / 2 for the backward's dH
    puro_status st = check_bf16_matrix(x, rows, swiglu ? 2 * cols : (bwd ? cols / 2 : cols), ld);
    if (st != PURO_OK) return st;
    if (bwd) {
        st = check_bf16_matrix(src.gu, rows, cols, src.ld_gu);
        if (st != PURO_OK) return st;
        if (src.ld_gu >= ((int64_t)1 << 23)) return PURO_ERR_SHAPE;
    }
    const bool qk = src.kind == Source::kQkBwd;
    if ((swiglu || rms || bwd || qk) && (amax_in || mode == PURO_SCALE_BLOCK_128x128)) return PURO_ERR_UNSUPPORTED;
    if (rms) {
        // a row needs its columns (the mean of an empty row is undefined)
        if (rows > 0 && cols == 0) return PURO_ERR_SHAPE;
        if (!(src.eps >= 0.0f) || !(src.eps <= 3.4028235e38f)) return PURO_ERR_UNSUPPORTED;
        if (rows > 0 && (!src.gamma || !src.rstd)) return PURO_ERR_NULL;
        if (rows > 0 && (!aligned16(src.gamma) || (reinterpret_cast<uintptr_t>(src.rstd) & 15) != 0))
            return PURO_ERR_ALIGN;
    }
    if (!fmt_ok(fmt) || (rnd != PURO_SCALE_FP32 && rnd != PURO_SCALE_POW2 && rnd != PURO_SCALE_POW2_FLOOR))
        return PURO_ERR_UNSUPPORTED;
    const bool pow2 = rnd == PURO_SCALE_POW2 || rnd == PURO_SCALE_POW2_FLOOR;
    if ((cols % 16) != 0) return PURO_ERR_ALIGN;
    // a 128-row tile spans less than 2^31 bytes (32-bit buffer offsets)
    if (ld >= ((int64_t)1 << 23)) return PURO_ERR_SHAPE;
    QuantArgs a{};
    a.x = x; a.rows = rows; a.cols = cols; a.ld = ld;
    a.q = q; a.scale = scale; a.qT = qT; a.scaleT = scaleT;
    a.amax = amax_in;
    a.supplied = amax_in != nullptr;
    a.pow2 = rnd == PURO_SCALE_POW2 ? 1 : (rnd == PURO_SCALE_POW2_FLOOR ? 2 : 0);
    a.kmajor = kmajor;
    a.gamma = src.gamma;
    a.rstd = src.rstd;
    a.x2 = src.gu;
    a.ld2 = src.ld_gu;
    // outputs of an empty tensor are never written (torch hands out NULL for them)
    const bool empty = rows == 0 || cols == 0;
    int qmode;
    switch (mode) {
    case PURO_SCALE_TENSOR:
        if (!empty && !q && !qT) return PURO_ERR_NULL;
        if (!scale) return PURO_ERR_NULL;
        if (qT && (rows % 16) != 0) return PURO_ERR_ALIGN;
        qmode = kQTensor;
        break;
    case PURO_SCALE_ROW_1x128:
        if (!empty && (!q || !scale || (qT && !scaleT))) return PURO_ERR_NULL;
        if (!pow2 || amax_in) return PURO_ERR_UNSUPPORTED;
        if ((cols % kGroup) != 0 || (qT && (rows % kGroup) != 0)) return PURO_ERR_ALIGN;
        qmode = kQRow;
        break;
    case PURO_SCALE_COL_128x1:
        if (!empty && (!qT || !scaleT)) return PURO_ERR_NULL;
        if (!pow2 || amax_in) return PURO_ERR_UNSUPPORTED;
        if ((rows % kGroup) != 0) return PURO_ERR_ALIGN;
        a.q = nullptr; a.scale = nullptr;
        qmode = kQCol;
        break;
    case PURO_SCALE_BLOCK_128x128:
        if (!empty && (!q || !scale || (qT && !scaleT))) return PURO_ERR_NULL;
        if (!pow2 || amax_in) return PURO_ERR_UNSUPPORTED;
        if ((rows % kGroup) != 0 || (cols % kGroup) != 0) return PURO_ERR_ALIGN;
        qmode = kQBlock;
        break;
    default:
        return PURO_ERR_UNSUPPORTED;
    }
    if (rms) {
        if (qmode == kQTensor) {
            if (!ws) return PURO_ERR_NULL;
            if (ws_bytes < rmsnorm_ws_bytes(rows)) return PURO_ERR_WORKSPACE;
        } else if (rows == 0) {
            return PURO_OK;
        }
        launch_rmsnorm_quantize(fmt, qmode, a, src.eps, ws, stream);
        return launched();
    }
    if (bwd) {
        if (qmode == kQTensor) {
            if (!ws) return PURO_ERR_NULL;
            if (ws_bytes < swiglu_bwd_ws_bytes(rows, cols)) return PURO_ERR_WORKSPACE;
        } else if (empty) {
            return PURO_OK;
        }
        launch_swiglu_bwd_quantize(fmt, qmode, a, ws, stream);
        return launched();
    }
    if (qk) {
        const bool sums = src.qk->dgq || src.qk->dgk;
        if (qmode == kQTensor || sums) {
            if (!ws) return PURO_ERR_NULL;
            if (!aligned16(ws)) return PURO_ERR_ALIGN;
            if (ws_bytes < qk_bwd_quantize_ws_bytes(rows, src.qk->hq, src.qk->hk, src.qk->D)) return PURO_ERR_WORKSPACE;
        } else if (empty) {
            return PURO_OK;
        }
        launch_qk_norm_rope_bwd_quantize(fmt, qmode, a, *src.qk, ws, stream);
        return launched();
    }
    if (qmode == kQTensor && !amax_in) {
        if (static_ws) {
            // the library's own scratch (arguments are valid by now)
            if (quant_tensor_ws_bytes(rows, cols) > kStaticScratchBytes) return PURO_ERR_WORKSPACE;
            if (static_scratch(&ws) != hipSuccess) return PURO_ERR_HIP;
            ws_bytes = kStaticScratchBytes;
        }
        if (!ws) return PURO_ERR_NULL;
        if (ws_bytes < quant_tensor_ws_bytes(rows, cols)) return PURO_ERR_WORKSPACE;
        launch_quantize_tensor(fmt, a, ws, stream, swiglu);
        return launched();
    }
    // an empty tensor has no groups
    if ((rows == 0 || cols == 0) && qmode != kQTensor) return PURO_OK;
    launch_quantize(fmt, qmode, a, stream, swiglu);
    return launched();
}

}  // namespace

extern "C" {

puro_status puro_quantize_fp8(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld,
                              puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                              const float* amax_in, uint8_t* q, float* scale, uint8_t* qT,
                              float* scaleT, void* ws, size_t ws_bytes, hipStream_t stream) {
    return quantize_impl(x, rows, cols, ld, fmt, mode, rnd, amax_in, q, scale, qT, scaleT, ws, ws_bytes, stream);
}

static_assert(PURO_QUANTIZE_STATIC_SCRATCH_BYTES == kStaticScratchBytes, "scratch size");

puro_status puro_quantize_fp8_static(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld,
                                     puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                     const float* amax_in, uint8_t* q, float* scale, uint8_t* qT, float* scaleT,
                                     hipStream_t stream) {
    return quantize_impl(x, rows, cols, ld, fmt, mode, rnd, amax_in, q, scale, qT, scaleT, nullptr, 0, stream,
                         Source(), true);
}

// ---------------------------------------------------- SwiGLU + quantise
size_t puro_swiglu_quantize_workspace_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return 0;
    return quant_tensor_ws_bytes(rows, cols);
}

puro_status puro_swiglu_quantize_fp8(const uint16_t* gu, int64_t rows, int64_t cols, int64_t ld,
                                     puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                     uint8_t* q, float* scale, uint8_t* qT, float* scaleT, void* ws,
                                     size_t ws_bytes, hipStream_t stream) {
    Source src;
    src.kind = Source::kSwiglu;
    return quantize_impl(gu, rows, cols, ld, fmt, mode, rnd, nullptr, q, scale, qT, scaleT, ws, ws_bytes, stream,
                         src);
}

// ------------------------------------------- SwiGLU backward + quantise
size_t puro_swiglu_bwd_quantize_workspace_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return 0;
    return swiglu_bwd_ws_bytes(rows, 2 * cols);
}

puro_status puro_swiglu_bwd_quantize_fp8(const uint16_t* dh, int64_t ld_dh, const uint16_t* gu, int64_t ld_gu,
                                         int64_t rows, int64_t cols, puro_fp8_format fmt, puro_scale_mode mode,
                                         puro_scale_rounding rnd, uint8_t* q, float* scale, uint8_t* qT,
                                         float* scaleT, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (cols < 0 || cols > ((int64_t)1 << 30)) return PURO_ERR_SHAPE;
    Source src;
    src.kind = Source::kSwigluBwd;
    src.gu = gu;
    src.ld_gu = ld_gu;
    return quantize_impl(dh, rows, 2 * cols, ld_dh, fmt, mode, rnd, nullptr, q, scale, qT, scaleT, ws, ws_bytes,
                         stream, src);
}

// --------------------------------------------------- RMSNorm + quantise
size_t puro_rmsnorm_quantize_workspace_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return 0;
    return rmsnorm_ws_bytes(rows);
}

puro_status puro_rmsnorm_quantize_fp8(const uint16_t* x, const uint16_t* gamma, int64_t rows, int64_t cols,
                                      int64_t ld, float eps, puro_fp8_format fmt, puro_scale_mode mode,
                                      puro_scale_rounding rnd, uint8_t* q, float* scale, uint8_t* qT,
                                      float* scaleT, float* rstd, void* ws, size_t ws_bytes, hipStream_t stream) {
    Source src;
    src.kind = Source::kRmsnorm;
    src.gamma = gamma;
    src.rstd = rstd;
    src.eps = eps;
    return quantize_impl(x, rows, cols, ld, fmt, mode, rnd, nullptr, q, scale, qT, scaleT, ws, ws_bytes, stream,
                         src);
}

}  // extern "C"

// ------------------------------- query / key norm with position rotation
namespace {

constexpr int kMaxHeadDim = 256;
// Tokens of a call: a launch holds fewer than 2^32 threads (the forward has a
// wave per token) and at most 65535 block rows (the quantiser's, of 128 tokens).
constexpr int64_t kMaxTokens = (int64_t)1 << 25, kMaxTokensQuant = (int64_t)1 << 22;

bool finite_nonneg(float v) { return v >= 0.0f && v <= 3.4028235e38f; }

// Sizes of a query / key call; tokens = batch * seq.
puro_status check_qk_sizes(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim, int64_t* tokens) {
    if (batch < 0 || seq < 0 || heads_q < 0 || heads_k < 0) return PURO_ERR_SHAPE;
    if (heads_q > 65535 || heads_k > 65535) return PURO_ERR_SHAPE;
    if (batch > INT32_MAX || seq > INT32_MAX || batch * seq > kMaxTokens) return PURO_ERR_SHAPE;
    if (head_dim < 8 || head_dim > kMaxHeadDim) return PURO_ERR_SHAPE;
    if ((head_dim % 8) != 0) return PURO_ERR_ALIGN;
    *tokens = batch * seq;
    return PURO_OK;
}

// Heads that the call touches: their place, and for outputs that no two of
// them overlap. Strides of dimensions of size one are not looked at.
puro_status check_heads(const puro_heads* h, int64_t batch, int64_t seq, int heads, int head_dim, bool output,
                        HeadsArg* arg) {
    *arg = HeadsArg{};
    if (batch == 0 || seq == 0 || heads == 0) return PURO_OK;
    if (!h || !h->data) return PURO_ERR_NULL;
    struct Dim { int64_t n, stride; } d[3] = {{batch, h->batch_stride}, {seq, h->row_stride}, {heads, h->head_stride}};
    __int128 span = 0;
    for (Dim& x : d) {
        if (x.n == 1) x.stride = 0;
        if (x.stride < 0) return PURO_ERR_SHAPE;
        if ((x.stride % 8) != 0) return PURO_ERR_ALIGN;
        span += (__int128)(x.n - 1) * x.stride;
    }
    if (span > ((__int128)1 << 46)) return PURO_ERR_SHAPE;
    if (!aligned16(h->data)) return PURO_ERR_ALIGN;
    *arg = HeadsArg{h->data, d[0].stride, d[1].stride, d[2].stride};
    if (output) {
        // by rising stride, each dimension steps past everything below it
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2 - i; ++j)
                if (d[j].stride > d[j + 1].stride) { const Dim t = d[j]; d[j] = d[j + 1]; d[j + 1] = t; }
        int64_t extent = head_dim;
        for (const Dim& x : d) {
            if (x.n == 1) continue;
            if (x.stride < extent) return PURO_ERR_SHAPE;
            extent += (x.n - 1) * x.stride;
        }
    }
    return PURO_OK;
}

puro_status check_rope(const puro_rope* r, int64_t seq, int64_t tokens, int head_dim, RopeArgs* arg) {
    *arg = RopeArgs{};
    if (!r || r->dim == 0) return PURO_OK;
    if (r->dim < 0 || r->dim > head_dim || r->len < 0 || r->len > INT32_MAX) return PURO_ERR_SHAPE;
    if ((r->dim % 16) != 0) return PURO_ERR_ALIGN;
    if (r->interleaved != 0 && r->interleaved != 1) return PURO_ERR_UNSUPPORTED;
    if (tokens > 0) {
        if (!r->positions && seq > r->len) return PURO_ERR_SHAPE;
        if (r->len == 0) return PURO_ERR_SHAPE;       // (no entry to stand in for one outside)
        if (!r->table) return PURO_ERR_NULL;
        if (!aligned16(r->table) || ((uintptr_t)r->positions & 3) != 0) return PURO_ERR_ALIGN;
    }
    *arg = RopeArgs{reinterpret_cast<const float2*>(r->table), r->positions, (int)r->len, r->dim, r->interleaved};
    return PURO_OK;
}

// What the three calls have in common: sizes, rotation, weights and the heads
// before the norm (needed by the backward only where there is a weight).
puro_status check_qk(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim, const puro_heads* q,
                     const puro_heads* k, const uint16_t* gamma_q, const uint16_t* gamma_k, float eps,
                     const puro_rope* rope, bool backward, QkArgs* a) {
    puro_status st = check_qk_sizes(batch, seq, heads_q, heads_k, head_dim, &a->tokens);
    if (st != PURO_OK) return st;
    if (!finite_nonneg(eps)) return PURO_ERR_UNSUPPORTED;
    if ((gamma_q && !aligned16(gamma_q)) || (gamma_k && !aligned16(gamma_k))) return PURO_ERR_ALIGN;
    st = check_rope(rope, seq, a->tokens, head_dim, &a->rope);
    if (st != PURO_OK) return st;
    if (!backward || gamma_q) st = check_heads(q, batch, seq, heads_q, head_dim, false, &a->q);
    if (st != PURO_OK) return st;
    if (!backward || gamma_k) st = check_heads(k, batch, seq, heads_k, head_dim, false, &a->k);
    if (st != PURO_OK) return st;
    a->gq = gamma_q; a->gk = gamma_k;
    a->eps = eps;
    a->seq = (int)seq; a->hq = heads_q; a->hk = heads_k; a->D = head_dim;
    return PURO_OK;
}

// dgamma of heads that have no gamma is not defined.
puro_status check_dgamma(const QkArgs& a) {
    if ((a.dgq && !a.gq) || (a.dgk && !a.gk)) return PURO_ERR_NULL;
    if (((uintptr_t)a.dgq & 3) != 0 || ((uintptr_t)a.dgk & 3) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

}  // namespace

extern "C" {

puro_status puro_rope_table(float* table, int64_t len, int dim, double theta, hipStream_t stream) {
    if (len < 0 || len > INT32_MAX || dim < 0 || dim > kMaxHeadDim) return PURO_ERR_SHAPE;
    if ((dim % 16) != 0) return PURO_ERR_ALIGN;
    if (!(theta > 0.0) || !(theta <= 1.7976931348623157e308)) return PURO_ERR_UNSUPPORTED;
    if (len * (dim / 2) > (int64_t)1 << 31) return PURO_ERR_SHAPE;
    if (len == 0 || dim == 0) return PURO_OK;
    if (!table) return PURO_ERR_NULL;
    if (!aligned16(table)) return PURO_ERR_ALIGN;
    launch_rope_table(reinterpret_cast<float2*>(table), len, dim, theta, stream);
    return launched();
}

puro_status puro_qk_norm_rope_fwd(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                  const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                  const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                  const puro_heads* q_out, const puro_heads* k_out, hipStream_t stream) {
    QkArgs a{};
    puro_status st = check_qk(batch, seq, heads_q, heads_k, head_dim, q, k, gamma_q, gamma_k, eps, rope, false, &a);
    if (st != PURO_OK) return st;
    if ((st = check_heads(q_out, batch, seq, heads_q, head_dim, true, &a.oq)) != PURO_OK) return st;
    if ((st = check_heads(k_out, batch, seq, heads_k, head_dim, true, &a.ok)) != PURO_OK) return st;
    if (a.tokens == 0 || heads_q + heads_k == 0) return PURO_OK;
    launch_qk_norm_rope_fwd(a, stream);
    return launched();
}

size_t puro_qk_norm_rope_bwd_workspace_size(int64_t batch, int64_t seq, int head_dim) {
    int64_t tokens;
    if (check_qk_sizes(batch, seq, 0, 0, head_dim, &tokens) != PURO_OK) return 0;
    return qk_bwd_ws_bytes(tokens, head_dim);
}

puro_status puro_qk_norm_rope_bwd(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                  const puro_heads* dq, const puro_heads* dk, const puro_heads* dv,
                                  const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                  const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                  const puro_heads* dq_in, const puro_heads* dk_in, const puro_heads* dv_in,
                                  float* dgamma_q, float* dgamma_k, void* ws, size_t ws_bytes,
                                  hipStream_t stream) {
    QkArgs a{};
    puro_status st = check_qk(batch, seq, heads_q, heads_k, head_dim, q, k, gamma_q, gamma_k, eps, rope, true, &a);
    if (st != PURO_OK) return st;
    if ((st = check_heads(dq, batch, seq, heads_q, head_dim, false, &a.dq)) != PURO_OK) return st;
    if ((st = check_heads(dk, batch, seq, heads_k, head_dim, false, &a.dk)) != PURO_OK) return st;
    if ((st = check_heads(dq_in, batch, seq, heads_q, head_dim, true, &a.oq)) != PURO_OK) return st;
    if ((st = check_heads(dk_in, batch, seq, heads_k, head_dim, true, &a.ok)) != PURO_OK) return st;
    if (dv || dv_in) {
        if (!dv || !dv_in) return PURO_ERR_NULL;
        if ((st = check_heads(dv, batch, seq, heads_k, head_dim, false, &a.dv)) != PURO_OK) return st;
        if ((st = check_heads(dv_in, batch, seq, heads_k, head_dim, true, &a.ov)) != PURO_OK) return st;
    }
    a.dgq = dgamma_q; a.dgk = dgamma_k;
    if ((st = check_dgamma(a)) != PURO_OK) return st;
    const bool sums = dgamma_q || dgamma_k;
    if (sums) {
        if (!ws) return PURO_ERR_NULL;
        if (!aligned16(ws)) return PURO_ERR_ALIGN;
        if (ws_bytes < qk_bwd_ws_bytes(a.tokens, head_dim)) return PURO_ERR_WORKSPACE;
    }
    if (!sums && (a.tokens == 0 || heads_q + heads_k == 0)) return PURO_OK;
    launch_qk_norm_rope_bwd(a, ws, stream);
    return launched();
}

size_t puro_qk_norm_rope_bwd_quantize_workspace_size(int64_t batch, int64_t seq, int heads_q, int heads_k,
                                                     int head_dim) {
    int64_t tokens;
    if (check_qk_sizes(batch, seq, heads_q, heads_k, head_dim, &tokens) != PURO_OK) return 0;
    return qk_bwd_quantize_ws_bytes(tokens, heads_q, heads_k, head_dim);
}

puro_status puro_qk_norm_rope_bwd_quantize_fp8(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                               const puro_heads* dq, const puro_heads* dk, const puro_heads* dv,
                                               const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                               const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                               puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                               uint8_t* q8, float* scale, uint8_t* qT, float* scaleT,
                                               float* dgamma_q, float* dgamma_k, void* ws, size_t ws_bytes,
                                               hipStream_t stream) {
    QkArgs a{};
    puro_status st = check_qk(batch, seq, heads_q, heads_k, head_dim, q, k, gamma_q, gamma_k, eps, rope, true, &a);
    if (st != PURO_OK) return st;
    if (head_dim != 64 && head_dim != 128) return PURO_ERR_UNSUPPORTED;
    if (a.tokens > kMaxTokensQuant) return PURO_ERR_SHAPE;
    if ((st = check_heads(dq, batch, seq, heads_q, head_dim, false, &a.dq)) != PURO_OK) return st;
    if ((st = check_heads(dk, batch, seq, heads_k, head_dim, false, &a.dk)) != PURO_OK) return st;
    if ((st = check_heads(dv, batch, seq, heads_k, head_dim, false, &a.dv)) != PURO_OK) return st;
    a.dgq = dgamma_q; a.dgk = dgamma_k;
    if ((st = check_dgamma(a)) != PURO_OK) return st;
    Source src;
    src.kind = Source::kQkBwd;
    src.qk = &a;
    const int64_t cols = ((int64_t)heads_q + 2 * heads_k) * head_dim;
    return quantize_impl(a.dq.p ? a.dq.p : a.dk.p, a.tokens, cols, cols, fmt, mode, rnd, nullptr, q8, scale, qT, scaleT, ws,
                         ws_bytes, stream, src);
}

// ------------------------------------------------------------------- GEMM
size_t puro_fp8_gemm_workspace_size(int64_t M, int64_t N, int64_t K, puro_out_dtype d_type) {
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    return gemm_workspace_bytes(M, N, K, d_type == PURO_OUT_FP32 ? kOutF32 : kOutBF16);
}

puro_status puro_fp8_gemm_plan(int64_t M, int64_t N, int64_t K, puro_scale_mode a_mode,
                               puro_scale_mode b_mode, int* tile_m, int* tile_n, int* stages, int* splits,
                               int* launches) {
    if (M < 0 || N < 0 || K < 0) return PURO_ERR_SHAPE;
    auto ok = [](puro_scale_mode m) {
        const int g = (int)m & ~(int)PURO_SCALE_KMAJOR;
        return m == PURO_SCALE_TENSOR || g == PURO_SCALE_ROW_1x128 || g == PURO_SCALE_BLOCK_128x128;
    };
    if (!ok(a_mode) || !ok(b_mode)) return PURO_ERR_UNSUPPORTED;
    int tm = 0, tn = 0, ns = 0, s = 1;
    gemm_plan(M, N, K, a_mode != PURO_SCALE_TENSOR || b_mode != PURO_SCALE_TENSOR, &tm, &tn, &ns, &s);
    if (tile_m) *tile_m = tm;
    if (tile_n) *tile_n = tn;
    if (stages) *stages = ns;
    if (splits) *splits = s;
    if (launches) *launches = (M > 0 && N > 0) ? 1 + (s > 1) : 0;
    return PURO_OK;
}

static puro_status check_operand(const puro_fp8_operand* o, int64_t rows, int64_t K, int* smode, int* kmajor) {
    if (!o) return PURO_ERR_NULL;
    // the scale is read whenever the operand has rows (also for K == 0, where
    // the result is a scaled empty sum); the data only when there is a k
    if (rows > 0 && (!o->scale || (K > 0 && !o->data))) return PURO_ERR_NULL;
    if (!fmt_ok(o->fmt)) return PURO_ERR_UNSUPPORTED;
    if (o->ld < K) return PURO_ERR_SHAPE;
    if ((o->ld % 16) != 0 || !aligned16(o->data)) return PURO_ERR_ALIGN;
    // buffer offsets within one tile of 256 rows stay below 2^31
    if (o->ld > kMaxPitch) return PURO_ERR_SHAPE;
    *kmajor = ((int)o->mode & PURO_SCALE_KMAJOR) != 0;
    switch ((int)o->mode & ~(int)PURO_SCALE_KMAJOR) {
    case PURO_SCALE_TENSOR:
        if (*kmajor) return PURO_ERR_UNSUPPORTED;
        *smode = kSTensor;
        break;
    case PURO_SCALE_ROW_1x128: *smode = kSRow; break;
    case PURO_SCALE_BLOCK_128x128: *smode = kSBlock; break;
    default: return PURO_ERR_UNSUPPORTED;
    }
    if (*smode != kSTensor && (K % kGroup) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

}  // extern "C"

namespace {

// puro_fp8_gemm with a choice of grouped-scale layout per operand.
// bias / residual: the BF16 epilogue (both NULL: none).
puro_status gemm_impl(int64_t M, int64_t N, int64_t K, const puro_fp8_operand* A, const puro_fp8_operand* B,
                      void* D, puro_out_dtype d_type, int64_t ldd, int accumulate, void* ws, size_t ws_bytes,
                      hipStream_t stream, const uint16_t* bias = nullptr, const uint16_t* residual = nullptr,
                      int64_t ldr = 0) {
    if (M < 0 || N < 0 || K < 0) return PURO_ERR_SHAPE;
    if (M > INT32_MAX / 2 || N > INT32_MAX / 2 || K > INT32_MAX / 2) return PURO_ERR_SHAPE;
    int sa = 0, sb = 0, a_kmajor = 0, b_kmajor = 0;
    puro_status st = check_operand(A, M, K, &sa, &a_kmajor);
    if (st != PURO_OK) return st;
    st = check_operand(B, N, K, &sb, &b_kmajor);
    if (st != PURO_OK) return st;
    if (d_type != PURO_OUT_BF16 && d_type != PURO_OUT_FP32) return PURO_ERR_UNSUPPORTED;
    if ((K % 16) != 0) return PURO_ERR_ALIGN;
    if (ldd < N) return PURO_ERR_SHAPE;
    if (M == 0 || N == 0) return PURO_OK;
    if (!D) return PURO_ERR_NULL;
    if ((ldd % 4) != 0 || !aligned16(D)) return PURO_ERR_ALIGN;
    const bool epi = bias || residual;
    if (epi) {
        if (d_type != PURO_OUT_BF16 || accumulate) return PURO_ERR_UNSUPPORTED;
        if (bias && !aligned16(bias)) return PURO_ERR_ALIGN;
        // ldr as the operands' pitch: buffer offsets over a tile's rows stay below 2^31
        if (residual && (ldr < N || ldr > kMaxPitch)) return PURO_ERR_SHAPE;
        if (residual && (!aligned16(residual) || (ldr % 4) != 0)) return PURO_ERR_ALIGN;
        // the residual may be D itself (an in-place residual add), but not overlap it otherwise
        if (residual && residual != D) {
            const uintptr_t r0 = (uintptr_t)residual, r1 = r0 + (uintptr_t)(((M - 1) * ldr + N) * 2);
            const uintptr_t d0 = (uintptr_t)D, d1 = d0 + (uintptr_t)(((M - 1) * ldd + N) * 2);
            if (r0 < d1 && d0 < r1) return PURO_ERR_SHAPE;
        }
        if (residual == D && ldr != ldd) return PURO_ERR_SHAPE;
    }
    const int out = d_type == PURO_OUT_FP32 ? kOutF32 : (epi ? kOutBF16Epi : kOutBF16);
    const size_t need = gemm_workspace_bytes(M, N, K, out);
    if (need > 0 && !ws) return PURO_ERR_NULL;
    if (ws_bytes < need) return PURO_ERR_WORKSPACE;
    GemmProblem g{};
    g.M = M; g.N = N; g.K = K;
    g.A = A->data; g.lda = A->ld; g.fa = A->fmt; g.sa_mode = sa; g.sa = A->scale;
    g.B = B->data; g.ldb = B->ld; g.fb = B->fmt; g.sb_mode = sb; g.sb = B->scale;
    g.D = D; g.ldd = ldd; g.out = out; g.accumulate = accumulate != 0;
    g.sa_kmajor = a_kmajor; g.sb_kmajor = b_kmajor;
    g.bias = bias; g.residual = residual; g.ldr = ldr;
    // a Wgrad's dW is far larger than the L2 and next read by another kernel:
    // stream it past the caches (BF16 outputs always are)
    g.nt_f32 = 1;
    launch_gemm(g, ws, stream);
    return launched();
}

}  // namespace

extern "C" {

puro_status puro_fp8_gemm(int64_t M, int64_t N, int64_t K, const puro_fp8_operand* A,
                          const puro_fp8_operand* B, void* D, puro_out_dtype d_type, int64_t ldd,
                          int accumulate, void* ws, size_t ws_bytes, hipStream_t stream) {
    return gemm_impl(M, N, K, A, B, D, d_type, ldd, accumulate, ws, ws_bytes, stream);
}

puro_status puro_fp8_gemm_epilogue(int64_t M, int64_t N, int64_t K, const puro_fp8_operand* A,
                                   const puro_fp8_operand* B, uint16_t* D, int64_t ldd, const uint16_t* bias,
                                   const uint16_t* residual, int64_t ldr, void* ws, size_t ws_bytes,
                                   hipStream_t stream) {
    return gemm_impl(M, N, K, A, B, D, PURO_OUT_BF16, ldd, 0, ws, ws_bytes, stream, bias, residual, ldr);
}

// ----------------------------------------------------------- linear layer
namespace {

// The linear layer keeps its grouped scales k-block-major: the GEMMs load a
// k slice's scales as contiguous runs.
constexpr puro_scale_mode kRowKM = (puro_scale_mode)(PURO_SCALE_ROW_1x128 | PURO_SCALE_KMAJOR);
constexpr puro_scale_mode kBlockKM = (puro_scale_mode)(PURO_SCALE_BLOCK_128x128 | PURO_SCALE_KMAJOR);

// The power-of-two rule of a blockwise recipe.
puro_scale_rounding block_rule(const puro_linear_recipe* r) {
    return r->rnd == PURO_SCALE_POW2_FLOOR ? PURO_SCALE_POW2_FLOOR : PURO_SCALE_POW2;
}

bool recipe_ok(const puro_linear_recipe* r) {
    return r && fmt_ok(r->x_fmt) && fmt_ok(r->w_fmt) && fmt_ok(r->dy_fmt) &&
           (r->blockwise == 0 || r->blockwise == 1) &&
           (r->rnd == PURO_SCALE_FP32 || r->rnd == PURO_SCALE_POW2 || r->rnd == PURO_SCALE_POW2_FLOOR);
}

puro_status check_linear_dims(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r) {
    if (!recipe_ok(r)) return PURO_ERR_UNSUPPORTED;
    if (M < 0 || N < 0 || K < 0) return PURO_ERR_SHAPE;
    // each of M, N and K is the row pitch of an FP8 operand of one of the
    // three GEMMs (Xq, dYq, the transposed copies), limited to 2^22 bytes;
    // rejected here, before the quantisers write anything
    if (M > kMaxPitch || N > kMaxPitch || K > kMaxPitch) return PURO_ERR_SHAPE;
    const int64_t g = r->blockwise ? kGroup : 16;
    if ((M % g) != 0 || (N % g) != 0 || (K % g) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

struct FwdLayout {
    size_t xq, wq, xs_row, w_blk, part_x, part_w, gemm, total;
};

FwdLayout fwd_layout(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r) {
    Carver c;
    FwdLayout l{};
    l.xq = c.take((size_t)M * K);
    l.wq = c.take((size_t)N * K);
    if (r->blockwise) {
        l.xs_row = c.take((size_t)M * (K / kGroup) * sizeof(float));
        l.w_blk = c.take((size_t)(N / kGroup) * (K / kGroup) * sizeof(float));
    } else {
        l.part_x = c.take(quant_tensor_ws_bytes(M, K));
        l.part_w = c.take(quant_tensor_ws_bytes(N, K));
    }
    l.gemm = c.take(gemm_workspace_bytes(M, N, K, kOutBF16));
    l.total = c.used;
    return l;
}

struct BwdLayout {
    size_t dyq, dyq_t, dy_scale, dy_scale_t, part, gemm, total;
};

BwdLayout bwd_layout(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r) {
    Carver c;
    BwdLayout l{};
    l.dyq = c.take((size_t)M * N);
    l.dyq_t = c.take((size_t)N * M);
    if (r->blockwise) {
        l.dy_scale = c.take((size_t)M * (N / kGroup) * sizeof(float));
        l.dy_scale_t = c.take((size_t)N * (M / kGroup) * sizeof(float));
    } else {
        l.dy_scale = c.take(sizeof(float));
        l.part = c.take(quant_tensor_ws_bytes(M, N));
    }
    const size_t g1 = gemm_workspace_bytes(M, K, N, kOutBF16);
    const size_t g2 = gemm_workspace_bytes(N, K, M, kOutF32);
    l.gemm = c.take(g1 > g2 ? g1 : g2);
    l.total = c.used;
    return l;
}

}  // namespace

size_t puro_linear_saved_bytes(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r,
                               size_t sizes[4]) {
    size_t s[4] = {0, 0, 0, 0};
    if (recipe_ok(r) && M >= 0 && N >= 0 && K >= 0) {
        s[0] = (size_t)K * M;
        s[1] = r->blockwise ? (size_t)K * (M / kGroup) * sizeof(float) : sizeof(float);
        s[2] = (size_t)K * N;
        s[3] = r->blockwise ? (size_t)(K / kGroup) * (N / kGroup) * sizeof(float) : sizeof(float);
    }
    if (sizes)
        for (int i = 0; i < 4; ++i) sizes[i] = s[i];
    return s[0] + s[1] + s[2] + s[3];
}

size_t puro_linear_fwd_workspace_size(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r) {
    if (check_linear_dims(M, N, K, r) != PURO_OK) return 0;
    return fwd_layout(M, N, K, r).total;
}

size_t puro_linear_bwd_workspace_size(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* r) {
    if (check_linear_dims(M, N, K, r) != PURO_OK) return 0;
    return bwd_layout(M, N, K, r).total;
}

puro_status puro_linear_fwd(const uint16_t* X, const uint16_t* W, int64_t M, int64_t N, int64_t K,
                            const puro_linear_recipe* r, uint16_t* Y, const puro_linear_saved* saved,
                            void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_linear_dims(M, N, K, r);
    if (st != PURO_OK) return st;
    if (!saved || !X || !W || !Y || !saved->xq_t || !saved->x_scale || !saved->wq_t || !saved->w_scale)
        return PURO_ERR_NULL;
    if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || !aligned16(saved->xq_t) ||
        !aligned16(saved->wq_t))
        return PURO_ERR_ALIGN;
    const FwdLayout l = fwd_layout(M, N, K, r);
    if (!ws) return PURO_ERR_NULL;
    if (ws_bytes < l.total) return PURO_ERR_WORKSPACE;
    uint8_t* w8 = reinterpret_cast<uint8_t*>(ws);
    uint8_t* xq = w8 + l.xq;
    uint8_t* wq = w8 + l.wq;
    puro_fp8_operand A{}, B{};
    if (!r->blockwise) {
        // X and W with their own amax each: q (Fprop) and qT (kept for Wgrad
        // and Dgrad), in one amax launch and one quantise launch for both
        QuantArgs ax{}, aw{};
        ax.x = X; ax.rows = M; ax.cols = K; ax.ld = K;
        ax.q = xq; ax.scale = saved->x_scale; ax.qT = saved->xq_t;
        ax.pow2 = r->rnd == PURO_SCALE_POW2 ? 1 : (r->rnd == PURO_SCALE_POW2_FLOOR ? 2 : 0);
        aw = ax;
        aw.x = W; aw.rows = N;
        aw.q = wq; aw.scale = saved->w_scale; aw.qT = saved->wq_t;
        if (r->x_fmt == r->w_fmt) {
            launch_quantize_tensor_pair(r->x_fmt, ax, w8 + l.part_x, aw, w8 + l.part_w, stream);
        } else {
            launch_quantize_tensor(r->x_fmt, ax, w8 + l.part_x, stream);
            launch_quantize_tensor(r->w_fmt, aw, w8 + l.part_w, stream);
        }
        if ((st = launched()) != PURO_OK) return st;
        A = puro_fp8_operand{xq, K, r->x_fmt, PURO_SCALE_TENSOR, saved->x_scale};
        B = puro_fp8_operand{wq, K, r->w_fmt, PURO_SCALE_TENSOR, saved->w_scale};
    } else {
        // X: 1x128 row groups for Fprop and, from the same read, the 128x1
        // column-grouped transposed copy kept for Wgrad.
        float* xs_row = reinterpret_cast<float*>(w8 + l.xs_row);
        float* w_blk = reinterpret_cast<float*>(w8 + l.w_blk);
        st = quantize_impl(X, M, K, K, r->x_fmt, kRowKM, block_rule(r), nullptr, xq, xs_row, saved->xq_t,
                           saved->x_scale, nullptr, 0, stream);
        if (st != PURO_OK) return st;
        // W: 128x128 blocks, plus the transposed copy (same blocks) kept for Dgrad.
        st = quantize_impl(W, N, K, K, r->w_fmt, kBlockKM, block_rule(r), nullptr, wq, w_blk, saved->wq_t,
                           saved->w_scale, nullptr, 0, stream);
        if (st != PURO_OK) return st;
        A = puro_fp8_operand{xq, K, r->x_fmt, kRowKM, xs_row};
        B = puro_fp8_operand{wq, K, r->w_fmt, kBlockKM, w_blk};
    }
    return gemm_impl(M, N, K, &A, &B, Y, PURO_OUT_BF16, N, 0, w8 + l.gemm, ws_bytes - l.gemm, stream);
}

puro_status puro_linear_bwd(const uint16_t* dY, const puro_linear_saved* saved, int64_t M, int64_t N,
                            int64_t K, const puro_linear_recipe* r, uint16_t* dX, float* dW,
                            int accumulate_dW, void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_linear_dims(M, N, K, r);
    if (st != PURO_OK) return st;
    if (!saved || !dY || !saved->xq_t || !saved->x_scale || !saved->wq_t || !saved->w_scale)
        return PURO_ERR_NULL;
    if (!aligned16(dY) || !aligned16(saved->xq_t) || !aligned16(saved->wq_t) || (dX && !aligned16(dX)) ||
        (dW && !aligned16(dW)))
        return PURO_ERR_ALIGN;
    if (!dX && !dW) return PURO_OK;
    const BwdLayout l = bwd_layout(M, N, K, r);
    if (!ws) return PURO_ERR_NULL;
    if (ws_bytes < l.total) return PURO_ERR_WORKSPACE;
    uint8_t* w8 = reinterpret_cast<uint8_t*>(ws);
    uint8_t* dyq = w8 + l.dyq;
    uint8_t* dyq_t = w8 + l.dyq_t;
    float* dys = reinterpret_cast<float*>(w8 + l.dy_scale);
    float* dys_t = reinterpret_cast<float*>(w8 + l.dy_scale_t);
    void* gws = w8 + l.gemm;
    const size_t gws_bytes = ws_bytes - l.gemm;
    puro_fp8_operand dA{}, dB{}, wA{}, wB{};
    if (!r->blockwise) {
        st = puro_quantize_fp8(dY, M, N, N, r->dy_fmt, PURO_SCALE_TENSOR, r->rnd, nullptr, dyq, dys, dyq_t,
                               nullptr, w8 + l.part, quant_tensor_ws_bytes(M, N), stream);
        if (st != PURO_OK) return st;
        dA = puro_fp8_operand{dyq, N, r->dy_fmt, PURO_SCALE_TENSOR, dys};
        dB = puro_fp8_operand{saved->wq_t, N, r->w_fmt, PURO_SCALE_TENSOR, saved->w_scale};
        wA = puro_fp8_operand{dyq_t, M, r->dy_fmt, PURO_SCALE_TENSOR, dys};
        wB = puro_fp8_operand{saved->xq_t, M, r->x_fmt, PURO_SCALE_TENSOR, saved->x_scale};
    } else {
        st = quantize_impl(dY, M, N, N, r->dy_fmt, kRowKM, block_rule(r), nullptr, dyq, dys, dyq_t, dys_t, nullptr,
                           0, stream);
        if (st != PURO_OK) return st;
        dA = puro_fp8_operand{dyq, N, r->dy_fmt, kRowKM, dys};
        dB = puro_fp8_operand{saved->wq_t, N, r->w_fmt, kBlockKM, saved->w_scale};
        wA = puro_fp8_operand{dyq_t, M, r->dy_fmt, kRowKM, dys_t};
        wB = puro_fp8_operand{saved->xq_t, M, r->x_fmt, kRowKM, saved->x_scale};
    }
    if (dX) {
        st = gemm_impl(M, K, N, &dA, &dB, dX, PURO_OUT_BF16, K, 0, gws, gws_bytes, stream);
        if (st != PURO_OK) return st;
    }
    if (dW) {
        st = gemm_impl(N, K, M, &wA, &wB, dW, PURO_OUT_FP32, K, accumulate_dW, gws, gws_bytes, stream);
        if (st != PURO_OK) return st;
    }
    return PURO_OK;
}

}  // extern "C"

// ------------------------------------------ LM head with cross-entropy loss
namespace {

puro_status check_lm_head(const uint16_t* X, const uint16_t* W, const int32_t* targets, int64_t M, int64_t V,
                          int64_t K, puro_lm_head_recipe r) {
    if (r != PURO_LM_HEAD_BF16 && r != PURO_LM_HEAD_FP8) return PURO_ERR_UNSUPPORTED;
    if (M <= 0 || V <= 0 || K <= 0) return PURO_ERR_SHAPE;
    // BF16 operand pitches (2 M, 2 V, 2 K bytes for the transposed copies) within 2^22
    const int64_t lim = (int64_t)1 << 21;
    if (M > lim || V > lim || K > lim) return PURO_ERR_SHAPE;
    if ((M % kGroup) != 0 || (V % kGroup) != 0 || (K % kGroup) != 0) return PURO_ERR_ALIGN;
    if (!X || !W || !targets) return PURO_ERR_NULL;
    if (!aligned16(X) || !aligned16(W) || ((uintptr_t)targets & 3) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

}  // namespace

extern "C" {

size_t puro_lm_head_ce_workspace_size(int64_t M, int64_t V, int64_t K, puro_lm_head_recipe recipe, int backward) {
    if (check_lm_head(reinterpret_cast<const uint16_t*>(16), reinterpret_cast<const uint16_t*>(16),
                      reinterpret_cast<const int32_t*>(16), M, V, K, recipe) != PURO_OK)
        return 0;
    return lm_head_ws_bytes(M, V, K, recipe == PURO_LM_HEAD_FP8, backward != 0);
}

puro_status puro_lm_head_ce_fwd(const uint16_t* X, const uint16_t* W, const int32_t* targets, int64_t M,
                                int64_t V, int64_t K, puro_lm_head_recipe recipe, float* lse, float* loss,
                                void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_lm_head(X, W, targets, M, V, K, recipe);
    if (st != PURO_OK) return st;
    if (!lse || !loss || !ws) return PURO_ERR_NULL;
    if (!aligned16(lse) || !aligned16(loss)) return PURO_ERR_ALIGN;
    if (ws_bytes < lm_head_ws_bytes(M, V, K, recipe == PURO_LM_HEAD_FP8, false)) return PURO_ERR_WORKSPACE;
    launch_lm_head_fwd(X, W, targets, M, V, K, recipe == PURO_LM_HEAD_FP8, lse, loss, ws, stream);
    return launched();
}

puro_status puro_lm_head_ce_bwd(const uint16_t* X, const uint16_t* W, const int32_t* targets, const float* lse,
                                int64_t M, int64_t V, int64_t K, puro_lm_head_recipe recipe, float grad_scale,
                                uint16_t* dX, float* dW, void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_lm_head(X, W, targets, M, V, K, recipe);
    if (st != PURO_OK) return st;
    if (!lse || !dX || !dW || !ws) return PURO_ERR_NULL;
    if (!aligned16(lse) || !aligned16(dX) || !aligned16(dW)) return PURO_ERR_ALIGN;
    if (!(grad_scale == grad_scale) || grad_scale > 3.4028235e38f || grad_scale < -3.4028235e38f)
        return PURO_ERR_UNSUPPORTED;
    if (ws_bytes < lm_head_ws_bytes(M, V, K, recipe == PURO_LM_HEAD_FP8, true)) return PURO_ERR_WORKSPACE;
    launch_lm_head_bwd(X, W, targets, lse, M, V, K, recipe == PURO_LM_HEAD_FP8, grad_scale, dX, dW, ws, stream);
    return launched();
}

}  // extern "C"

// ------------------------------------- LM head with a teacher's top logits
namespace {

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

puro_status check_distill_sizes(int64_t M, int64_t V, int64_t K, int64_t topk) {
    // BF16 operand pitches (2 M, 2 V, 2 K bytes, padded to 128 values) within 2^22
    const int64_t lim = (int64_t)1 << 21;
    if (M < 0 || V <= 0 || K <= 0 || M > lim || V > lim || K > lim) return PURO_ERR_SHAPE;
    // the logits' grid: a launch holds fewer than 2^32 threads, 2^24 tiles of 256 x 256
    if (M * V > (int64_t)1 << 39) return PURO_ERR_SHAPE;
    if (topk < 1 || topk > kDistillMaxTop) return PURO_ERR_SHAPE;
    if ((K % 8) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

puro_status check_distill(const uint16_t* X, const uint16_t* W, const int32_t* ids, const float* teacher, int64_t M,
                          int64_t V, int64_t K, int64_t topk, puro_distill_target target, float tau, DistillArgs* a) {
    const puro_status st = check_distill_sizes(M, V, K, topk);
    if (st != PURO_OK) return st;
    if (target != PURO_DISTILL_LOGITS && target != PURO_DISTILL_PROBS) return PURO_ERR_UNSUPPORTED;
    const float least = 1.17549435e-38f, most = 1.0f / least;
    if (!(tau >= least) || !(tau <= most)) return PURO_ERR_UNSUPPORTED;
    if (M > 0) {
        if (!X || !W || !ids || !teacher) return PURO_ERR_NULL;
        if (!aligned16(X) || !aligned16(W) || !aligned4(ids) || !aligned4(teacher)) return PURO_ERR_ALIGN;
    }
    *a = DistillArgs{X, W, ids, teacher, M, V, K, topk, target == PURO_DISTILL_PROBS, tau};
    return PURO_OK;
}

}  // namespace

extern "C" {

size_t puro_lm_head_distill_workspace_size(int64_t M, int64_t V, int64_t K, int64_t topk, int backward) {
    if (check_distill_sizes(M, V, K, topk) != PURO_OK || M == 0) return 0;
    return lm_distill_ws_bytes(M, V, K, topk, backward != 0);
}

puro_status puro_lm_head_distill_fwd(const uint16_t* X, const uint16_t* W, const int32_t* ids, const float* teacher,
                                     int64_t M, int64_t V, int64_t K, int64_t topk, puro_distill_target target,
                                     float temperature, float* lse, float* loss, float* z_top, void* ws,
                                     size_t ws_bytes, hipStream_t stream) {
    DistillArgs a;
    const puro_status st = check_distill(X, W, ids, teacher, M, V, K, topk, target, temperature, &a);
    if (st != PURO_OK) return st;
    if (M == 0) return PURO_OK;
    if (!lse || !loss || !z_top || !ws) return PURO_ERR_NULL;
    if (!aligned4(lse) || !aligned4(loss) || !aligned4(z_top) || !aligned16(ws)) return PURO_ERR_ALIGN;
    if (ws_bytes < lm_distill_ws_bytes(M, V, K, topk, false)) return PURO_ERR_WORKSPACE;
    launch_lm_distill_fwd(a, lse, loss, z_top, ws, stream);
    return launched();
}

puro_status puro_lm_head_distill_bwd(const uint16_t* X, const uint16_t* W, const int32_t* ids, const float* teacher,
                                     const float* lse, const float* z_top, int64_t M, int64_t V, int64_t K,
                                     int64_t topk, puro_distill_target target, float temperature,
                                     const float* dloss, float grad_scale, uint16_t* dX, void* dW,
                                     puro_out_dtype dw_type, int accumulate_dW, void* ws, size_t ws_bytes,
                                     hipStream_t stream) {
    DistillArgs a;
    const puro_status st = check_distill(X, W, ids, teacher, M, V, K, topk, target, temperature, &a);
    if (st != PURO_OK) return st;
    // (an infinite factor times a dloss of 0 would be NaN)
    const float factor = grad_scale / temperature;
    if (!(factor >= -3.4028235e38f) || !(factor <= 3.4028235e38f)) return PURO_ERR_UNSUPPORTED;
    if (!(grad_scale >= -3.4028235e38f) || !(grad_scale <= 3.4028235e38f)) return PURO_ERR_UNSUPPORTED;
    if (dw_type != PURO_OUT_BF16 && dw_type != PURO_OUT_FP32) return PURO_ERR_UNSUPPORTED;
    if (dW && accumulate_dW && dw_type != PURO_OUT_FP32) return PURO_ERR_UNSUPPORTED;
    if ((dX && !aligned16(dX)) || (dW && !aligned16(dW))) return PURO_ERR_ALIGN;
    if (M == 0) {
        // sums of nothing
        if (!dW || accumulate_dW) return PURO_OK;
        launch_zero(dW, V * K * (dw_type == PURO_OUT_FP32 ? 4 : 2), stream);
        return launched();
    }
    if (!lse || !z_top || !ws) return PURO_ERR_NULL;
    if (!aligned4(lse) || !aligned4(z_top) || !aligned4(dloss) || !aligned16(ws)) return PURO_ERR_ALIGN;
    if (ws_bytes < lm_distill_ws_bytes(M, V, K, topk, true)) return PURO_ERR_WORKSPACE;
    if (!dX && !dW) return PURO_OK;
    launch_lm_distill_bwd(a, lse, z_top, dloss, grad_scale, dX, dW, dw_type == PURO_OUT_BF16, accumulate_dW != 0, ws, stream);
    return launched();
}

}  // extern "C"

// --------------------------------------------- 8-bit integer linear layers
namespace {

// The int32 sums of a product are exact: 2^14 K < 2^31 (codes of -128 too).
constexpr int64_t kMaxInt8K = 131056;

// x [rows, width] and its int8 copy's columns, as the quantisers take them.
puro_status check_int8_source(const uint16_t* x, int64_t rows, int64_t cols, int64_t width, int64_t ld) {
    if (cols < 0 || cols > ((int64_t)1 << 30)) return PURO_ERR_SHAPE;
    const puro_status st = check_bf16_matrix(x, rows, width, ld);
    if (st != PURO_OK) return st;
    if ((cols % 16) != 0) return PURO_ERR_ALIGN;
    return ld < ((int64_t)1 << 23) ? PURO_OK : PURO_ERR_SHAPE;
}

// The rows' codes and scales.
puro_status check_int8_rows(const int8_t* q, const float* scale) {
    if (!q || !scale) return PURO_ERR_NULL;
    return aligned16(q) && ((uintptr_t)scale & 3) == 0 ? PURO_OK : PURO_ERR_ALIGN;
}

}  // namespace

extern "C" {

size_t puro_quantize_int8_workspace_size(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0 || rows > (int64_t)65535 * kGroup || cols > ((int64_t)1 << 23)) return 0;
    return quant_int8_ws_bytes(rows, cols);
}

puro_status puro_quantize_int8(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, int8_t* q, float* scale,
                               int8_t* qT, int64_t ld_qT, float* scaleT, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
    puro_status st = check_int8_source(x, rows, cols, cols, ld);
    if (st != PURO_OK) return st;
    if (qT && (ld_qT < rows || ld_qT > kMaxPitch)) return PURO_ERR_SHAPE;
    if (qT && ((ld_qT % 16) != 0 || !aligned16(qT) || ((uintptr_t)scaleT & 3) != 0)) return PURO_ERR_ALIGN;
    if (rows == 0 || cols == 0) return PURO_OK;
    if (!q && !qT) return PURO_ERR_NULL;
    if (q && (st = check_int8_rows(q, scale)) != PURO_OK) return st;
    if (qT) {
        if (!scaleT || !ws) return PURO_ERR_NULL;
        if (!aligned16(ws)) return PURO_ERR_ALIGN;
        if (ws_bytes < quant_int8_ws_bytes(rows, cols)) return PURO_ERR_WORKSPACE;
    }
    const QuantInt8Args a{x, rows, cols, ld, q, scale, nullptr, 0.0f, nullptr, 0};
    if (qT) launch_quantize_int8_both(a, qT, ld_qT, scaleT, ws, stream);
    else launch_quantize_int8(a, stream);
    return launched();
}

puro_status puro_rmsnorm_quantize_int8(const uint16_t* x, const uint16_t* gamma, int64_t rows, int64_t cols,
                                       int64_t ld, float eps, int8_t* q, float* scale, float* rstd,
                                       hipStream_t stream) {
    puro_status st = check_int8_source(x, rows, cols, cols, ld);
    if (st != PURO_OK) return st;
    if (!finite_nonneg(eps)) return PURO_ERR_UNSUPPORTED;
    if (rows == 0) return PURO_OK;
    if (cols == 0) return PURO_ERR_SHAPE;      // (the mean of an empty row is undefined)
    if (!gamma) return PURO_ERR_NULL;
    if (!aligned16(gamma) || ((uintptr_t)rstd & 3) != 0) return PURO_ERR_ALIGN;
    if ((st = check_int8_rows(q, scale)) != PURO_OK) return st;
    launch_quantize_int8(QuantInt8Args{x, rows, cols, ld, q, scale, gamma, eps, rstd, 0}, stream);
    return launched();
}

puro_status puro_swiglu_quantize_int8(const uint16_t* gu, int64_t rows, int64_t cols, int64_t ld, int8_t* q,
                                      float* scale, hipStream_t stream) {
    if (cols > ((int64_t)1 << 30)) return PURO_ERR_SHAPE;
    puro_status st = check_int8_source(gu, rows, cols, cols < 0 ? cols : 2 * cols, ld);
    if (st != PURO_OK) return st;
    if (rows == 0 || cols == 0) return PURO_OK;
    if ((st = check_int8_rows(q, scale)) != PURO_OK) return st;
    launch_quantize_int8(QuantInt8Args{gu, rows, cols, ld, q, scale, nullptr, 0.0f, nullptr, 1}, stream);
    return launched();
}

size_t puro_int8_gemm_workspace_size(int64_t M, int64_t N, int64_t K) {
    if (M <= 0 || N <= 0 || K <= 0 || M > kMaxPitch || N > kMaxPitch || K > kMaxInt8K) return 0;
    return int8_gemm_ws_bytes(M, N, K);
}

puro_status puro_int8_gemm(int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda, const float* a_scale,
                           const int8_t* B, int64_t ldb, const float* b_scale, void* D, puro_out_dtype d_type,
                           int64_t ldd, int accumulate, const uint16_t* bias, const uint16_t* residual, int64_t ldr,
                           void* ws, size_t ws_bytes, hipStream_t stream) {
    if (M < 0 || N < 0 || K < 0 || M > kMaxPitch || N > kMaxPitch || K > kMaxInt8K) return PURO_ERR_SHAPE;
    // (a launch holds fewer than 2^32 threads: 2^22 tiles of 128 x 128 with 512)
    if (M * N > (int64_t)1 << 36) return PURO_ERR_SHAPE;
    if (d_type != PURO_OUT_BF16 && d_type != PURO_OUT_FP32) return PURO_ERR_UNSUPPORTED;
    const bool f32 = d_type == PURO_OUT_FP32;
    if ((accumulate && !f32) || ((bias || residual) && f32)) return PURO_ERR_UNSUPPORTED;
    if ((K % 16) != 0 || (lda % 16) != 0 || (ldb % 16) != 0 || (ldd % 4) != 0) return PURO_ERR_ALIGN;
    if (lda < K || ldb < K || lda > kMaxPitch || ldb > kMaxPitch || ldd < N) return PURO_ERR_SHAPE;
    if (residual && (ldr < N || ldr > kMaxPitch)) return PURO_ERR_SHAPE;
    if (residual && (ldr % 4) != 0) return PURO_ERR_ALIGN;
    if (M == 0 || N == 0) return PURO_OK;
    if (!a_scale || !b_scale || !D || (K > 0 && (!A || !B))) return PURO_ERR_NULL;
    if (!aligned16(A) || !aligned16(B) || !aligned16(a_scale) || !aligned16(b_scale) || !aligned16(D) || !aligned16(bias) ||
        !aligned16(residual))
        return PURO_ERR_ALIGN;
    if (residual == D && residual && ldr != ldd) return PURO_ERR_SHAPE;
    if (residual && residual != D) {
        const uintptr_t r0 = (uintptr_t)residual, r1 = r0 + (uintptr_t)(((M - 1) * ldr + N) * 2);
        const uintptr_t d0 = (uintptr_t)D, d1 = d0 + (uintptr_t)(((M - 1) * ldd + N) * 2);
        if (r0 < d1 && d0 < r1) return PURO_ERR_SHAPE;
    }
    const size_t need = int8_gemm_ws_bytes(M, N, K);
    if (need > 0) {
        if (!ws) return PURO_ERR_NULL;
        if (!aligned16(ws)) return PURO_ERR_ALIGN;
        if (ws_bytes < need) return PURO_ERR_WORKSPACE;
    }
    launch_int8_gemm(Int8Problem{M, N, K, A, B, lda, ldb, a_scale, b_scale, D, ldd, f32, accumulate != 0, bias, residual, ldr},
                     ws, stream);
    return launched();
}

}  // extern "C"

// ------------------------------------------------- the int8 linear layer
namespace {

int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }

puro_status check_int8_linear(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 0 || M > kMaxInt8K || N > kMaxInt8K || K > kMaxInt8K) return PURO_ERR_SHAPE;
    return (N % 16) == 0 && (K % 16) == 0 ? PURO_OK : PURO_ERR_ALIGN;
}

// The workspace of one tensor [rows, cols] quantised for a pass: its codes, scales,
// and (both) the transposed copy and what makes it.
struct Int8Copies {
    size_t q, scale, qT, scaleT, part;
    Int8Copies(Carver& c, int64_t rows, int64_t cols, bool row, bool transposed) : q(0), scale(0), qT(0), scaleT(0), part(0) {
        if (row) {
            q = c.take((size_t)rows * cols);
            scale = c.take((size_t)rows * sizeof(float));
        }
        if (transposed) {
            qT = c.take((size_t)up16(rows) * cols);
            scaleT = c.take((size_t)cols * sizeof(float));
        }
        part = c.take(rows > 0 && cols > 0 ? quant_int8_ws_bytes(rows, cols) : 0);
    }
};

struct Int8FwdLayout {
    Carver c;
    Int8Copies x, w;
    size_t gemm;
    Int8FwdLayout(int64_t M, int64_t N, int64_t K)
        : x(c, M, K, true, false), w(c, N, K, true, false), gemm(c.take(int8_gemm_ws_bytes(M, N, K))) {}
};

struct Int8BwdLayout {
    Carver c;
    Int8Copies dy;
    size_t gemm;
    Int8BwdLayout(int64_t M, int64_t N, int64_t K) : dy(c, M, N, true, true) {
        const size_t a = int8_gemm_ws_bytes(M, K, N), b = int8_gemm_ws_bytes(N, K, up16(M));
        gemm = c.take(a > b ? a : b);
    }
};

// One product D [M, N] of dense operands.
void int8_product(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* sa, const void* B, int64_t ldb,
                  const float* sb, void* D, bool f32, int accumulate, void* ws, hipStream_t stream) {
    if (M == 0 || N == 0) return;
    launch_int8_gemm(Int8Problem{M, N, K, (const int8_t*)A, (const int8_t*)B, lda, ldb, sa, sb, D, N, f32, accumulate, nullptr, nullptr, 0},
                     ws, stream);
}

// The copies of X (for dW) and of W (for dX), each with its scales or not there.
puro_status check_int8_saved(const puro_linear_saved* s) {
    if (!s->xq_t != !s->x_scale || !s->wq_t != !s->w_scale) return PURO_ERR_NULL;
    return aligned16(s->xq_t) && aligned16(s->x_scale) && aligned16(s->wq_t) && aligned16(s->w_scale) ? PURO_OK : PURO_ERR_ALIGN;
}

}  // namespace

extern "C" {

size_t puro_int8_linear_fwd_workspace_size(int64_t M, int64_t N, int64_t K) {
    return check_int8_linear(M, N, K) == PURO_OK ? Int8FwdLayout(M, N, K).c.used : 0;
}

size_t puro_int8_linear_bwd_workspace_size(int64_t M, int64_t N, int64_t K) {
    return check_int8_linear(M, N, K) == PURO_OK ? Int8BwdLayout(M, N, K).c.used : 0;
}

puro_status puro_int8_linear_fwd(const uint16_t* X, const uint16_t* W, int64_t M, int64_t N, int64_t K, uint16_t* Y,
                                 const puro_linear_saved* saved, void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_int8_linear(M, N, K);
    if (st != PURO_OK) return st;
    const Int8FwdLayout l(M, N, K);
    if (l.c.used > 0 && !ws) return PURO_ERR_NULL;
    if ((M > 0 && K > 0 && !X) || (N > 0 && K > 0 && !W) || (M > 0 && N > 0 && !Y)) return PURO_ERR_NULL;
    if (saved && K > 0 && M > 0 && N > 0 && (st = check_int8_saved(saved)) != PURO_OK) return st;
    if (!aligned16(X) || !aligned16(W) || !aligned16(Y) || !aligned16(ws)) return PURO_ERR_ALIGN;
    if (ws_bytes < l.c.used) return PURO_ERR_WORKSPACE;
    uint8_t* w = reinterpret_cast<uint8_t*>(ws);
    auto rows_of = [&](const uint16_t* x, int64_t rows, const Int8Copies& at) {
        return QuantInt8Args{x, rows, K, K, (int8_t*)(w + at.q), (float*)(w + at.scale), nullptr, 0.0f, nullptr, 0};
    };
    if (M == 0 || N == 0) return PURO_OK;          // (the backward reads nothing of what is saved then)
    if (K == 0) {                                  // (sums of nothing: there are no scales to multiply them by)
        launch_zero(Y, M * N * 2, stream);
        return launched();
    }
    const QuantInt8Args x = rows_of(X, M, l.x), v = rows_of(W, N, l.w);
    auto quantize = [&](const QuantInt8Args& a, void* qT, float* scaleT, size_t part) {
        if (qT) launch_quantize_int8_both(a, (int8_t*)qT, up16(a.rows), scaleT, w + part, stream);
        else launch_quantize_int8(a, stream);
    };
    if (!saved || (!saved->xq_t && !saved->wq_t)) {
        launch_quantize_int8_two(x, v, stream);
    } else {
        quantize(x, saved->xq_t, saved->x_scale, l.x.part);
        quantize(v, saved->wq_t, saved->w_scale, l.w.part);
    }
    int8_product(M, N, K, w + l.x.q, K, (float*)(w + l.x.scale), w + l.w.q, K, (float*)(w + l.w.scale), Y, false, 0, w + l.gemm, stream);
    return launched();
}

puro_status puro_int8_linear_bwd(const uint16_t* dY, const puro_linear_saved* saved, int64_t M, int64_t N, int64_t K,
                                 uint16_t* dX, float* dW, int accumulate_dW, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
    puro_status st = check_int8_linear(M, N, K);
    if (st != PURO_OK) return st;
    if (!aligned16(dY) || !aligned16(dX) || !aligned16(dW) || !aligned16(ws)) return PURO_ERR_ALIGN;
    if (K == 0 || N == 0) {
        // (dX is a sum over no channels)
        if (!dX || M == 0 || K == 0) return PURO_OK;
        launch_zero(dX, M * K * 2, stream);
        return launched();
    }
    if (M == 0) {
        if (!dW || accumulate_dW) return PURO_OK;
        launch_zero(dW, N * K * 4, stream);
        return launched();
    }
    const Int8BwdLayout l(M, N, K);
    if (!dY || !saved || !ws) return PURO_ERR_NULL;
    if ((st = check_int8_saved(saved)) != PURO_OK) return st;
    if ((dX && !saved->wq_t) || (dW && !saved->xq_t)) return PURO_ERR_NULL;
    if (ws_bytes < l.c.used) return PURO_ERR_WORKSPACE;
    if (!dX && !dW) return PURO_OK;
    uint8_t* w = reinterpret_cast<uint8_t*>(ws);
    const QuantInt8Args a{dY, M, N, N, dX ? (int8_t*)(w + l.dy.q) : nullptr, (float*)(w + l.dy.scale), nullptr, 0.0f, nullptr, 0};
    if (dW) launch_quantize_int8_both(a, (int8_t*)(w + l.dy.qT), up16(M), (float*)(w + l.dy.scaleT), w + l.dy.part, stream);
    else launch_quantize_int8(a, stream);
    if (dX) int8_product(M, K, N, w + l.dy.q, N, a.scale, saved->wq_t, N, saved->w_scale, dX, false, 0, w + l.gemm, stream);
    if (dW)
        int8_product(N, K, up16(M), w + l.dy.qT, up16(M), (float*)(w + l.dy.scaleT), saved->xq_t, up16(M), saved->x_scale, dW, true,
                     accumulate_dW != 0, w + l.gemm, stream);
    return launched();
}

}  // extern "C"

// ---------------------------------------- verification of drafted tokens
namespace {

puro_status check_verify_sizes(int64_t B, int64_t T, int64_t draft_rows, int64_t V) {
    if (B < 0 || T < 0 || draft_rows < 0 || V < 1) return PURO_ERR_SHAPE;
    const int64_t rows = (int64_t)1 << 20;
    // (a launch holds fewer than 2^24 blocks of 256 threads, a block at least 4096 entries of a long row)
    if (B > (int64_t)1 << 16 || T > rows || draft_rows > T || V > (int64_t)1 << 21) return PURO_ERR_SHAPE;
    if (T * V > (int64_t)1 << 35 || B * V > (int64_t)1 << 35) return PURO_ERR_SHAPE;
    return PURO_OK;
}

}  // namespace

extern "C" {

size_t puro_verify_drafts_workspace_size(int64_t B, int64_t T, int64_t draft_rows, int64_t V) {
    if (check_verify_sizes(B, T, draft_rows, V) != PURO_OK || B == 0) return 0;
    return verify_ws_bytes(B, T, draft_rows, V);
}

puro_status puro_verify_drafts(int64_t B, int64_t T, int64_t draft_rows, int64_t V, puro_verify_kind kind,
                               puro_out_dtype dtype, const void* target, int64_t ld_target, const void* draft,
                               int64_t ld_draft, const int32_t* draft_ids, const int32_t* offsets,
                               const float* uniform, const float* uniform_sample, double temperature,
                               int32_t* tokens, int32_t* accepted, void* ws, size_t ws_bytes, hipStream_t stream) {
    const puro_status st = check_verify_sizes(B, T, draft_rows, V);
    if (st != PURO_OK) return st;
    if (kind != PURO_VERIFY_LOGITS && kind != PURO_VERIFY_PROBS) return PURO_ERR_UNSUPPORTED;
    if (dtype != PURO_OUT_BF16 && dtype != PURO_OUT_FP32) return PURO_ERR_UNSUPPORTED;
    const bool logits = kind == PURO_VERIFY_LOGITS, greedy = logits && temperature == 0.0;
    if (logits && !greedy && (!(temperature >= 0x1p-20) || !(temperature <= 0x1p20))) return PURO_ERR_UNSUPPORTED;
    const bool drafted = draft && !greedy;
    if (T > 0 && (ld_target < V || ld_target > kMaxPitch)) return PURO_ERR_SHAPE;
    if (drafted && draft_rows > 0 && (ld_draft < V || ld_draft > kMaxPitch)) return PURO_ERR_SHAPE;
    if (B == 0) return PURO_OK;
    if (!offsets || !accepted || !ws) return PURO_ERR_NULL;
    if (T > 0 && (!target || !draft_ids || !tokens || (!greedy && (!uniform || !uniform_sample)))) return PURO_ERR_NULL;
    const uintptr_t e = dtype == PURO_OUT_BF16 ? 1 : 3;
    if (((uintptr_t)target & e) != 0 || (drafted && ((uintptr_t)draft & e) != 0) || !aligned16(ws)) return PURO_ERR_ALIGN;
    for (const void* p : {(const void*)draft_ids, (const void*)offsets, (const void*)uniform, (const void*)uniform_sample,
                          (const void*)tokens, (const void*)accepted})
        if (((uintptr_t)p & 3) != 0) return PURO_ERR_ALIGN;
    if (ws_bytes < verify_ws_bytes(B, T, draft_rows, V)) return PURO_ERR_WORKSPACE;
    // what is written overlaps nothing that is read but, as a whole, the ids
    auto overlap = [](const void* p, int64_t n, const void* q, int64_t m) {
        const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
        return p && q && a < b + (uintptr_t)(4 * m) && b < a + (uintptr_t)(4 * n);
    };
    if ((tokens != draft_ids && overlap(tokens, T, draft_ids, T)) || overlap(tokens, T, offsets, B + 1) || overlap(tokens, T, accepted, B) ||
        overlap(accepted, B, draft_ids, T) || overlap(accepted, B, offsets, B + 1))
        return PURO_ERR_SHAPE;
    launch_verify(VerifyArgs{target, drafted ? draft : nullptr, ld_target, ld_draft, draft_ids, offsets, uniform, uniform_sample,
                             (int)B, (int)T, (int)draft_rows, (int)V, logits, dtype == PURO_OUT_BF16, logits ? temperature : 1.0, tokens,
                             accepted},
                  ws, stream);
    return launched();
}

}  // extern "C"

// ------------------------------------------------------------------- MuonH
namespace {

puro_status check_muonh_shape(int64_t count, int64_t rows, int64_t cols) {
    if (count <= 0 || rows <= 0 || cols <= 0) return PURO_ERR_SHAPE;
    const int64_t lim = (int64_t)1 << 21;
    if (count > 65535 || rows > lim || cols > lim) return PURO_ERR_SHAPE;
    if ((rows % kGroup) != 0 || (cols % kGroup) != 0) return PURO_ERR_ALIGN;
    return PURO_OK;
}

bool finite_f32(float v) { return v == v && v <= 3.4028235e38f && v >= -3.4028235e38f; }

}  // namespace

extern "C" {

size_t puro_muonh_workspace_size(int64_t count, int64_t rows, int64_t cols) {
    if (check_muonh_shape(count, rows, cols) != PURO_OK) return 0;
    return muonh_ws_bytes(count, rows, cols);
}

puro_status puro_muonh_step(int64_t count, int64_t rows, int64_t cols, float* W, uint16_t* w_bf16, const float* G,
                            float* buf, const float* radius, float mu, int nesterov, float eta, int ns_steps,
                            uint16_t* u_out, void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_muonh_shape(count, rows, cols);
    if (st != PURO_OK) return st;
    if (!W || !G || !buf || !radius || !ws) return PURO_ERR_NULL;
    if (!aligned16(W) || !aligned16(G) || !aligned16(buf) || ((uintptr_t)radius & 3) != 0 ||
        (w_bf16 && !aligned16(w_bf16)) || (u_out && !aligned16(u_out)))
        return PURO_ERR_ALIGN;
    if (!finite_f32(mu) || !finite_f32(eta) || ns_steps < 0 || ns_steps > 64) return PURO_ERR_UNSUPPORTED;
    if (ws_bytes < muonh_ws_bytes(count, rows, cols)) return PURO_ERR_WORKSPACE;
    launch_muonh_step(count, rows, cols, W, w_bf16, G, buf, radius, mu, nesterov != 0, eta, ns_steps, u_out, ws,
                      stream);
    return launched();
}

size_t puro_newton_schulz_workspace_size(int64_t count, int64_t r, int64_t c) {
    if (check_muonh_shape(count, r, c) != PURO_OK || r > c) return 0;
    return newton_schulz_ws_bytes(count, r, c);
}

puro_status puro_newton_schulz_bf16(int64_t count, int64_t r, int64_t c, const uint16_t* X, int steps,
                                    uint16_t* out, void* ws, size_t ws_bytes, hipStream_t stream) {
    puro_status st = check_muonh_shape(count, r, c);
    if (st != PURO_OK) return st;
    if (r > c) return PURO_ERR_SHAPE;
    if (!X || !out || !ws) return PURO_ERR_NULL;
    if (!aligned16(X) || !aligned16(out)) return PURO_ERR_ALIGN;
    if (steps < 0 || steps > 64) return PURO_ERR_UNSUPPORTED;
    if (ws_bytes < newton_schulz_ws_bytes(count, r, c)) return PURO_ERR_WORKSPACE;
    launch_newton_schulz(X, count, r, c, steps, out, ws, stream);
    return launched();
}

}  // extern "C"
