// Verification of drafted tokens for gfx950: which drafts of a sequence are kept,
// and the token drawn from what the target's probabilities leave over.
//
// With p, q the target's and the draft's probabilities of a row, draft d is kept
// with probability min(1, p(d) / q(d)), and the first that is not is replaced by a
// draw from max(p - q, 0) / sum max(p - q, 0): the kept or drawn token is then
// distributed as p.
//
// A vocabulary row is worked on by blocks of a chunk each; every sum over a row is
// one of its chunks' sums, in order, so that all blocks see the same values.
//  * LOGITS: the chunks' largest logits and sums of exponentials of every row;
//  * every sequence's chunks of the row where its drafts end: the block finds that
//    row (each draft's probability from the rows' sums), and sums what is left over;
//  * one block per sequence: the chunk, then the entry where the running sum passes
//    the random number's share.
// Exponentials, probabilities and sums are binary64: with 10^5 entries a running
// sum that errs by 10^-8 moves the drawn token once in 10^3 draws.

#include <algorithm>
#include <cmath>

#include "device_common.h"
#include "kernels.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;       // entries per block
constexpr double kInf = __builtin_huge_val();

// Values of a row: four consecutive words, of any alignment that the elements have.
__device__ __forceinline__ float value(const uint16_t* p, int64_t v) { return __uint_as_float((uint32_t)p[v] << 16); }
__device__ __forceinline__ float value(const float* p, int64_t v) { return p[v]; }

__device__ __forceinline__ double shfl_xor(double v, int o) { return __shfl_xor(v, o, 64); }

// Sums over a block in a fixed order, in every thread.
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// The larger of two values, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

struct Args : VerifyArgs {
    int chunks;
    double c;             // log2(e) / temperature
    double2* stats;       // [T + draft_rows][chunks]: largest logit (greedy: and its id), sum of exponentials
    double2* left;        // [B][chunks]: sums of max(p - q, 0) and of p
    double4* row;         // [B]: the row's largest logits and reciprocal sums, target and draft
    int* kept;            // [B]: drafts kept (-1: invalid)
};

// Rows of sequence b: its first, and how many (0: none; -1: invalid).
struct Rows {
    int start, n;
};
__device__ __forceinline__ Rows rows_of(const Args& a, int b) {
    const int64_t start = a.offsets[b], end = a.offsets[b + 1];
    if (start < 0 || end < start || end > a.T) return {0, -1};
    const int n = (int)(end - start);
    // its draft rows: start - b .. end - 2 - b
    if (a.draft && n > 1 && (start - b < 0 || end - 1 - b > a.draft_rows)) return {0, -1};
    return {(int)start, n};
}

// ---- LOGITS: (largest, sum of 2^((z - largest) c)) of every chunk of every row.
template <typename E>
__global__ __launch_bounds__(kThreads) void chunk_sums_kernel(Args a) {
    __shared__ double red[4];
    __shared__ float redm[4];
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks), r = (int)(blockIdx.x / (unsigned)a.chunks);
    const E* z = r < a.T ? (const E*)a.target + (int64_t)r * a.ld_t : (const E*)a.draft + (int64_t)(r - a.T) * a.ld_d;
    const int v0 = chunk * kChunk, v1 = min(a.V, v0 + kChunk);
    float m = -INFINITY;
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads) m = max_nan(m, value(z, v));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max_nan(m, __shfl_xor(m, o, 64));
    if ((threadIdx.x & 63) == 0) redm[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max_nan(max_nan(redm[0], redm[1]), max_nan(redm[2], redm[3]));
    double s = 0.0;
    if (m != -INFINITY)
        for (int v = v0 + threadIdx.x; v < v1; v += kThreads) s += exp2(((double)value(z, v) - (double)m) * a.c);
    s = block_sum(s, red);
    if (threadIdx.x == 0) a.stats[(int64_t)r * a.chunks + chunk] = make_double2((double)m, s);
}

// A row's largest logit and the reciprocal of its sum, by one wave.
__device__ __forceinline__ double2 row_norm(const Args& a, int64_t r) {
    const double2* st = a.stats + r * a.chunks;
    const int lane = threadIdx.x & 63;
    double m = -kInf;
    for (int c = lane; c < a.chunks; c += 64) m = st[c].x > m || st[c].x != st[c].x ? st[c].x : m;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const double t = shfl_xor(m, o);
        m = t > m || t != t ? t : m;
    }
    double s = 0.0;
    for (int c = lane; c < a.chunks; c += 64) {
        const double2 v = st[c];
        if (v.y != 0.0) s += v.y * exp2((v.x - m) * a.c);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += shfl_xor(s, o);
    return make_double2(m, 1.0 / s);
}

// The probability of a row's value x.
__device__ __forceinline__ double prob(const Args& a, float x, double m, double inv) {
    return a.logits ? exp2(((double)x - m) * a.c) * inv : (double)x;
}

// Drafts kept of a sequence's n rows, by the whole block: four at a time.
template <typename E>
__device__ __forceinline__ int kept_drafts(const Args& a, int b, Rows rows, int* ok) {
    const int wave = threadIdx.x >> 6;
    for (int i0 = 0; i0 < rows.n - 1; i0 += 4) {
        const int i = i0 + wave;
        bool keep = false;
        if (i < rows.n - 1) {
            const int64_t t = rows.start + i;
            const int d = a.ids[t];
            if (d >= 0 && d < a.V) {
                double2 np = make_double2(0.0, 0.0), nq = np;
                if (a.logits) np = row_norm(a, t);
                const double p = prob(a, value((const E*)a.target + t * a.ld_t, d), np.x, np.y);
                double q = 1.0;
                if (a.draft) {
                    if (a.logits) nq = row_norm(a, a.T + t - b);
                    q = prob(a, value((const E*)a.draft + (t - b) * a.ld_d, d), nq.x, nq.y);
                }
                keep = (double)a.u[t] * q < p;
            }
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) ok[wave] = keep;
        __syncthreads();
        for (int w = 0; w < 4; ++w)
            if (!ok[w]) return min(i0 + w, rows.n - 1);
    }
    return max(rows.n - 1, 0);
}

// What is left over of entry v: (max(p - q, 0), p), NaN where p or q is.
template <typename E>
__device__ __forceinline__ double2 left_over(const Args& a, const E* zp, const E* zq, int onehot, const double4& n, int v) {
    const double p = prob(a, value(zp, v), n.x, n.y);
    double q = v == onehot ? 1.0 : 0.0;
    if (zq) q = prob(a, value(zq, v), n.z, n.w);
    const double d = p - q;
    return make_double2(d <= 0.0 ? 0.0 : d, p);
}

// The row where a sequence's drafts end: its values, the draft's (or the id that
// stands for them) unless it is the last one.
template <typename E>
struct EndRow {
    const E *zp, *zq;
    int onehot;
};
template <typename E>
__device__ __forceinline__ EndRow<E> end_row(const Args& a, int b, Rows rows, int kept) {
    const int64_t t = rows.start + kept;
    EndRow<E> r{(const E*)a.target + t * a.ld_t, nullptr, -1};
    if (kept < rows.n - 1) {
        if (a.draft) r.zq = (const E*)a.draft + (t - b) * a.ld_d;
        else r.onehot = a.ids[t];
    }
    return r;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void left_over_kernel(Args a) {
    __shared__ double red[4];
    __shared__ double2 norms[2];
    __shared__ int ok[4];
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks), b = (int)(blockIdx.x / (unsigned)a.chunks);
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) {
        if (chunk == 0 && threadIdx.x == 0) a.kept[b] = rows.n;
        return;
    }
    const int kept = kept_drafts<E>(a, b, rows, ok);
    const EndRow<E> e = end_row<E>(a, b, rows, kept);
    double4 n = make_double4(0.0, 1.0, 0.0, 1.0);
    if (a.logits) {
        const int wave = threadIdx.x >> 6;
        const int64_t t = rows.start + kept;
        if (wave == 0) norms[0] = row_norm(a, t);
        if (wave == 1) norms[1] = e.zq ? row_norm(a, a.T + t - b) : make_double2(0.0, 0.0);
        __syncthreads();
        n = make_double4(norms[0].x, norms[0].y, norms[1].x, norms[1].y);
    }
    if (chunk == 0 && threadIdx.x == 0) {
        a.kept[b] = kept;
        a.row[b] = n;
    }
    const int v0 = chunk * kChunk, v1 = min(a.V, v0 + kChunk);
    double r = 0.0, p = 0.0;
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads) {
        const double2 l = left_over(a, e.zp, e.zq, e.onehot, n, v);
        r += l.x;
        p += l.y;
    }
    r = block_sum(r, red);
    p = block_sum(p, red);
    if (threadIdx.x == 0) a.left[(int64_t)b * a.chunks + chunk] = make_double2(r, p);
}

__device__ __forceinline__ void write_tokens(const Args& a, int b, Rows rows, int kept, int token) {
    for (int i = threadIdx.x; i < rows.n; i += kThreads)
        a.tokens[rows.start + i] = i < kept ? a.ids[rows.start + i] : i == kept ? token : -1;
    if (threadIdx.x == 0) a.accepted[b] = kept;
}

template <typename E>
__global__ __launch_bounds__(kThreads) void draw_kernel(Args a) {
    __shared__ double sum[kThreads];
    __shared__ int found;
    const int b = blockIdx.x;
    const int kept = a.kept[b];
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    // totals, and the chunk in which the running sum passes the target
    const double2* left = a.left + (int64_t)b * a.chunks;
    double rt = 0.0, pt = 0.0;
    for (int c = 0; c < a.chunks; ++c) {
        rt += left[c].x;
        pt += left[c].y;
    }
    const bool use_p = !(rt > 0.0);
    const double total = use_p ? pt : rt;
    if (!(pt > 0.0 && pt < kInf && rt >= 0.0)) {
        write_tokens(a, b, rows, kept, -1);
        return;
    }
    const double goal = (double)a.us[b] * total;
    int chunk = -1, last = 0;
    double before = 0.0, run = 0.0, last_before = 0.0;
    for (int c = 0; c < a.chunks; ++c) {
        const double s = use_p ? left[c].y : left[c].x;
        if (s > 0.0) {
            last = c;
            last_before = run;
        }
        if (chunk < 0 && run + s > goal) {
            chunk = c;
            before = run;
        }
        run += s;
    }
    if (chunk < 0) {
        chunk = last;
        before = last_before;
    }
    // within the chunk: each thread a run of entries
    const EndRow<E> e = end_row<E>(a, b, rows, kept);
    const double4 n = a.row[b];
    constexpr int PER = kChunk / kThreads;
    const int v0 = chunk * kChunk + threadIdx.x * PER, v1 = min(a.V, v0 + PER);
    double s = 0.0;
    for (int v = v0; v < v1; ++v) {
        const double2 l = left_over(a, e.zp, e.zq, e.onehot, n, v);
        s += use_p ? l.y : l.x;
    }
    sum[threadIdx.x] = s;
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    if (threadIdx.x == 0) {
        double at = before;
        int lastt = 0;
        double last_at = before;
        for (int i = 0; i < kThreads; ++i) {
            if (sum[i] > 0.0) {
                lastt = i;
                last_at = at;
            }
            if (at + sum[i] > goal) {
                lastt = i;
                last_at = at;
                break;
            }
            at += sum[i];
        }
        found = lastt;
        sum[0] = last_at;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const int f0 = chunk * kChunk + found * PER, f1 = min(a.V, f0 + PER);
        double at = sum[0];
        int token = -1;
        for (int v = f0; v < f1; ++v) {
            const double2 l = left_over(a, e.zp, e.zq, e.onehot, n, v);
            const double x = use_p ? l.y : l.x;
            at += x;
            if (x > 0.0) token = v;
            if (at > goal) break;
        }
        found = token;
    }
    __syncthreads();
    write_tokens(a, b, rows, kept, found);
}

// ---- temperature 0: (largest logit, its lowest id) of every chunk of the target's rows.
template <typename E>
__global__ __launch_bounds__(kThreads) void chunk_max_kernel(Args a) {
    __shared__ float redm[4];
    __shared__ int redi[4];
    const int chunk = (int)(blockIdx.x % (unsigned)a.chunks), r = (int)(blockIdx.x / (unsigned)a.chunks);
    const E* z = (const E*)a.target + (int64_t)r * a.ld_t;
    const int v0 = chunk * kChunk, v1 = min(a.V, v0 + kChunk);
    float m = -INFINITY;
    int at = a.V;
    auto take = [&](float x, int v) {
        if (x > m || (x == m && v < at) || (x != x && m == m)) { m = x; at = v; }
    };
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads) take(value(z, v), v);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const float x = __shfl_xor(m, o, 64);
        const int v = __shfl_xor(at, o, 64);
        take(x, v);
    }
    if ((threadIdx.x & 63) == 0) { redm[threadIdx.x >> 6] = m; redi[threadIdx.x >> 6] = at; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) take(redm[w], redi[w]);
        a.stats[(int64_t)r * a.chunks + chunk] = make_double2((double)m, (double)at);
    }
}

// A row's choice, -1 where it has none (NaN, +infinity or nothing but -infinity).
__device__ __forceinline__ int row_choice(const Args& a, int64_t r) {
    const double2* st = a.stats + r * a.chunks;
    double m = -kInf;
    int at = -1;
    for (int c = 0; c < a.chunks; ++c) {
        if (st[c].x != st[c].x || st[c].x == kInf) return -1;
        if (st[c].x > m) { m = st[c].x; at = (int)st[c].y; }
    }
    return at;
}

__global__ __launch_bounds__(kThreads) void greedy_kernel(Args a) {
    __shared__ int first;
    const int b = blockIdx.x;
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    if (threadIdx.x == 0) first = rows.n - 1;
    __syncthreads();
    for (int i = threadIdx.x; i < rows.n - 1; i += kThreads) {
        const int c = row_choice(a, rows.start + i);
        if (c < 0 || c != a.ids[rows.start + i]) {
            atomicMin(&first, i);      // (the least of integers: the same in any order)
            break;
        }
    }
    __syncthreads();
    const int kept = first;
    write_tokens(a, b, rows, kept, row_choice(a, rows.start + kept));
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
    int chunks;
    size_t stats, left, row, kept, total;
};
Layout layout(int64_t B, int64_t T, int64_t draft_rows, int64_t V) {
    Layout l{};
    l.chunks = (int)((V + kChunk - 1) / kChunk);
    l.left = up((size_t)(T + draft_rows) * l.chunks * sizeof(double2));
    l.row = l.left + up((size_t)B * l.chunks * sizeof(double2));
    l.kept = l.row + up((size_t)B * sizeof(double4));
    l.total = l.kept + up((size_t)B * sizeof(int));
    return l;
}

template <typename E>
void launch(const Args& a, hipStream_t stream) {
    if (a.temperature == 0.0) {
        if (a.T > 0) chunk_max_kernel<E><<<(unsigned)a.T * a.chunks, kThreads, 0, stream>>>(a);
        greedy_kernel<<<a.B, kThreads, 0, stream>>>(a);
        return;
    }
    const unsigned rows = (unsigned)(a.T + (a.draft ? a.draft_rows : 0));
    if (a.logits && rows > 0) chunk_sums_kernel<E><<<rows * a.chunks, kThreads, 0, stream>>>(a);
    left_over_kernel<E><<<(unsigned)a.B * a.chunks, kThreads, 0, stream>>>(a);
    draw_kernel<E><<<a.B, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t verify_ws_bytes(int64_t B, int64_t T, int64_t draft_rows, int64_t V) { return layout(B, T, draft_rows, V).total; }

void launch_verify(const VerifyArgs& v, void* ws, hipStream_t stream) {
    const Layout l = layout(v.B, v.T, v.draft_rows, v.V);
    uint8_t* w = reinterpret_cast<uint8_t*>(ws);
    Args a;
    static_cast<VerifyArgs&>(a) = v;
    a.chunks = l.chunks;
    a.c = v.temperature == 0.0 ? 0.0 : 1.4426950408889634 / v.temperature;
    a.stats = reinterpret_cast<double2*>(w);
    a.left = reinterpret_cast<double2*>(w + l.left);
    a.row = reinterpret_cast<double4*>(w + l.row);
    a.kept = reinterpret_cast<int*>(w + l.kept);
    if (v.bf16) launch<uint16_t>(a, stream);
    else launch<float>(a, stream);
}

}  // namespace puro
