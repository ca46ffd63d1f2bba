// Verification of drafted tokens for gfx950: which drafts of a sequence are kept,
// and the token drawn from what the target's probabilities leave over.
//
// With p, q the target's and the draft's probabilities of a row, draft d is kept
// with probability min(1, p(d) / q(d)), and the first that is not is replaced by a
// draw from max(p - q, 0) / sum max(p - q, 0): the kept or drawn token is then
// distributed as p.
//
// A vocabulary row is worked on in pieces of 2048 entries, a wave each; every sum
// over a row is made of its pieces' sums, in a fixed order.
//  * LOGITS: of every row the pieces' largest logits and sums of exponentials, then
//    of every sequence, by a block of 16 waves (a row each), the row where its
//    drafts end and that row's sums. PROBS: the drafts' entries alone say that row;
//  * the pieces of that row: what is left over of each, and of p;
//  * a block per sequence: the piece, then the entry where the running sum passes
//    the random number's share.
// Exponentials, probabilities and sums are binary64: with 10^5 entries a running
// sum that errs by 10^-8 moves the drawn token once in 10^3 draws.

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kPiece = 2048;       // entries per wave
constexpr double kInf = __builtin_huge_val();

struct Args : VerifyArgs {
    int pieces;           // of a row
    double c;             // log2(e) / temperature
    double2* stats;       // [T + draft_rows][pieces]: largest logit; sum of 2^((z - largest) c) (greedy: its id)
    double2* left;        // [B][pieces]: sums of max(p - q, 0) and of p
    double4* row;         // [B]: the end row's largest logits and reciprocal sums, target and draft
    int* kept;            // [B]: drafts kept
};

// ---- values of a row ---------------------------------------------------------

__device__ __forceinline__ float value(const uint16_t* p, int64_t v) { return __uint_as_float((uint32_t)p[v] << 16); }
__device__ __forceinline__ float value(const float* p, int64_t v) { return p[v]; }

// E entries in 16 bytes; a row begins at any element, so that the 16-byte loads are
// of no more than its alignment.
template <typename E> constexpr int kPerVector = 16 / (int)sizeof(E);
__device__ __forceinline__ void unpack(const uint4& w, float x[8], const uint16_t*) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16lo(u[i]); x[2 * i + 1] = bf16hi(u[i]); }
}
__device__ __forceinline__ void unpack(const uint4& w, float x[4], const float*) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}

// The lane's entries of a piece, vector i at v0 + (i 64 + lane) * kPerVector, `fill`
// past the row's end.
template <typename E>
struct Piece {
    static constexpr int N = kPiece / 64 / kPerVector<E>;
    float x[N][kPerVector<E>];
    __device__ __forceinline__ static int at(int v0, int i) { return v0 + (i * 64 + (threadIdx.x & 63)) * kPerVector<E>; }
    __device__ __forceinline__ void load(const E* row, int v0, int V, float fill) {
        if (v0 + kPiece <= V) {
            uint4 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) __builtin_memcpy(&w[i], row + at(v0, i), 16);
#pragma unroll
            for (int i = 0; i < N; ++i) unpack(w[i], x[i], row);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int v = at(v0, i);
                if (v + kPerVector<E> <= V) {
                    uint4 w;
                    __builtin_memcpy(&w, row + v, 16);
                    unpack(w, x[i], row);
                } else {
#pragma unroll
                    for (int e = 0; e < kPerVector<E>; ++e) x[i][e] = v + e < V ? value(row, v + e) : fill;
                }
            }
        }
    }
};

// ---- arithmetic ----------------------------------------------------------------

// 2^t in binary64 within 2^-45 relative, 0 far below: 2^n by the exponent, n the
// nearest integer, times a polynomial of the rest f in [-1/2, 1/2] (interpolation
// of degree 9 at the Chebyshev nodes, relative error 1.9e-14). t finite or
// -infinity, at most 1000.
__device__ __forceinline__ double exp2_f64(double t) {
    t = fmax(t, -2000.0);
    const double n = __builtin_rint(t), f = t - n;
    double p = 0x1.b6571d9fbc782p-24;
    p = __builtin_fma(p, f, 0x1.63ef9699f65f0p-20);
    p = __builtin_fma(p, f, 0x1.ffcb7678dfe12p-17);
    p = __builtin_fma(p, f, 0x1.43088e257f900p-13);
    p = __builtin_fma(p, f, 0x1.5d87fe908f6f7p-10);
    p = __builtin_fma(p, f, 0x1.3b2ab72b175e9p-7);
    p = __builtin_fma(p, f, 0x1.c6b08d704411ap-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff8149f2p-3);
    p = __builtin_fma(p, f, 0x1.62e42fefa39f7p-1);
    p = __builtin_fma(p, f, 0x1.000000000003dp+0);
    return __builtin_ldexp(p, (int)n);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
// The larger of two values, NaN if either is.
template <typename F>
__device__ __forceinline__ F max_nan(F a, F b) { return a > b || a != a ? a : b; }

// A row's normaliser: its largest logit m and the reciprocal of its sum; not finite
// (then NaN) for a row with a NaN or an infinity, or without any probability.
struct Norm {
    double m, inv;
};
// The probability of a logit x, or x itself.
__device__ __forceinline__ double prob(const Args& a, float x, const Norm& n) {
    return a.logits ? exp2_f64(__builtin_fma((double)x, a.c, -(n.m * a.c))) * n.inv : (double)x;
}
__device__ __forceinline__ bool bad(const Norm& n) { return !(n.inv < kInf); }

// ---- sequences -------------------------------------------------------------------

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
template <typename E>
__device__ __forceinline__ const E* target_row(const Args& a, int64_t t) { return (const E*)a.target + t * a.ld_t; }
template <typename E>
__device__ __forceinline__ const E* draft_row(const Args& a, int64_t t) { return (const E*)a.draft + t * a.ld_d; }

// ---- LOGITS: (largest, sum of 2^((z - largest) c)) of every piece of every row.
// Bound by memory and, as closely, by its arithmetic: some 17 binary64 instructions
// an entry.
template <typename E>
__global__ __launch_bounds__(kThreads) void piece_sums_kernel(Args a, int total) {
    const int at = (int)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (at >= total) return;
    const int r = at / a.pieces, v0 = (at - r * a.pieces) * kPiece;
    const E* z = r < a.T ? target_row<E>(a, r) : draft_row<E>(a, r - a.T);
    Piece<E> x;
    x.load(z, v0, a.V, -INFINITY);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < x.N; ++i)
#pragma unroll
        for (int e = 0; e < kPerVector<E>; ++e) m = max_nan(m, x.x[i][e]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max_nan(m, __shfl_xor(m, o, 64));
    double s = 0.0;
    if (m > -INFINITY && m < INFINITY) {
        const double mc = (double)m * a.c;
#pragma unroll
        for (int i = 0; i < x.N; ++i)
#pragma unroll
            for (int e = 0; e < kPerVector<E>; ++e) s += exp2_f64(__builtin_fma((double)x.x[i][e], a.c, -mc));
        s = wave_sum(s);
    } else if (m != -INFINITY) {
        s = __builtin_nan("");
    }
    if ((threadIdx.x & 63) == 0) a.stats[at] = make_double2((double)m, s);
}

// A row's normaliser from its pieces, by one wave.
__device__ __forceinline__ Norm row_norm(const Args& a, int64_t r) {
    const double2* st = a.stats + r * a.pieces;
    const int lane = threadIdx.x & 63;
    double m = -kInf;
    for (int c = lane; c < a.pieces; c += 64) m = max_nan(m, st[c].x);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max_nan(m, __shfl_xor(m, o, 64));
    if (!(m > -kInf && m < kInf)) return {m, __builtin_nan("")};
    double s = 0.0;
    for (int c = lane; c < a.pieces; c += 64) {
        const double2 v = st[c];
        s += v.y * exp2_f64(__builtin_fma(v.x, a.c, -(m * a.c)));
    }
    return {m, 1.0 / wave_sum(s)};
}

// Where a sequence's drafts end, by a block of 16 waves: eight rows at a time, a
// wave for each one's normaliser and for its draft's.
constexpr int kEndWaves = 16, kEndRows = kEndWaves / 2;
template <typename E>
__global__ __launch_bounds__(kEndWaves * 64) void end_rows_kernel(Args a) {
    __shared__ Norm norms[kEndWaves];
    __shared__ int ok[kEndRows];
    const int b = blockIdx.x, wave = threadIdx.x >> 6;
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) return;
    for (int i0 = 0;; i0 += kEndRows) {
        const int i = i0 + (wave & (kEndRows - 1));
        const int64_t t = rows.start + i;
        const bool drafted = i < rows.n - 1;
        if (wave < kEndRows ? i < rows.n : drafted && a.draft) {
            const Norm n = row_norm(a, wave < kEndRows ? t : a.T + t - b);
            if ((threadIdx.x & 63) == 0) norms[wave] = n;
        }
        __syncthreads();
        if (wave < kEndRows && (threadIdx.x & 63) == 0) {
            bool keep = false;
            const int d = drafted ? a.ids[t] : -1;
            if (d >= 0 && d < a.V && !bad(norms[wave])) {
                const double p = prob(a, value(target_row<E>(a, t), d), norms[wave]);
                const double q = a.draft ? prob(a, value(draft_row<E>(a, t - b), d), norms[wave + kEndRows]) : 1.0;
                keep = (double)a.u[t] * q < p;
            }
            ok[wave] = keep;
        }
        __syncthreads();
        int w = 0;
        while (w < kEndRows && ok[w]) ++w;
        if (w < kEndRows) {              // (the last row is not kept, at the latest)
            if (threadIdx.x == 0) {
                const bool last = i0 + w == rows.n - 1;
                const Norm p = norms[w], q = last || !a.draft ? Norm{0.0, 0.0} : norms[w + kEndRows];
                a.kept[b] = i0 + w;
                a.row[b] = make_double4(p.m, p.inv, q.m, q.inv);
            }
            return;
        }
        __syncthreads();
    }
}

// The same of probabilities, whose entries say it alone: by one wave, 64 drafts at a
// time (every wave of every block that needs it, rather than a launch of its own).
template <typename E>
__device__ __forceinline__ int kept_of_probs(const Args& a, int b, Rows rows) {
    for (int i0 = 0;; i0 += 64) {
        const int i = i0 + (threadIdx.x & 63);
        const int64_t t = rows.start + i;
        bool keep = false;
        if (i < rows.n - 1) {
            const int d = a.ids[t];
            if (d >= 0 && d < a.V) {
                const double p = (double)value(target_row<E>(a, t), d);
                const double q = a.draft ? (double)value(draft_row<E>(a, t - b), d) : 1.0;
                keep = (double)a.u[t] * q < p;
            }
        }
        const uint64_t not_kept = __builtin_amdgcn_ballot_w64(!keep);
        if (not_kept) return i0 + __builtin_ctzll(not_kept);        // (the last row's at the latest)
    }
}

// The row where a sequence's drafts end: its values, and the draft's (or the id
// that stands for them) unless it is the last one.
template <typename E>
struct EndRow {
    const E *zp, *zq;
    int onehot;
    Norm np, nq;
    __device__ __forceinline__ EndRow(const Args& a, int b, Rows rows, int kept) : zq(nullptr), onehot(-1), np{0.0, 1.0}, nq{0.0, 1.0} {
        const int64_t t = rows.start + kept;
        zp = target_row<E>(a, t);
        if (kept < rows.n - 1) {
            if (a.draft) zq = draft_row<E>(a, t - b);
            else onehot = a.ids[t];
        }
        if (a.logits) {
            const double4 n = a.row[b];
            np = {n.x, n.y};
            nq = {n.z, n.w};
        }
    }
    // (max(p - q, 0), p) of entry v with the values x and y, NaN where p or q is
    __device__ __forceinline__ double2 left(const Args& a, int v, float x, float y) const {
        const double p = prob(a, x, np);
        const double q = zq ? prob(a, y, nq) : v == onehot ? 1.0 : 0.0;
        const double d = p - q;
        return make_double2(d <= 0.0 ? 0.0 : d, p);
    }
};

// What is left over in every piece of the end rows.
template <typename E>
__global__ __launch_bounds__(kThreads) void left_over_kernel(Args a, int total) {
    const int at = (int)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (at >= total) return;
    const int b = at / a.pieces, piece = at - b * a.pieces, v0 = piece * kPiece;
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) return;
    int kept;
    if (a.logits) {
        kept = a.kept[b];
    } else {
        kept = kept_of_probs<E>(a, b, rows);
        if (piece == 0 && (threadIdx.x & 63) == 0) a.kept[b] = kept;
    }
    const EndRow<E> e(a, b, rows, kept);
    const float fill = a.logits ? -INFINITY : 0.0f;
    double r = 0.0, p = 0.0;
    if (bad(e.np) || bad(e.nq)) {
        r = p = __builtin_nan("");
    } else {
        Piece<E> x, y;
        x.load(e.zp, v0, a.V, fill);
        if (e.zq) y.load(e.zq, v0, a.V, fill);
#pragma unroll
        for (int i = 0; i < x.N; ++i)
#pragma unroll
            for (int k = 0; k < kPerVector<E>; ++k) {
                const double2 l = e.left(a, x.at(v0, i) + k, x.x[i][k], e.zq ? y.x[i][k] : 0.0f);
                r += l.x;
                p += l.y;
            }
        r = wave_sum(r);
        p = wave_sum(p);
    }
    if ((threadIdx.x & 63) == 0) a.left[at] = make_double2(r, p);
}

// ---- the draw ----------------------------------------------------------------------

// Whether sequence b begins before an earlier offset (by the whole block): its
// tokens would be written over another's.
__device__ __forceinline__ bool overlaps(const Args& a, int b) {
    const int start = a.offsets[b];
    bool any = false;
    for (int i = threadIdx.x; i < b; i += kThreads) any = any || a.offsets[i] > start;
    return __syncthreads_or(any) != 0;
}

__device__ __forceinline__ void write_tokens(const Args& a, int b, Rows rows, int kept, int token) {
    for (int i = threadIdx.x; i < rows.n; i += kThreads)
        a.tokens[rows.start + i] = i < kept ? a.ids[rows.start + i] : i == kept ? token : -1;
    if (threadIdx.x == 0) a.accepted[b] = kept;
}

// Sum of the threads' values before this one's, and of all of them, in a fixed order.
struct Scan {
    double before, all;
};
__device__ __forceinline__ Scan block_scan(double v, double* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(s, o, 64);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    double before = 0.0, all = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = all;
        all += red[w];
    }
    // (what lies before the lane: the lane below's inclusive sum)
    const double below = __shfl_up(s, 1, 64);
    return {before + (lane > 0 ? below : 0.0), all};
}

// The first thread (and its item) that says `hit`, else the last that says
// `positive`, else -1: items are numbered thread * PER + item, in order.
__device__ __forceinline__ int first_or_last(int hit, int positive, int* red) {
    if (threadIdx.x == 0) {
        red[0] = INT32_MAX;
        red[1] = -1;
    }
    __syncthreads();
    if (hit >= 0) atomicMin(&red[0], hit);           // (the least, or greatest, integer: the same in any order)
    if (positive >= 0) atomicMax(&red[1], positive);
    __syncthreads();
    return red[0] != INT32_MAX ? red[0] : red[1];
}

template <typename E>
__global__ __launch_bounds__(kThreads) void draw_kernel(Args a) {
    __shared__ double red[kWaves];
    __shared__ double start;
    __shared__ int pick[2];
    const int b = blockIdx.x;
    Rows rows = rows_of(a, b);
    if (overlaps(a, b)) rows.n = -1;
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    const int kept = a.kept[b];
    // the piece: each thread some of them in a row
    const double2* left = a.left + (int64_t)b * a.pieces;
    const int per = (a.pieces + kThreads - 1) / kThreads;
    const int c0 = min(a.pieces, (int)threadIdx.x * per), c1 = min(a.pieces, c0 + per);
    double rs = 0.0, ps = 0.0;
    for (int c = c0; c < c1; ++c) {
        rs += left[c].x;
        ps += left[c].y;
    }
    const Scan r = block_scan(rs, red), p = block_scan(ps, red);
    if (!(p.all > 0.0 && p.all < kInf && r.all >= 0.0)) {
        write_tokens(a, b, rows, kept, -1);
        return;
    }
    const bool use_p = !(r.all > 0.0);
    const Scan s = use_p ? p : r;
    const double goal = (double)a.us[b] * s.all;
    int hit = -1, positive = -1;
    double run = s.before;
    for (int c = c0; c < c1; ++c) {
        const double x = use_p ? left[c].y : left[c].x;
        if (x > 0.0) positive = c;
        if (hit < 0 && x > 0.0 && run + x > goal) hit = c;
        run += x;
    }
    const int piece = first_or_last(hit, positive, pick);
    run = s.before;
    for (int c = c0; c < c1; ++c) {
        if (c == piece) start = run;
        run += use_p ? left[c].y : left[c].x;
    }
    __syncthreads();
    // the entry: each thread eight of the piece in a row
    constexpr int PER = kPiece / kThreads;
    const EndRow<E> e(a, b, rows, kept);
    const int v0 = piece * kPiece + threadIdx.x * PER;
    double w[PER], sum = 0.0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int v = v0 + k;
        w[k] = 0.0;
        if (v < a.V) {
            const double2 l = e.left(a, v, value(e.zp, v), e.zq ? value(e.zq, v) : 0.0f);
            w[k] = use_p ? l.y : l.x;
        }
        sum += w[k];
    }
    run = start + block_scan(sum, red).before;
    hit = positive = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        run += w[k];
        if (w[k] > 0.0) positive = v0 + k;
        if (hit < 0 && w[k] > 0.0 && run > goal) hit = v0 + k;
    }
    write_tokens(a, b, rows, kept, first_or_last(hit, positive, pick));
}

// ---- temperature 0: (largest logit, its lowest id) of every piece of the target's rows.
template <typename E>
__global__ __launch_bounds__(kThreads) void piece_max_kernel(Args a, int total) {
    const int at = (int)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (at >= total) return;
    const int r = at / a.pieces, v0 = (at - r * a.pieces) * kPiece;
    Piece<E> x;
    x.load(target_row<E>(a, r), v0, a.V, -INFINITY);
    float m = -INFINITY;
    int id = a.V;
    auto take = [&](float v, int i) {
        if (v > m || (v == m && i < id) || (v != v && m == m)) { m = v; id = i; }
    };
#pragma unroll
    for (int i = 0; i < x.N; ++i)
#pragma unroll
        for (int e = 0; e < kPerVector<E>; ++e) take(x.x[i][e], x.at(v0, i) + e);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const float v = __shfl_xor(m, o, 64);
        const int i = __shfl_xor(id, o, 64);
        take(v, i);
    }
    if ((threadIdx.x & 63) == 0) a.stats[at] = make_double2((double)m, (double)id);
}

// A row's choice, -1 where it has none (NaN, +infinity or nothing but -infinity), by
// one wave.
__device__ __forceinline__ int row_choice(const Args& a, int64_t r) {
    const double2* st = a.stats + r * a.pieces;
    double m = -kInf, id = 0.0;
    auto take = [&](double v, double i) {
        if (v > m || (v == m && i < id) || (v != v && m == m)) { m = v; id = i; }
    };
    for (int c = threadIdx.x & 63; c < a.pieces; c += 64) take(st[c].x, st[c].y);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const double v = __shfl_xor(m, o, 64), i = __shfl_xor(id, o, 64);
        take(v, i);
    }
    return m > -kInf && m < kInf ? (int)id : -1;
}

__global__ __launch_bounds__(kThreads) void greedy_kernel(Args a) {
    __shared__ int choice[kWaves];
    const int b = blockIdx.x, wave = threadIdx.x >> 6;
    Rows rows = rows_of(a, b);
    if (overlaps(a, b)) rows.n = -1;
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    for (int i0 = 0;; i0 += kWaves) {
        if (i0 + wave < rows.n) {
            const int c = row_choice(a, rows.start + i0 + wave);
            if ((threadIdx.x & 63) == 0) choice[wave] = c;
        }
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            const int i = i0 + w;
            if (i == rows.n - 1 || choice[w] < 0 || choice[w] != a.ids[rows.start + i]) {
                write_tokens(a, b, rows, i, choice[w]);
                return;
            }
        }
        __syncthreads();
    }
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct Layout {
    int pieces;
    size_t left, row, kept, total;       // (the rows' sums first)
};
Layout layout(int64_t B, int64_t T, int64_t draft_rows, int64_t V) {
    Layout l{};
    l.pieces = (int)((V + kPiece - 1) / kPiece);
    l.left = up((size_t)(T + draft_rows) * l.pieces * sizeof(double2));
    l.row = l.left + up((size_t)B * l.pieces * sizeof(double2));
    l.kept = l.row + up((size_t)B * sizeof(double4));
    l.total = l.kept + up((size_t)B * sizeof(int));
    return l;
}

template <typename E>
void launch(const Args& a, hipStream_t stream) {
    auto blocks = [](int64_t n) { return (unsigned)((n + kWaves - 1) / kWaves); };
    if (a.temperature == 0.0) {
        const int total = a.T * a.pieces;
        if (total > 0) piece_max_kernel<E><<<blocks(total), kThreads, 0, stream>>>(a, total);
        greedy_kernel<<<a.B, kThreads, 0, stream>>>(a);
        return;
    }
    if (a.logits) {
        const int total = (a.T + (a.draft ? a.draft_rows : 0)) * a.pieces;
        if (total > 0) piece_sums_kernel<E><<<blocks(total), kThreads, 0, stream>>>(a, total);
        end_rows_kernel<E><<<a.B, kEndWaves * 64, 0, stream>>>(a);
    }
    const int total = a.B * a.pieces;
    left_over_kernel<E><<<blocks(total), kThreads, 0, stream>>>(a, total);
    draw_kernel<E><<<a.B, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t verify_ws_bytes(int64_t B, int64_t T, int64_t draft_rows, int64_t V) { return layout(B, T, draft_rows, V).total; }

void launch_verify(const VerifyArgs& v, void* ws, hipStream_t stream) {
    const Layout l = layout(v.B, v.T, v.draft_rows, v.V);
    uint8_t* w = reinterpret_cast<uint8_t*>(ws);
    Args a;
    static_cast<VerifyArgs&>(a) = v;
    a.pieces = l.pieces;
    a.c = v.temperature == 0.0 ? 0.0 : 1.4426950408889634 / v.temperature;
    a.stats = reinterpret_cast<double2*>(w);
    a.left = reinterpret_cast<double2*>(w + l.left);
    a.row = reinterpret_cast<double4*>(w + l.row);
    a.kept = reinterpret_cast<int*>(w + l.kept);
    if (v.bf16) launch<uint16_t>(a, stream);
    else launch<float>(a, stream);
}

}  // namespace puro
