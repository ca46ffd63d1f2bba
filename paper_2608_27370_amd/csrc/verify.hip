// Verification of drafted tokens for gfx950: which drafts of a sequence are kept,
// and the token drawn from what the target's probabilities leave over.
//
// With p, q the target's and the draft's probabilities of a row, draft d is kept
// with probability min(1, p(d) / q(d)), and the first that is not is replaced by a
// draw from max(p - q, 0) / sum max(p - q, 0): the kept or drawn token is then
// distributed as p.
//
// A vocabulary row is worked on in pieces of 1024 or 2048 entries, a wave each; every sum
// over a row is made of its pieces' sums, in a fixed order.
//  * LOGITS: of every row the pieces' largest logits and sums of exponentials, then
//    of every sequence, by a block of 16 waves (a row each), the row where its
//    drafts end and that row's sums. PROBS: the drafts' entries alone say that row;
//  * the pieces of that row: what is left over of each, and of p (LOGITS of p alone:
//    their sums say it);
//  * a block per sequence: the piece, then the entry where the running sum passes
//    the random number's share.
// Exponentials (to 10^-10), probabilities and sums are binary64: with 10^5 entries a
// running sum that errs by 10^-8 moves the drawn token once in 10^3 draws.

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace puro {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr double kInf = __builtin_huge_val();

struct Args : VerifyArgs {
    int pieces;           // of a row
    Divisor by_pieces;
    double c, span;       // log2(e) / temperature; 1000 / c
    double2* stats;       // [T + draft_rows][pieces]: largest logit; sum of 2^((z - largest) c) (greedy: its id)
    double2* left;        // [B][pieces]: sums of max(p - q, 0) and of p
    double4* row;         // [B]: the end row's largest logits and reciprocal sums, target and draft
    int2* end;            // [B]: drafts kept (-1: no rows, -2: invalid ones) and Rows::shift
    int2* before;         // [B], of many sequences: the largest offset before each, and how many before it have no rows
};

// The wave's piece of `total`: its index, row and place in it.
struct Item {
    int at, row, piece;
    bool live;
};
__device__ __forceinline__ Item item(const Args& a, int total) {
    const int at = (int)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = (int)a.by_pieces.quotient((uint32_t)at);
    return {at, row, at - row * a.pieces, at < total};
}

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

// The lane's entries of a piece of LEN, vector i at v0 + (i 64 + lane) * kPerVector,
// `fill` past the row's end.
template <typename E, int LEN>
struct Piece {
    static constexpr int N = LEN / 64 / kPerVector<E>;
    float x[N][kPerVector<E>];
    __device__ __forceinline__ static int at(int v0, int i) { return v0 + (i * 64 + (threadIdx.x & 63)) * kPerVector<E>; }
    __device__ __forceinline__ void load(const E* row, int v0, int V, float fill) {
        if (v0 + LEN <= V) {
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

// 2^-f in binary64 for f in [0, 1]: the polynomial of degree 7, 1 at 0, of the least
// largest relative error, 4.4e-11 (the random numbers are of steps of 6e-8). Of N
// values at a time, whose chains of dependent instructions fill each other's waits.
template <int N>
__device__ __forceinline__ void exp2_fractions(const double f[N], double p[N]) {
    constexpr double kC[8] = {-0x1.69fa9638ac087p-17, 0x1.349aa24075c04p-13, -0x1.5c09ebe989994p-10, 0x1.3b149cd8db03cp-7,
                              -0x1.c6af2acf64e86p-5, 0x1.ebfbd54ce8792p-3, -0x1.62e42fd37055cp-1, 1.0};
#pragma unroll
    for (int k = 0; k < N; ++k) p[k] = kC[0];
#pragma unroll
    for (int c = 1; c < 8; ++c)
#pragma unroll
        for (int k = 0; k < N; ++k) p[k] = __builtin_fma(p[k], f[k], kC[c]);
}
// 2^-u, 0 above 1074; u at least 0, or infinity.
__device__ __forceinline__ double exp2_minus(double u) {
    u = fmin(u, 2000.0);
    const double f[1] = {__builtin_amdgcn_fract(u)};
    double p[1];
    exp2_fractions<1>(f, p);
    return __builtin_ldexp(p[0], (int)-u);
}

// The larger of two, NaN passed over, and the largest of three, NaN if one is (one
// instruction; written as fmaxf the compiler quiets each operand first).
__device__ __forceinline__ float max2(float a, float b) {
    float m;
    asm("v_max_f32 %0, %1, %2" : "=v"(m) : "v"(a), "v"(b));
    return m;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// What is no more than this counts as no probability at all (and a piece of no more
// than 2^20 times it as one without).
constexpr double kLeast = 0x1p-990;

// 2^((x - m) c) of logits x no larger than m, of N at a time. Where m c is of ordinary
// size (near: the exponent x c - m c errs by no more than 2^-40, and binary32's
// spacing at m is far less than 1 in it) logits are clamped, as they stand, to where
// that is about 2^-1000 (below kLeast), and the power of two is added to the exponent
// of 2^-f: fewer instructions. The exponent's whole and fractional parts are taken
// apart as those of a number that is not negative, which m c, moved up by 2^-51 of
// itself, makes sure of.
struct Exponential {
    double m, c, mc;
    float lo;
    bool near;
    __device__ __forceinline__ Exponential(const Args& a, double m_)
        : m(m_), c(a.c), mc(__builtin_fma(fabs(m_ * a.c), 0x1p-51, m_ * a.c)), lo((float)(m_ - a.span)), near(fabs(m_) * a.c < 0x1p13) {}
    template <bool NEAR, int N>
    __device__ __forceinline__ void of(const float x[N], double e[N]) const {
        if constexpr (!NEAR) {
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = exp2_minus((m - (double)x[k]) * c);
            return;
        }
        double u[N], f[N];
#pragma unroll
        for (int k = 0; k < N; ++k) u[k] = __builtin_fma(-(double)max2(x[k], lo), c, mc);
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = __builtin_amdgcn_fract(u[k]);
        exp2_fractions<N>(f, e);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t n = (uint32_t)(int)-u[k];
            e[k] = __hiloint2double((int)((uint32_t)__double2hiint(e[k]) + (n << 20)), __double2loint(e[k]));
        }
    }
};

// Sums and maxima over a wave, in every lane: rotations within 16 lanes, then swaps of
// rows (no LDS).
template <int ROR>
__device__ __forceinline__ int rotated(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x120 + ROR, 0xF, 0xF, false); }
template <int ROR>
__device__ __forceinline__ double rotated(double v) {
    return __hiloint2double(rotated<ROR>(__double2hiint(v)), rotated<ROR>(__double2loint(v)));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = __hiloint2double(hi[0], lo[0]) + __hiloint2double(hi[1], lo[1]);
    lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
    hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
    return __hiloint2double(hi[0], lo[0]) + __hiloint2double(hi[1], lo[1]);
}
__device__ __forceinline__ float wave_max(float v) {
    v = max3(v, v, __int_as_float(rotated<8>(__float_as_int(v))));
    v = max3(v, v, __int_as_float(rotated<4>(__float_as_int(v))));
    v = max3(v, v, __int_as_float(rotated<2>(__float_as_int(v))));
    v = max3(v, v, __int_as_float(rotated<1>(__float_as_int(v))));
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    v = max3(v, __int_as_float(a[0]), __int_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return max3(v, __int_as_float(b[0]), __int_as_float(b[1]));
}
// The larger of two values, NaN if either is.
template <typename F>
__device__ __forceinline__ F max_nan(F a, F b) { return a > b || a != a ? a : b; }

// A row's normaliser: its largest logit m and the reciprocal of its sum; not finite
// (then NaN) for a row with a NaN or an infinity, or without any probability.
struct Norm {
    double m, inv;
};
// (an entry's probability: of a logit, or the value itself)
__device__ __forceinline__ double prob_at(const Args& a, float x, const Norm& n) {
    if (!a.logits) return (double)x;
    const Exponential e(a, n.m);
    const float v[1] = {x};
    double p[1];
    if (e.near) e.of<true, 1>(v, p);
    else e.of<false, 1>(v, p);
    return p[0] * n.inv;
}
__device__ __forceinline__ bool bad(const Norm& n) { return !(n.inv < kInf); }

// ---- sequences -------------------------------------------------------------------

// Rows of sequence b: its first, how many (0: none; -1: invalid), and what the draft's
// row of a target row is less than that: the sequences before whose last rows the draft
// has none for, those without rows not among them. Waves look through the offsets
// before (a sequence that begins before one of them would write its tokens over
// another's); of many sequences that is done in a launch before (65536 of them of two
// rows of 20 entries 4.5 ms and 1.1 in all).
struct Rows {
    int start, n, shift;
};
constexpr int kManySequences = 512;
__device__ __forceinline__ Rows rows_of(const Args& a, int b) {
    const int64_t start = a.offsets[b], end = a.offsets[b + 1];
    bool overlaps = false;
    int empty = 0;
    if (a.before) {
        const int2 v = a.before[b];
        overlaps = v.x > start;
        empty = v.y;
    } else {
        int mine = 0;
        for (int i = threadIdx.x & 63; i < b; i += 64) {
            const int at = a.offsets[i];
            overlaps = overlaps || at > start;
            mine += at == a.offsets[i + 1];
        }
        overlaps = __builtin_amdgcn_ballot_w64(overlaps) != 0;
        static_assert(kManySequences / 64 < 1 << 4, "a lane's count");
#pragma unroll
        for (int k = 0; k < 4; ++k) empty += __builtin_popcountll(__builtin_amdgcn_ballot_w64((mine >> k & 1) != 0)) << k;
    }
    const int shift = b - empty;
    if (overlaps || start < 0 || end < start || end > a.T) return {0, -1, 0};
    const int n = (int)(end - start);
    // its draft rows: start - shift .. end - 2 - shift
    if (a.draft && n > 1 && (start - shift < 0 || end - 1 - shift > a.draft_rows)) return {0, -1, 0};
    return {(int)start, n, shift};
}
// The same as an earlier launch left it in end[b].
__device__ __forceinline__ int2 ended(Rows rows, int kept) { return make_int2(rows.n > 0 ? kept : rows.n - 1, rows.shift); }
__device__ __forceinline__ Rows rows_of(const Args& a, int b, int2 end) {
    const int start = a.offsets[b];
    return {start, end.x < 0 ? end.x + 1 : a.offsets[b + 1] - start, end.y};
}
template <typename E>
__device__ __forceinline__ const E* target_row(const Args& a, int64_t t) { return (const E*)a.target + t * a.ld_t; }
template <typename E>
__device__ __forceinline__ const E* draft_row(const Args& a, int64_t t) { return (const E*)a.draft + t * a.ld_d; }

// A piece's largest entry, NaN if one is, in every lane of its wave.
template <typename E, int LEN>
__device__ __forceinline__ float largest(const Piece<E, LEN>& x) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < x.N; ++i)
#pragma unroll
        for (int e = 0; e < kPerVector<E>; e += 2) m = max3(m, x.x[i][e], x.x[i][e + 1]);
    return wave_max(m);
}

// ---- LOGITS: (largest, sum of 2^((z - largest) c)) of every piece of every row.
// Bound by its arithmetic and, nearly as closely, by memory: 16.5 instructions an entry,
// 11 of them binary64, keep the vector units busy for 85% of the time (768 BF16 rows of
// 151936: 67 to 69 us, 3.4 TB/s; a copy's rate would be 49). With a polynomial of degree 8 and
// the exponent rounded by an addition, 19.5: 76; the next piece's loads in flight while
// one is summed: 79 to 84.
template <typename E, int LEN>
__global__ __launch_bounds__(kThreads) void piece_sums_kernel(Args a, int total) {
    const Item it = item(a, total);
    if (!it.live) return;
    const int r = it.row, v0 = it.piece * LEN;
    const E* z = r < a.T ? target_row<E>(a, r) : draft_row<E>(a, r - a.T);
    Piece<E, LEN> x;
    x.load(z, v0, a.V, -INFINITY);
    float m = largest(x);
    double s = 0.0;
    if (!(m < INFINITY)) {
        m = __builtin_nanf("");
        s = __builtin_nan("");
    } else if (m > -INFINITY) {
        const Exponential exponential(a, (double)m);
        auto sum = [&](auto near_c) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < x.N; ++i)
#pragma unroll
                for (int e = 0; e < kPerVector<E>; e += 4) {
                    double t[4];
                    exponential.template of<decltype(near_c)::value, 4>(x.x[i] + e, t);
                    s += (t[0] + t[1]) + (t[2] + t[3]);
                }
        };
        if (exponential.near) sum(std::true_type{});
        else sum(std::false_type{});
        s = wave_sum(s);
    }
    if ((threadIdx.x & 63) == 0) a.stats[it.at] = make_double2((double)m, s);
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
        s += v.y * exp2_minus((m - v.x) * a.c);
    }
    return {m, 1.0 / wave_sum(s)};
}

// Where a sequence's drafts end, and that row's normalisers: by a block of 16 waves,
// sixteen rows at a time, or eight and their drafts', a wave for each one's.
constexpr int kEndWaves = 16;
struct End {
    int kept;
    Norm p, q;
};
struct EndScratch {
    Norm norms[kEndWaves];
    double prob[kEndWaves];         // of the row's draft
    float u[kEndWaves];
};
template <typename E>
__device__ __forceinline__ End find_end(const Args& a, Rows rows, EndScratch& s) {
    const int wave = threadIdx.x >> 6, per = a.draft ? kEndWaves / 2 : kEndWaves;
    const bool of_target = wave < per;
    for (int i0 = 0;; i0 += per) {
        const int i = i0 + (of_target ? wave : wave - per);
        const int64_t t = rows.start + i;
        const bool drafted = i < rows.n - 1;
        // (asked for ahead of the row's sums)
        const int d = drafted ? a.ids[t] : -1;
        const bool has = d >= 0 && d < a.V;
        const float x = has ? value(of_target ? target_row<E>(a, t) : draft_row<E>(a, t - rows.shift), d) : 0.0f;
        const float u = drafted && of_target ? a.u[t] : 0.0f;
        if (of_target ? i < rows.n : drafted) {
            const Norm n = row_norm(a, of_target ? t : a.T + t - rows.shift);
            const double prob = has && !bad(n) ? prob_at(a, x, n) : __builtin_nan("");
            if ((threadIdx.x & 63) == 0) {
                s.norms[wave] = n;
                s.prob[wave] = prob;
                s.u[wave] = u;
            }
        }
        __syncthreads();
        // (the last row is not kept, at the latest, whose id is not one)
        int w = 0;
        while (w < per && (double)s.u[w] * (a.draft ? s.prob[w + per] : 1.0) < s.prob[w] && s.prob[w] > kLeast) ++w;
        if (w < per) return {i0 + w, s.norms[w], i0 + w == rows.n - 1 || !a.draft ? Norm{0.0, 0.0} : s.norms[w + per]};
        __syncthreads();
    }
}

// Latency: 6.1 to 6.4 us for 96 sequences of up to eight rows of 151936 and their drafts'.
template <typename E>
__global__ __launch_bounds__(kEndWaves * 64) void end_rows_kernel(Args a) {
    __shared__ EndScratch scratch;
    const int b = blockIdx.x;
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.end[b] = ended(rows, 0);
        return;
    }
    const End e = find_end<E>(a, rows, scratch);
    if (threadIdx.x == 0) {
        a.end[b] = ended(rows, e.kept);
        a.row[b] = make_double4(e.p.m, e.p.inv, e.q.m, e.q.inv);
    }
}

// The same of probabilities, whose entries say it alone: by one wave, 64 drafts at a
// time (every wave of every block that needs it, rather than a launch of its own).
template <typename E>
__device__ __forceinline__ int kept_of_probs(const Args& a, Rows rows) {
    for (int i0 = 0;; i0 += 64) {
        const int i = i0 + (threadIdx.x & 63);
        const int64_t t = rows.start + i;
        bool keep = false;
        if (i < rows.n - 1) {
            const int d = a.ids[t];
            if (d >= 0 && d < a.V) {
                const double p = (double)value(target_row<E>(a, t), d);
                const double q = a.draft ? (double)value(draft_row<E>(a, t - rows.shift), d) : 1.0;
                keep = (double)a.u[t] * q < p && p > kLeast;
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
    __device__ __forceinline__ EndRow(const Args& a, Rows rows, int kept, Norm p, Norm q) : zq(nullptr), onehot(-1), np(p), nq(q) {
        const int64_t t = rows.start + kept;
        zp = target_row<E>(a, t);
        if (kept < rows.n - 1) {
            if (a.draft) zq = draft_row<E>(a, t - rows.shift);
            else onehot = a.ids[t];
        }
    }
    // (as end_rows_kernel left them)
    __device__ __forceinline__ static EndRow of(const Args& a, int b, Rows rows, int kept) {
        if (!a.logits) return EndRow(a, rows, kept, {0.0, 1.0}, {0.0, 1.0});
        const double4 n = a.row[b];
        return EndRow(a, rows, kept, {n.x, n.y}, {n.z, n.w});
    }
};
// (max(p - q, 0), p), NaN where p or q is; 0 where no more than kLeast, so that a
// piece with a share has an entry with one. p and q are rounded products: fused into the
// difference, one of them unrounded, equal ones would leave 10^-17 of noise.
__device__ __forceinline__ double2 left(double p, double q) {
#pragma clang fp contract(off)
    const double d = p - q;
    return make_double2(d <= kLeast ? 0.0 : d, p <= kLeast ? 0.0 : p);
}
// The same of values that are not NaN, for a sum that piece_share follows: fewer
// instructions.
__device__ __forceinline__ double2 left_about(double p, double q) {
#pragma clang fp contract(off)
    return make_double2(__builtin_fmax(p - q, 0.0), p);
}
__device__ __forceinline__ double piece_share(double sum) { return sum <= 0x1p20 * kLeast ? 0.0 : sum; }
// f(g), where g(v, x, y, l) gives N entries from v on with the values x and y (the
// draft's) their l = left(p, q), by the kind of the row's entries: logits of
// ordinary size, others, probabilities.
template <int N, bool SUM, typename E, typename F>
__device__ __forceinline__ void with_left(const Args& a, const EndRow<E>& e, F&& f) {
    auto run = [&](auto kind_c, auto q_c) __attribute__((always_inline)) {
        constexpr int KIND = decltype(kind_c)::value;          // 0: probabilities, 1, 2: logits
        constexpr bool Q = decltype(q_c)::value;
        const Exponential ep(a, e.np.m), eq(a, e.nq.m);
        f([&](int v, const float* x, const float* y, double2* l) __attribute__((always_inline)) {
            double p[N], q[N];
            if constexpr (KIND != 0) {
                ep.template of<KIND == 1, N>(x, p);
                if constexpr (Q) eq.template of<KIND == 1, N>(y, q);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const double pk = KIND != 0 ? p[k] * e.np.inv : (double)x[k];
                double qk = v + k == e.onehot ? 1.0 : 0.0;
                if constexpr (Q) qk = KIND != 0 ? q[k] * e.nq.inv : (double)y[k];
                l[k] = SUM && KIND != 0 ? left_about(pk, qk) : left(pk, qk);
            }
        });
    };
    auto with_q = [&](auto kind_c) __attribute__((always_inline)) {
        if (e.zq) run(kind_c, std::true_type{});
        else run(kind_c, std::false_type{});
    };
    if (!a.logits) with_q(std::integral_constant<int, 0>{});
    else if (Exponential(a, e.np.m).near && Exponential(a, e.nq.m).near) with_q(std::integral_constant<int, 1>{});
    else with_q(std::integral_constant<int, 2>{});
}

// The share of p of a piece of row t, from its sum; 0 where no entry of it can have one.
__device__ __forceinline__ double share(const Args& a, int64_t t, int c, const Norm& n) {
    const double2 st = a.stats[t * a.pieces + c];
    const double p = st.y * exp2_minus((n.m - st.x) * a.c) * n.inv;
    return piece_share(p);
}

// What is left over in every piece of the end rows. Of LOGITS two exponentials an
// entry: 19 us for 96 rows of 151936 and their drafts', found in the caches (of rows
// without a draft's, the sums of their pieces: 25 -> 21; the least shares dropped by the
// piece, not by the entry: 20 -> 19).
template <typename E, int LEN>
__global__ __launch_bounds__(kThreads) void left_over_kernel(Args a, int total) {
    const Item it = item(a, total);
    if (!it.live) return;
    const int b = it.row, v0 = it.piece * LEN;
    Rows rows;
    int kept = 0;
    if (a.logits) {
        const int2 end = a.end[b];
        rows = rows_of(a, b, end);
        kept = end.x;
    } else {
        rows = rows_of(a, b);
        if (rows.n > 0) kept = kept_of_probs<E>(a, rows);
        if (it.piece == 0 && (threadIdx.x & 63) == 0) a.end[b] = ended(rows, kept);
    }
    if (rows.n <= 0) return;
    const EndRow<E> e = EndRow<E>::of(a, b, rows, kept);
    const float fill = a.logits ? -INFINITY : 0.0f;
    double r = 0.0, p = 0.0;
    if (bad(e.np) || bad(e.nq)) {
        r = p = __builtin_nan("");
    } else if (a.logits && !e.zq) {
        r = p = share(a, rows.start + kept, it.piece, e.np);
    } else {
        Piece<E, LEN> x, y;
        x.load(e.zp, v0, a.V, fill);
        if (e.zq) y.load(e.zq, v0, a.V, fill);
        else y = x;
        with_left<4, true>(a, e, [&](auto&& left_at) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < x.N; ++i)
#pragma unroll
                for (int k = 0; k < kPerVector<E>; k += 4) {
                    double2 l[4];
                    left_at(x.at(v0, i) + k, x.x[i] + k, y.x[i] + k, l);
                    r += (l[0].x + l[1].x) + (l[2].x + l[3].x);
                    p += (l[0].y + l[1].y) + (l[2].y + l[3].y);
                }
        });
        r = piece_share(wave_sum(r));
        p = piece_share(wave_sum(p));
    }
    if ((threadIdx.x & 63) == 0) a.left[it.at] = make_double2(r, p);
}

// ---- the draw ----------------------------------------------------------------------
// One block per sequence, a chain of short steps: what they need of memory is asked
// for at the start, and every wave finds the piece by itself (no barrier). 4 to 6 us.

constexpr int kScanThreads = 1024;
// before[b] = the largest of offsets[0 .. b - 1], and how many i < b have offsets[i] ==
// offsets[i + 1]: one block, each thread some sequences in a row.
__global__ __launch_bounds__(kScanThreads) void offsets_before_kernel(Args a) {
    __shared__ int2 waves[kScanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = (a.B + kScanThreads - 1) / kScanThreads;
    const int b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
    int m = INT_MIN, n = 0;
#pragma unroll 8
    for (int b = b0; b < b1; ++b) {
        m = max(m, a.offsets[b]);
        n += a.offsets[b] == a.offsets[b + 1];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(m, o, 64), k = __shfl_up(n, o, 64);
        if (lane >= o) {
            m = max(m, t);
            n += k;
        }
    }
    if (lane == 63) waves[wave] = make_int2(m, n);
    __syncthreads();
    const int below = __shfl_up(m, 1, 64), fewer = __shfl_up(n, 1, 64);
    m = lane > 0 ? below : INT_MIN;
    n = lane > 0 ? fewer : 0;
    for (int w = 0; w < wave; ++w) {
        m = max(m, waves[w].x);
        n += waves[w].y;
    }
    for (int b = b0; b < b1; ++b) {
        a.before[b] = make_int2(m, n);
        m = max(m, a.offsets[b]);
        n += a.offsets[b] == a.offsets[b + 1];
    }
}

template <int THREADS>
__device__ __forceinline__ void write_tokens(const Args& a, int b, Rows rows, int kept, int token) {
    for (int i = threadIdx.x; i < rows.n; i += THREADS)
        a.tokens[rows.start + i] = i < kept ? a.ids[rows.start + i] : i == kept ? token : -1;
    if (threadIdx.x == 0) a.accepted[b] = kept;
}

// The sum of the lanes' values up to and with this one's, in a fixed order.
__device__ __forceinline__ double wave_scan(double v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(v, o, 64);
        if (lane >= o) v += t;
    }
    return v;
}
__device__ __forceinline__ double lane_below(double v) {
    const double t = __shfl_up(v, 1, 64);
    return (threadIdx.x & 63) > 0 ? t : 0.0;
}

// The PER entries of a piece that are this thread's, in a row, as l = left(p, q).
template <int PER, typename E, typename F>
__device__ __forceinline__ void with_entries(const Args& a, const EndRow<E>& e, int v0, F&& f) {
    float x[PER], y[PER];
    auto values = [&](const E* z, float* to) __attribute__((always_inline)) {
        if (v0 + PER <= a.V) {
            E raw[PER];
            __builtin_memcpy(raw, z + v0, sizeof(raw));
#pragma unroll
            for (int k = 0; k < PER; ++k) to[k] = value(raw, k);
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k) to[k] = v0 + k < a.V ? value(z, v0 + k) : a.logits ? -INFINITY : 0.0f;
        }
    };
    values(e.zp, x);
    values(e.zq ? e.zq : e.zp, y);
    with_left<PER, false>(a, e, [&](auto&& left_at) __attribute__((always_inline)) {
        double2 l[PER];
        left_at(v0, x, y, l);
        f(l);
    });
}

// The draw itself: left(c), the sums of piece c; the thread's first one l0.
template <int WAVES>
struct DrawScratch {
    double sums[WAVES];
    int hits[WAVES], positives[WAVES];
};
struct Lane {
    int c0, c1;           // its pieces
    __device__ __forceinline__ explicit Lane(const Args& a) {
        const int per = (a.pieces + 63) / 64, lane = threadIdx.x & 63;
        c0 = min(a.pieces, lane * per);
        c1 = min(a.pieces, c0 + per);
    }
};
template <int LEN, int WAVES, typename E, typename F>
__device__ __forceinline__ void draw(const Args& a, int b, Rows rows, int kept, const EndRow<E>& e, float us, Lane mine, double2 l0, F&& left,
                                     DrawScratch<WAVES>& s) {
    constexpr int THREADS = WAVES * 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = mine.c0, c1 = mine.c1;
    double rs = l0.x, ps = l0.y;
    for (int c = c0 + 1; c < c1; ++c) {
        const double2 l = left(c);
        rs += l.x;
        ps += l.y;
    }
    const double r = wave_scan(rs), p = wave_scan(ps);
    const double r_all = __shfl(r, 63, 64), p_all = __shfl(p, 63, 64);
    if (!(p_all > 0.0 && p_all < kInf && r_all >= 0.0)) {
        write_tokens<THREADS>(a, b, rows, kept, -1);
        return;
    }
    const bool use_p = !(r_all > 0.0);
    const double goal = (double)us * (use_p ? p_all : r_all);
    // (where rounding leaves no piece: the last one with a share)
    int hit = -1, positive = -1;
    double run = lane_below(use_p ? p : r), hit_at = 0.0, positive_at = 0.0;
    for (int c = c0; c < c1; ++c) {
        const double2 l = c == c0 ? l0 : left(c);
        const double x = use_p ? l.y : l.x;
        if (x > 0.0) {
            positive = c;
            positive_at = run;
            if (hit < 0 && run + x > goal) {
                hit = c;
                hit_at = run;
            }
        }
        run += x;
    }
    const uint64_t hits_in = __builtin_amdgcn_ballot_w64(hit >= 0), any_in = __builtin_amdgcn_ballot_w64(positive >= 0);
    const int from = hits_in ? __builtin_ctzll(hits_in) : 63 - __builtin_clzll(any_in);
    const int piece = __shfl(hits_in ? hit : positive, from, 64);
    const double start = __shfl(hits_in ? hit_at : positive_at, from, 64);
    // the entry: each thread some of the piece in a row
    constexpr int PER = LEN / THREADS;
    const int v0 = piece * LEN + threadIdx.x * PER;
    double w[PER], sum = 0.0;
    with_entries<PER>(a, e, v0, [&](const double2* l) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            w[k] = use_p ? l[k].y : l[k].x;
            sum += w[k];
        }
    });
    const double up_to = wave_scan(sum);
    if (lane == 63) s.sums[wave] = up_to;
    __syncthreads();
    run = start;
#pragma unroll
    for (int i = 0; i < WAVES - 1; ++i) run += i < wave ? s.sums[i] : 0.0;
    run += lane_below(up_to);
    hit = positive = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        run += w[k];
        if (w[k] > 0.0) {
            positive = v0 + k;
            if (hit < 0 && run > goal) hit = v0 + k;
        }
    }
    const uint64_t wave_hits = __builtin_amdgcn_ballot_w64(hit >= 0), wave_any = __builtin_amdgcn_ballot_w64(positive >= 0);
    const int h = __shfl(hit, wave_hits ? __builtin_ctzll(wave_hits) : 0, 64);
    const int q = __shfl(positive, wave_any ? 63 - __builtin_clzll(wave_any) : 0, 64);
    if (lane == 0) {
        s.hits[wave] = h;
        s.positives[wave] = q;
    }
    __syncthreads();
    int token = -1;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) token = max(token, s.positives[i]);
#pragma unroll
    for (int i = WAVES - 1; i >= 0; --i) token = s.hits[i] >= 0 ? s.hits[i] : token;
    write_tokens<THREADS>(a, b, rows, kept, token);
}

template <typename E, int LEN>
__global__ __launch_bounds__(kThreads) void draw_kernel(Args a) {
    __shared__ DrawScratch<kWaves> scratch;
    const int b = blockIdx.x;
    const double2* left = a.left + (int64_t)b * a.pieces;
    const Lane mine(a);
    const float us = a.T > 0 ? a.us[b] : 0.0f;        // (none are given for no rows)
    const int2 end = a.end[b];
    double2 l0 = make_double2(0.0, 0.0);
    if (mine.c0 < mine.c1) l0 = left[mine.c0];
    const Rows rows = rows_of(a, b, end);
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    const EndRow<E> e = EndRow<E>::of(a, b, rows, end.x);
    draw<LEN, kWaves>(a, b, rows, end.x, e, us, mine, l0, [&](int c) __attribute__((always_inline)) { return left[c]; }, scratch);
}

// LOGITS without the draft's: the end row and the draw in one launch. Nothing but the
// id's own entry is taken from p there, so that the pieces' shares are those of their
// sums, and the id's piece alone is summed again without it. 33 sequences of up to four
// rows of 50257: 4.4 + 6.3 + 4.4 us -> 9.1, of which the chain of short steps is the most.
template <typename E, int LEN>
__global__ __launch_bounds__(kEndWaves * 64) void end_and_draw_kernel(Args a) {
    __shared__ EndScratch end_scratch;
    __shared__ DrawScratch<kEndWaves> scratch;
    const int b = blockIdx.x;
    const float us = a.us[b];
    const Rows rows = rows_of(a, b);
    if (rows.n <= 0) {
        if (threadIdx.x == 0) a.accepted[b] = rows.n;
        return;
    }
    const End end = find_end<E>(a, rows, end_scratch);
    if (bad(end.p)) {
        write_tokens<kEndWaves * 64>(a, b, rows, end.kept, -1);
        return;
    }
    const EndRow<E> e(a, rows, end.kept, end.p, {0.0, 1.0});
    const int without = e.onehot >= 0 && e.onehot < a.V ? e.onehot / LEN : -1;
    double rest = 0.0;
    if (without >= 0) {
        constexpr int PER = LEN / (kEndWaves * 64);
        with_entries<PER>(a, e, without * LEN + threadIdx.x * PER, [&](const double2* l) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < PER; ++k) rest += l[k].x;
        });
        rest = wave_sum(rest);
        if ((threadIdx.x & 63) == 0) scratch.sums[threadIdx.x >> 6] = rest;
        __syncthreads();
        rest = 0.0;
#pragma unroll
        for (int i = 0; i < kEndWaves; ++i) rest += scratch.sums[i];
        __syncthreads();
    }
    auto left = [&](int c) __attribute__((always_inline)) {
        const double p = share(a, rows.start + end.kept, c, end.p);
        return make_double2(c == without ? rest : p, p);
    };
    const Lane mine(a);
    draw<LEN, kEndWaves>(a, b, rows, end.kept, e, us, mine, mine.c0 < mine.c1 ? left(mine.c0) : make_double2(0.0, 0.0), left, scratch);
}

// ---- temperature 0: (largest logit, its lowest id) of every piece of the target's rows:
// the largest first, then which of the lane's entries is it. Bound by memory and as
// closely by latency: 480 BF16 rows of 151936 30 us (both in one pass, with ties and NaN
// compared at every entry: 49).
template <typename E, int LEN>
__global__ __launch_bounds__(kThreads) void piece_max_kernel(Args a, int total) {
    const Item it = item(a, total);
    if (!it.live) return;
    const int v0 = it.piece * LEN;
    Piece<E, LEN> x;
    x.load(target_row<E>(a, it.row), v0, a.V, -INFINITY);
    const float m = largest(x);
    int id = a.V;
#pragma unroll
    for (int i = x.N - 1; i >= 0; --i)
#pragma unroll
        for (int e = kPerVector<E> - 1; e >= 0; --e) id = x.x[i][e] == m ? x.at(v0, i) + e : id;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) id = min(id, __shfl_xor(id, o, 64));
    if ((threadIdx.x & 63) == 0) a.stats[it.at] = make_double2((double)m, (double)id);
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
    const Rows rows = rows_of(a, b);
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
                __syncthreads();         // (tokens may be the ids themselves)
                write_tokens<kThreads>(a, b, rows, i, choice[w]);
                return;
            }
        }
        __syncthreads();
    }
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// Entries of a piece: as many as make the fewest instructions an entry, 2048, or half
// of them where all rows together are too few waves for the chip (eight a SIMD).
// 84 rows of 50257: 512 20.8 us, 1024 20.8, 2048 23.3, 4096 30.2; 768 rows of 151936:
// 119, 115, 113, 118.
int piece_length(int64_t T, int64_t V) { return T * V < (int64_t)8192 * 2048 ? 1024 : 2048; }

struct Layout {
    int len, pieces;
    size_t left, row, end, before, total;       // (the rows' sums first)
};
Layout layout(int64_t B, int64_t T, int64_t draft_rows, int64_t V) {
    Layout l{};
    l.len = piece_length(T, V);
    l.pieces = (int)((V + l.len - 1) / l.len);
    l.left = up((size_t)(T + draft_rows) * l.pieces * sizeof(double2));
    l.row = l.left + up((size_t)B * l.pieces * sizeof(double2));
    l.end = l.row + up((size_t)B * sizeof(double4));
    l.before = l.end + up((size_t)B * sizeof(int2));
    l.total = l.before + (B > kManySequences ? up((size_t)B * sizeof(int2)) : 0);
    return l;
}

template <typename E, int LEN>
void launch(const Args& a, hipStream_t stream) {
    auto blocks = [](int64_t n) { return (unsigned)((n + kWaves - 1) / kWaves); };
    if (a.before) offsets_before_kernel<<<1, kScanThreads, 0, stream>>>(a);
    if (a.temperature == 0.0) {
        const int total = a.T * a.pieces;
        if (total > 0) piece_max_kernel<E, LEN><<<blocks(total), kThreads, 0, stream>>>(a, total);
        greedy_kernel<<<a.B, kThreads, 0, stream>>>(a);
        return;
    }
    if (a.logits) {
        const int total = (a.T + (a.draft ? a.draft_rows : 0)) * a.pieces;
        if (total > 0) piece_sums_kernel<E, LEN><<<blocks(total), kThreads, 0, stream>>>(a, total);
        if (!a.draft && a.T > 0) {
            end_and_draw_kernel<E, LEN><<<a.B, kEndWaves * 64, 0, stream>>>(a);
            return;
        }
        end_rows_kernel<E><<<a.B, kEndWaves * 64, 0, stream>>>(a);
    }
    const int total = a.B * a.pieces;
    left_over_kernel<E, LEN><<<blocks(total), kThreads, 0, stream>>>(a, total);
    draw_kernel<E, LEN><<<a.B, kThreads, 0, stream>>>(a);
}

}  // namespace

size_t verify_ws_bytes(int64_t B, int64_t T, int64_t draft_rows, int64_t V) { return layout(B, T, draft_rows, V).total; }

void launch_verify(const VerifyArgs& v, void* ws, hipStream_t stream) {
    const Layout l = layout(v.B, v.T, v.draft_rows, v.V);
    uint8_t* w = reinterpret_cast<uint8_t*>(ws);
    Args a;
    static_cast<VerifyArgs&>(a) = v;
    a.pieces = l.pieces;
    a.by_pieces = Divisor::of((uint32_t)l.pieces);
    a.c = v.temperature == 0.0 ? 0.0 : 1.4426950408889634 / v.temperature;
    a.span = v.temperature == 0.0 ? 0.0 : 1000.0 / a.c;
    a.stats = reinterpret_cast<double2*>(w);
    a.left = reinterpret_cast<double2*>(w + l.left);
    a.row = reinterpret_cast<double4*>(w + l.row);
    a.end = reinterpret_cast<int2*>(w + l.end);
    a.before = v.B > kManySequences ? reinterpret_cast<int2*>(w + l.before) : nullptr;
    auto run = [&](auto len) {
        constexpr int LEN = decltype(len)::value;
        if (v.bf16) launch<uint16_t, LEN>(a, stream);
        else launch<float, LEN>(a, stream);
    };
    if (l.len == 1024) run(std::integral_constant<int, 1024>{});
    else run(std::integral_constant<int, 2048>{});
}

}  // namespace puro
