// The verdict over drafted tokens: the C entry points and the kernels.
//
// A row of target logits is p = softmax(x / T), of draft logits q.  The rows that follow a row are tried in order.  After k of them have failed what is left of p is
//     p_k = max(p - a_k q, 0) / b_k,   a_0 = 0, b_0 = 1,   a_k+1 = a_k + b_k,   b_k+1 = sum max(p - a_k+1 q, 0)
// (where p_k is positive, p_k - q = (p - (a_k + b_k) q) / b_k, and elsewhere both are cut), so that a failure costs one look at p and q and nothing is stored.  A draft
// with token t stays if u q(t) b_k < max(p(t) - a_k q(t), 0).  Without draft logits p_k is p without the failed tokens and b_k what they leave of its sum.
//
// All of it is in 64 bits: a verdict compares two numbers, and the token that follows is looked for among 150000 sums that lie 1e-5 apart.  Vector instructions of 64 bits
// run at the rate of plain 32-bit ones here, and the exponential is 15 of them.
//
//   k_verify_sums     largest logit and sum of exponentials of every part of every row            (the whole chip, all logits once)
//   k_verify_left     b_k of the rows whose first k drafts have failed, k = 1 .. width - 1          (drafts with logits and trees only)
//   k_verify_walk     the verdicts of all rows at once, then the walk through them; a block a sequence
//   k_verify_weights  sums of the parts of the row that the next token is drawn from
//   k_verify_pick     the part, and in it the token; a block a sequence
#include <algorithm>
#include <cmath>
#include <new>

#include "checks.h"
#include "st_device.h"

namespace st {

constexpr int kVerifyPart = 8192;      // logits of a part
constexpr int kVerifyRows = 1024;      // most rows of a sequence
constexpr int kVerifyWidth = 64;       // most rows that follow one (a lane each)
constexpr int kVerifySpans = ST_KV4_MAX_SPANS;

// Sequences of a call, by value: no copy to the device precedes the kernels, and a captured launch keeps them
struct VerifySpans {
    int32_t n;
    int32_t first[kVerifySpans + 1];  // their first rows among the call's
    float heat[kVerifySpans];
};
// A part of a row: its largest logit, where it is, and the sum of exp((x - top) / T); NaN where some logit is, or (T > 0) is +infinity
struct VerifyPart {
    float top;
    int32_t at;
    double sum;
};
// The row that a sequence's next token is drawn from
struct VerifyEnd {
    int32_t row;     // among the call's rows, -1: there is no token
    int32_t failed;  // drafts after it that failed, their tokens (without draft logits)
    double a;        // p's weights are max(p - a q, 0)
    double p_top, p_sum, q_top, q_sum;
    int32_t tokens[kVerifyWidth];
};
struct VerifyArgs {
    const int32_t *parent, *tokens;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const double *accept, *sample;
    int32_t vocab, parts, rows, width;
    VerifyPart *part;  // [target | draft][rows][parts]
    double *left;      // [width - 1][rows][parts]
    double *weight;    // [sequence][parts]
    VerifyEnd *end;    // [sequence]
    int32_t *path, *accepted, *next;
    int32_t path_stride;
};
struct Verify {
    st_verify_config c;
    int32_t parts;
    VerifyPart *part;
    double *left, *weight;
    VerifyEnd *end;
    hipStream_t stream;
};

struct LogitF32 {
    typedef float type;
    static constexpr int kPer16 = 4;
    static __device__ __forceinline__ float get(type x) { return x; }
    static __device__ __forceinline__ void spread(const u32x4 &w, float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
};
struct LogitBf16 {
    typedef uint16_t type;
    static constexpr int kPer16 = 8;
    static __device__ __forceinline__ float get(type x) { return bf16_to_f32(x); }
    static __device__ __forceinline__ void spread(const u32x4 &w, float *x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
    }
};
struct LogitF16 {
    typedef _Float16 type;
    static constexpr int kPer16 = 8;
    static __device__ __forceinline__ float get(type x) { return (float)x; }
    static __device__ __forceinline__ void spread(const u32x4 &w, float *x) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t word = w[i];  // (a bit cast of the element itself reads the vector's first one)
            const f16x2 h = __builtin_bit_cast(f16x2, word);
            x[2 * i] = (float)h.x, x[2 * i + 1] = (float)h.y;
        }
    }
};

// 2^t for t <= 0, off by less than 2e-14 of it: 2^n times the series of e^x, |x| <= ln 2 / 2, to its eleventh power
__device__ __forceinline__ double exp2_64(double t) {
    t = fmax(t, -2000.0);
    const double n = rint(t), x = (t - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800.0;
    p = fma(p, x, 1.0 / 3628800.0);
    p = fma(p, x, 1.0 / 362880.0);
    p = fma(p, x, 1.0 / 40320.0);
    p = fma(p, x, 1.0 / 5040.0);
    p = fma(p, x, 1.0 / 720.0);
    p = fma(p, x, 1.0 / 120.0);
    p = fma(p, x, 1.0 / 24.0);
    p = fma(p, x, 1.0 / 6.0);
    p = fma(p, x, 0.5);
    p = fma(p, x, 1.0);
    p = fma(p, x, 1.0);
    return ldexp(p, (int)n);
}
__device__ __forceinline__ double per_log2(float heat) { return 1.4426950408889634074 / (double)heat; }  // (x - top) / T as a power of 2
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, kWave);
    return v;
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d, kWave));
    return v;
}
__device__ __forceinline__ int span_of_row(const VerifySpans &t, int row) {
    const int lane = threadIdx.x & 63;
    return __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < t.n && t.first[lane] <= row)) - 1);
}

// A part of a row of logits in registers: thread i has vectors i, i + 256, ... of 16 bytes.  Rows may start anywhere: parts are cut at multiples of 16 bytes of the
// address, and vectors that are not wholly in the row are read number by number.
template <class L>
struct PartOf {
    static constexpr int E = L::kPer16, N = kVerifyPart / E / 256;
    const typename L::type *p;
    int mis, x0, vocab;  // numbers between the last multiple of 16 bytes and the row; the part's first number (may lie before the row)
    __device__ __forceinline__ PartOf(const void *logits, int64_t stride, int row, int part, int v) {
        p = static_cast<const typename L::type *>(logits) + row * stride;
        mis = (int)(((uintptr_t)p & 15) / sizeof(typename L::type));
        x0 = part * kVerifyPart - mis, vocab = v;
    }
    __device__ __forceinline__ int first(int i) const { return x0 + (i * 256 + (int)threadIdx.x) * E; }
    __device__ __forceinline__ void load(float (&x)[N][E]) const {  // what is not in the row: -infinity
        if (x0 >= 0 && x0 + kVerifyPart <= vocab) {
            u32x4 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const u32x4 *>(p + first(i));
#pragma unroll
            for (int i = 0; i < N; ++i) L::spread(w[i], x[i]);
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int a = first(i);
            if (a >= 0 && a + E <= vocab) {
                L::spread(*reinterpret_cast<const u32x4 *>(p + a), x[i]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = a + e >= 0 && a + e < vocab ? L::get(p[a + e]) : -INFINITY;
            }
        }
    }
    // the same numbers of another row (the draft's): its rows may start elsewhere within 16 bytes
    __device__ __forceinline__ void load_of(const void *logits, int64_t stride, int row, int part, float (&x)[N][E]) const {
        const PartOf other(logits, stride, row, part, vocab);
        if (other.mis == mis) return other.load(x);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = first(i) + e;
                x[i][e] = at >= 0 && at < vocab ? L::get(other.p[at]) : -INFINITY;
            }
    }
};

// Whether a row follows another: lanes of a wave look together
__device__ __forceinline__ bool has_followers(const int32_t *parent, int first, int rows, int local) {
    if (!parent) return local + 1 < rows;
    bool any = false;
    for (int c0 = local + 1; c0 < rows && !any; c0 += 64) {
        const int c = c0 + (threadIdx.x & 63);
        any = __builtin_amdgcn_ballot_w64(c < rows && parent[first + c] == local) != 0;
    }
    return any;
}

// ---------------------------------------------------------------------------------------
// Sums.  A block is one part of one row; the part stays in registers between its largest number and its sum.  Draft rows that nothing follows, and those of greedy
// sequences, are not read.
// ---------------------------------------------------------------------------------------
template <class L>
__global__ __launch_bounds__(256) void k_verify_sums(const VerifySpans t, const VerifyArgs a) {
    const bool is_draft = (int)blockIdx.y >= a.rows;
    const int row = blockIdx.y - (is_draft ? a.rows : 0), part = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
    const int j = span_of_row(t, row);
    const float heat = t.heat[j];
    if (is_draft && (heat == 0.f || !has_followers(a.parent, t.first[j], t.first[j + 1] - t.first[j], row - t.first[j]))) return;
    typedef PartOf<L> P;
    const P at = is_draft ? P(a.draft, a.draft_stride, row, part, a.vocab) : P(a.target, a.target_stride, row, part, a.vocab);
    float x[P::N][P::E];
    at.load(x);
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int e = 0; e < P::E; ++e) top = fmaxf(top, x[i][e]), nan |= x[i][e] != x[i][e];
    __shared__ float tops[4];
    __shared__ double sums[4];
    __shared__ int lowest[4];
    top = wave_max(top);
    if ((tid & 63) == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    double sum = nan ? (double)NAN : 0.0;
    int low = INT32_MAX;
    if (heat > 0.f) {
        const double c = per_log2(heat), base = top == -INFINITY ? 0.0 : (double)top;
#pragma unroll
        for (int i = 0; i < P::N; ++i)
#pragma unroll
            for (int e = 0; e < P::E; ++e) sum += exp2_64(((double)x[i][e] - base) * c);
        if (top == INFINITY) sum = (double)NAN;
    } else {
#pragma unroll
        for (int i = 0; i < P::N; ++i)
#pragma unroll
            for (int e = 0; e < P::E; ++e)
                if (x[i][e] == top) low = min(low, at.first(i) + e);
#pragma unroll
        for (int d = 32; d; d >>= 1) low = min(low, __shfl_xor(low, d, kWave));
    }
    sum = wave_sum64(sum);
    if ((tid & 63) == 0) sums[wave] = sum, lowest[wave] = low;
    __syncthreads();
    if (tid == 0)
        a.part[(size_t)blockIdx.y * a.parts + part] =
            VerifyPart{top, min(min(lowest[0], lowest[1]), min(lowest[2], lowest[3])), (sums[0] + sums[1]) + (sums[2] + sums[3])};
}

// A row from its parts, by one wave: largest logit, where, sum of exponentials below it
struct RowSum {
    double top, sum;
    int at;
    bool good;  // it is a distribution (heat 0: it has a largest number)
};
__device__ __forceinline__ RowSum row_sum(const VerifyPart *part, int parts, float heat) {
    const int lane = threadIdx.x & 63;
    float top = -INFINITY;
    for (int i = lane; i < parts; i += 64) top = fmaxf(top, part[i].top);
    top = wave_max(top);
    const double c = heat > 0.f ? per_log2(heat) : 0.0;
    double sum = 0.0;
    int at = INT32_MAX;
    for (int i = lane; i < parts; i += 64) {
        const VerifyPart p = part[i];
        if (p.top == top) at = min(at, p.at);
        if (heat > 0.f) sum += p.top == -INFINITY ? p.sum : p.sum * exp2_64(((double)p.top - (double)top) * c);
        else sum += p.sum;  // 0, or NaN
    }
    sum = wave_sum64(sum);
#pragma unroll
    for (int d = 32; d; d >>= 1) at = min(at, __shfl_xor(at, d, kWave));
    return RowSum{(double)top, sum, at, sum == sum && top > -INFINITY};
}

// The verdicts after one row, by one wave.  With draft logits only the first `known` drafts can be judged (b_1 .. b_known-1 have been summed).
struct Verdict {
    int stays;       // the row that stays (of the sequence), -1: none
    int next;        // drafts judged; where it is `known`, there are more
    bool more, good;
    double a;
    int failed, token;  // without draft logits: tokens that failed, lane i the i-th
    RowSum p, q;
};
template <class L>
__device__ __forceinline__ Verdict judge(const VerifyArgs &a, int first, int rows, int local, float heat, int known) {
    typedef typename L::type X;
    const int lane = threadIdx.x & 63, row = first + local;
    Verdict v{-1, 0, false, true, 0.0, 0, -1, {}, {}};
    v.p = row_sum(a.part + (size_t)row * a.parts, a.parts, heat);
    v.good = v.p.good;
    const bool with_q = a.draft && heat > 0.f;
    const X *pr = static_cast<const X *>(a.target) + row * a.target_stride, *qr = static_cast<const X *>(a.draft) + row * a.draft_stride;
    const double c = heat > 0.f ? per_log2(heat) : 0.0;
    bool have_q = false;
    double b = 1.0, rest = v.p.sum;  // rest: what the failed tokens leave of the sum, without draft logits
    for (int c0 = local + 1; c0 < rows; c0 += 64) {
        const int child = c0 + lane;
        const bool follows = child < rows && (a.parent ? a.parent[first + child] == local : child == local + 1);
        uint64_t bits = __builtin_amdgcn_ballot_w64(follows);
        if (!bits) {
            if (!a.parent) break;
            continue;
        }
        if (with_q && !have_q) {
            v.q = row_sum(a.part + (size_t)(a.rows + row) * a.parts, a.parts, heat);
            v.good = v.good && v.q.good, have_q = true;
        }
        if (!v.good) return v;
        int t = -1;
        double u = 0.0, pt = 0.0, qt = 0.0;
        if (follows) {
            t = a.tokens[first + child], u = a.accept[first + child];
            if (t >= 0 && t < a.vocab) {
                const double x = (double)L::get(pr[t]);
                pt = heat > 0.f ? exp2_64((x - v.p.top) * c) : 0.0;
                if (with_q) pt /= v.p.sum, qt = exp2_64(((double)L::get(qr[t]) - v.q.top) * c) / v.q.sum;
            }
        }
        while (bits) {
            const int l = __builtin_ctzll(bits);
            bits &= bits - 1;
            if (v.next >= a.width) return v;
            if (v.next >= known) {
                v.more = true;
                return v;
            }
            if (with_q && v.next > 0) {  // the sum of what is left
                const double *part = a.left + ((size_t)(v.next - 1) * a.rows + row) * a.parts;
                b = 0.0;
                for (int i = lane; i < a.parts; i += 64) b += part[i];
                b = wave_sum64(b);
            }
            ++v.next;
            const int token = __shfl(t, l, kWave);
            const double ul = __shfl(u, l, kWave), pl = __shfl(pt, l, kWave), ql = __shfl(qt, l, kWave);
            bool stays;
            if (token < 0 || token >= a.vocab) {
                stays = false;
            } else if (heat == 0.f) {
                stays = token == v.p.at;
            } else if (with_q) {
                stays = ul * ql * b < fmax(pl - v.a * ql, 0.0);
            } else {
                const bool again = __builtin_amdgcn_ballot_w64(lane < v.failed && v.token == token) != 0;
                stays = !again && ul * rest < pl;
                if (!stays && !again) rest -= pl;
                if (!stays && lane == v.failed) v.token = token;
                v.failed += !stays;
            }
            if (stays) {
                v.stays = c0 + l;
                return v;
            }
            if (with_q) v.a += b;
        }
    }
    return v;
}

// ---------------------------------------------------------------------------------------
// Left: b_k of one part of one row.  Rows whose verdict is known, or that have no more drafts, return.
// ---------------------------------------------------------------------------------------
template <class L>
__global__ __launch_bounds__(256) void k_verify_left(const VerifySpans t, const VerifyArgs a, int k) {
    const int row = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, j = span_of_row(t, row);
    const float heat = t.heat[j];
    if (heat == 0.f) return;
    const int first = t.first[j], rows = t.first[j + 1] - first;
    if (!has_followers(a.parent, first, rows, row - first)) return;
    const Verdict v = judge<L>(a, first, rows, row - first, heat, k);  // (every wave on its own, with the same result)
    if (!v.more) return;
    typedef PartOf<L> P;
    const P at(a.target, a.target_stride, row, part, a.vocab);
    const double c = per_log2(heat), p_of = 1.0 / v.p.sum, q_of = v.a / v.q.sum;
    double sum = 0.0;
    float x[P::N][P::E], y[P::N][P::E];
    at.load(x);
    at.load_of(a.draft, a.draft_stride, row, part, y);
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int e = 0; e < P::E; ++e)
            sum += fmax(exp2_64(((double)x[i][e] - v.p.top) * c) * p_of - exp2_64(((double)y[i][e] - v.q.top) * c) * q_of, 0.0);
    __shared__ double sums[4];
    sum = wave_sum64(sum);
    if ((tid & 63) == 0) sums[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) a.left[((size_t)(k - 1) * a.rows + row) * a.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// ---------------------------------------------------------------------------------------
// Walk: a wave judges every sixteenth row of a sequence, then one thread follows the rows that stay.
// ---------------------------------------------------------------------------------------
template <class L>
__global__ __launch_bounds__(1024) void k_verify_walk(const VerifySpans t, const VerifyArgs a) {
    const int j = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int first = t.first[j], rows = t.first[j + 1] - first;
    const float heat = t.heat[j];
    __shared__ int stays[kVerifyRows];
    __shared__ int end, count;
    for (int r = wave; r < rows; r += 16) {
        const Verdict v = judge<L>(a, first, rows, r, heat, kVerifyWidth);
        if (lane == 0) stays[r] = v.stays;
    }
    __syncthreads();
    int32_t *path = a.path + (int64_t)j * a.path_stride;
    if (tid == 0) {
        int at = 0, n = 0;
        while (stays[at] >= 0) at = stays[at], path[n++] = at;  // (a row that stays lies behind the row it follows)
        end = at, count = n;
        a.accepted[j] = n;
    }
    __syncthreads();
    for (int i = count + tid; i < a.path_stride; i += 1024) path[i] = -1;
    if (wave) return;
    const Verdict v = judge<L>(a, first, rows, end, heat, kVerifyWidth);  // once more for what it leaves
    if (heat == 0.f || !v.good) {
        if (lane == 0) a.end[j].row = -1, a.next[j] = v.good ? v.p.at : -1;
        return;
    }
    a.end[j].tokens[lane] = v.token;
    if (lane == 0) {
        VerifyEnd &e = a.end[j];
        e.row = first + end, e.failed = v.failed, e.a = v.a;
        e.p_top = v.p.top, e.p_sum = v.p.sum, e.q_top = v.q.top, e.q_sum = v.q.sum;
    }
}

// The weights of one part of a sequence's last row, from which its next token is drawn.  plain: p itself, whatever failed.
template <class L>
__device__ __forceinline__ void end_weights(const VerifyArgs &a, const VerifyEnd &e, float heat, bool plain, const PartOf<L> &at, int part,
                                            double (&w)[PartOf<L>::N][PartOf<L>::E]) {
    typedef PartOf<L> P;
    const double c = per_log2(heat), p_top = e.p_top, p_of = 1.0 / e.p_sum;
    float x[P::N][P::E];
    at.load(x);
    for (int f = 0; f < e.failed && !plain; ++f) {
        const int token = e.tokens[f];
        if (token < at.x0 || token >= at.x0 + kVerifyPart) continue;
#pragma unroll
        for (int i = 0; i < P::N; ++i)
#pragma unroll
            for (int k = 0; k < P::E; ++k)
                if (at.first(i) + k == token) x[i][k] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int k = 0; k < P::E; ++k) w[i][k] = exp2_64(((double)x[i][k] - p_top) * c) * p_of;
    if (plain || !(e.a > 0.0)) return;
    const double q_top = e.q_top, q_of = e.a / e.q_sum;
    at.load_of(a.draft, a.draft_stride, e.row, part, x);
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int k = 0; k < P::E; ++k) w[i][k] = fmax(w[i][k] - exp2_64(((double)x[i][k] - q_top) * c) * q_of, 0.0);
}

// ---------------------------------------------------------------------------------------
// Weights: the sum of one part
// ---------------------------------------------------------------------------------------
template <class L>
__global__ __launch_bounds__(256) void k_verify_weights(const VerifySpans t, const VerifyArgs a) {
    typedef PartOf<L> P;
    const int j = blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
    const VerifyEnd &e = a.end[j];
    if (e.row < 0) return;
    const P at(a.target, a.target_stride, e.row, part, a.vocab);
    double w[P::N][P::E], sum = 0.0;
    end_weights<L>(a, e, t.heat[j], false, at, part, w);
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int k = 0; k < P::E; ++k) sum += w[i][k];
    __shared__ double sums[4];
    sum = wave_sum64(sum);
    if ((tid & 63) == 0) sums[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) a.weight[(size_t)j * a.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// ---------------------------------------------------------------------------------------
// Pick: the first token at which the running sum of the weights passes sample * their sum.  Parts first, by every wave alike; in the part the sums of 64 vectors
// (a wave's share of one load), and of those the one that passes, number by number.  Where rounding lets none pass, the last token with a weight.
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_prefix64(double v) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double x = __shfl_up(v, d, kWave);
        if (lane >= d) v += x;
    }
    return v;
}

template <class L>
__global__ __launch_bounds__(256) void k_verify_pick(const VerifySpans t, const VerifyArgs a) {
    typedef PartOf<L> P;
    const int j = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const VerifyEnd &e = a.end[j];
    if (e.row < 0) return;
    const float heat = t.heat[j];
    const double c = per_log2(heat);
    double total = 0.0;
    for (int i = lane; i < a.parts; i += 64) total += a.weight[(size_t)j * a.parts + i];
    total = wave_sum64(total);
    const bool plain = !(total > 0.0);  // rounding has left nothing: p itself
    auto part_weight = [&](int i) {
        if (i >= a.parts) return 0.0;
        if (!plain) return a.weight[(size_t)j * a.parts + i];
        const VerifyPart p = a.part[(size_t)e.row * a.parts + i];
        return p.top == -INFINITY ? 0.0 : p.sum * exp2_64(((double)p.top - e.p_top) * c) / e.p_sum;
    };
    if (plain) {
        total = 0.0;
        for (int i = lane; i < a.parts; i += 64) total += part_weight(i);
        total = wave_sum64(total);
    }
    double goal = a.sample[j] * total, before = 0.0;
    int part = -1, full = -1;  // the part that passes the goal; the last one with a weight, and the sum before it
    double before_full = 0.0;
    for (int i0 = 0; i0 < a.parts && part < 0; i0 += 64) {
        const double v = part_weight(i0 + lane), sum = before + wave_prefix64(v);
        const uint64_t passes = __builtin_amdgcn_ballot_w64(sum > goal && v > 0.0), some = __builtin_amdgcn_ballot_w64(v > 0.0);
        const int l = passes ? __builtin_ctzll(passes) : some ? 63 - __builtin_clzll(some) : 0;
        const double at_l = __shfl(sum - v, l, kWave);
        if (passes) part = i0 + l, before_full = at_l;
        else if (some) full = i0 + l, before_full = at_l;
        before = __shfl(sum, 63, kWave);
    }
    if (part < 0) part = full;
    if (part < 0) {  // no weight anywhere: not a distribution after all
        if (tid == 0) a.next[j] = -1;
        return;
    }
    goal -= before_full;
    const P at(a.target, a.target_stride, e.row, part, a.vocab);
    double w[P::N][P::E], own[P::N];
    end_weights<L>(a, e, heat, plain, at, part, w);
    __shared__ double sums[P::N][4];
    __shared__ int chosen[4], final_one[4];
#pragma unroll
    for (int i = 0; i < P::N; ++i) {
        own[i] = 0.0;
#pragma unroll
        for (int k = 0; k < P::E; ++k) own[i] += w[i][k];
        const double s = wave_sum64(own[i]);
        if (lane == 0) sums[i][wave] = s;
    }
    __syncthreads();
    double run = 0.0;
    int first = INT32_MAX, latest = -1;
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const double s = sums[i][v];
            if (v == wave && s > 0.0) {
                double x = run + (wave_prefix64(own[i]) - own[i]);
#pragma unroll
                for (int k = 0; k < P::E; ++k) {
                    x += w[i][k];
                    if (w[i][k] > 0.0) {
                        latest = max(latest, at.first(i) + k);
                        if (x > goal) first = min(first, at.first(i) + k);
                    }
                }
            }
            run += s;
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) first = min(first, __shfl_xor(first, d, kWave)), latest = max(latest, __shfl_xor(latest, d, kWave));
    if (lane == 0) chosen[wave] = first, final_one[wave] = latest;
    __syncthreads();
    if (tid) return;
    first = min(min(chosen[0], chosen[1]), min(chosen[2], chosen[3]));
    latest = max(max(final_one[0], final_one[1]), max(final_one[2], final_one[3]));
    a.next[j] = first != INT32_MAX ? first : latest;
}

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
static int check_config(const st_verify_config *c) {
    if (!c) return fail(ST_EINVAL, "config is NULL");
    if (c->vocab <= 0 || c->vocab > 1 << 24) return fail(ST_EINVAL, "vocab must be from 1 to 2^24");
    if (c->dtype != ST_BF16 && c->dtype != ST_F16 && c->dtype != ST_F32) return fail(ST_EINVAL, "dtype must be ST_BF16, ST_F16 or ST_F32");
    if (c->max_rows <= 0 || c->max_rows > 32767) return fail(ST_EINVAL, "max_rows must be from 1 to 32767");  // (a grid has 65535 blocks in y)
    if (c->max_width <= 0 || c->max_width > kVerifyWidth) return fail(ST_EINVAL, "max_width must be from 1 to %d", kVerifyWidth);
    return ST_OK;
}
static void carve(const st_verify_config &c, char *ws, Verify *v, size_t *bytes) {
    size_t off = 0;
    auto take = [&](size_t n) {
        char *p = ws ? ws + off : nullptr;
        off += up256(n);
        return p;
    };
    v->c = c;
    v->parts = (c.vocab + 7 + kVerifyPart - 1) / kVerifyPart;  // (a row's first part may start up to 7 numbers before it)
    const size_t row = (size_t)c.max_rows * v->parts;
    v->part = reinterpret_cast<VerifyPart *>(take(sizeof(VerifyPart) * 2 * row));
    v->left = reinterpret_cast<double *>(take(sizeof(double) * (c.max_width - 1) * row));
    v->weight = reinterpret_cast<double *>(take(sizeof(double) * kVerifySpans * v->parts));
    v->end = reinterpret_cast<VerifyEnd *>(take(sizeof(VerifyEnd) * kVerifySpans));
    *bytes = off;
}

template <class L>
static void launch_verify(const Verify &v, const VerifySpans &t, const VerifyArgs &a, bool all_greedy) {
    const bool draft = a.draft && !all_greedy;
    hipLaunchKernelGGL(k_verify_sums<L>, dim3(a.parts, draft ? 2 * a.rows : a.rows), dim3(256), 0, v.stream, t, a);
    for (int k = 1; draft && k < a.width; ++k) hipLaunchKernelGGL(k_verify_left<L>, dim3(a.parts, a.rows), dim3(256), 0, v.stream, t, a, k);
    hipLaunchKernelGGL(k_verify_walk<L>, dim3(t.n), dim3(1024), 0, v.stream, t, a);
    if (all_greedy) return;
    hipLaunchKernelGGL(k_verify_weights<L>, dim3(a.parts, t.n), dim3(256), 0, v.stream, t, a);
    hipLaunchKernelGGL(k_verify_pick<L>, dim3(t.n), dim3(256), 0, v.stream, t, a);
}

}  // namespace st

using namespace st;

extern "C" {

int st_verify_query_sizes(const st_verify_config *cfg, size_t *workspace_bytes) {
    if (int rc = check_config(cfg)) return rc;
    Verify v;
    size_t bytes;
    carve(*cfg, nullptr, &v, &bytes);
    if (workspace_bytes) *workspace_bytes = bytes;
    return ST_OK;
}

int st_verify_create(const st_verify_config *cfg, void *workspace, size_t workspace_bytes, void *stream, st_verify **out) {
    if (!out) return fail(ST_EINVAL, "out is NULL");
    *out = nullptr;
    if (int rc = check_config(cfg)) return rc;
    if (!workspace) return fail(ST_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace & 255) return fail(ST_EINVAL, "workspace must be 256-byte aligned");
    Verify *v = new (std::nothrow) Verify();
    if (!v) return fail(ST_ENOMEM, "out of host memory");
    size_t bytes;
    carve(*cfg, (char *)workspace, v, &bytes);
    if (workspace_bytes < bytes) {
        delete v;
        return fail(ST_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, bytes);
    }
    v->stream = (hipStream_t)stream;
    *out = reinterpret_cast<st_verify *>(v);
    return ST_OK;
}

void st_verify_destroy(st_verify *h) { delete reinterpret_cast<Verify *>(h); }

int st_verify_drafts(st_verify *h, const int32_t *rows, int32_t n, const st_draft_tree *tree, const int32_t *tokens, const void *target,
                     int64_t target_stride, const void *draft, int64_t draft_stride, const float *temperature, const double *accept,
                     const double *sample, int32_t *path, int32_t path_stride, int32_t *accepted, int32_t *next) {
    const Verify *v = reinterpret_cast<const Verify *>(h);
    if (!v) return fail(ST_EINVAL, "verifier is NULL");
    if (n < 0 || n > kVerifySpans) return fail(ST_EINVAL, "%d sequences, 0 to %d are supported", n, kVerifySpans);
    if (!n) return ST_OK;
    if (!rows || !temperature) return fail(ST_EINVAL, "rows or temperature is NULL");
    VerifySpans t{};
    int64_t total = 0;
    bool all_greedy = true;
    t.n = n;
    for (int j = 0; j < n; ++j) {
        if (rows[j] < 1 || rows[j] > kVerifyRows) return fail(ST_ERANGE, "sequence %d: %d rows, 1 to %d are supported", j, rows[j], kVerifyRows);
        if (rows[j] > path_stride) return fail(ST_ERANGE, "sequence %d: %d rows, path_stride is %d", j, rows[j], path_stride);
        if (!(temperature[j] >= 0.f) || std::isinf(temperature[j])) return fail(ST_EINVAL, "sequence %d: bad temperature", j);
        t.first[j] = (int32_t)total;
        t.heat[j] = temperature[j];
        all_greedy = all_greedy && temperature[j] == 0.f;
        total += rows[j];
        if (total > v->c.max_rows) return fail(ST_ERANGE, "%lld rows or more, max_rows is %d", (long long)total, v->c.max_rows);
    }
    t.first[n] = (int32_t)total;
    if (tree) {
        if (!tree->parent || (uintptr_t)tree->parent & 3) return fail(ST_EINVAL, "tree: parent is NULL or not aligned to 4 bytes");
        if (tree->width < 1 || tree->width > v->c.max_width) return fail(ST_EINVAL, "tree: width %d, 1 to max_width %d are supported", tree->width, v->c.max_width);
    }
    const size_t size = v->c.dtype == ST_F32 ? 4 : 2;
    if (!tokens || !target || !accept || !sample || !path || !accepted || !next) return fail(ST_EINVAL, "an array is NULL");
    if (((uintptr_t)tokens | (uintptr_t)path | (uintptr_t)accepted | (uintptr_t)next) & 3) return fail(ST_EINVAL, "tokens, path, accepted or next is not aligned to 4 bytes");
    if (((uintptr_t)accept | (uintptr_t)sample) & 7) return fail(ST_EINVAL, "accept or sample is not aligned to 8 bytes");
    if (((uintptr_t)target | (uintptr_t)draft) & (size - 1)) return fail(ST_EINVAL, "target or draft is not aligned to its numbers");
    if (target_stride < v->c.vocab || (draft && draft_stride < v->c.vocab)) return fail(ST_EINVAL, "a row stride is less than vocab %d", v->c.vocab);
    const VerifyArgs a{tree ? tree->parent : nullptr, tokens, target, draft, target_stride, draft_stride, accept, sample, v->c.vocab, v->parts, (int32_t)total,
                       tree ? tree->width : 1, v->part, v->left, v->weight, v->end, path, accepted, next, path_stride};
    if (v->c.dtype == ST_F32) launch_verify<LogitF32>(*v, t, a, all_greedy);
    else if (v->c.dtype == ST_BF16) launch_verify<LogitBf16>(*v, t, a, all_greedy);
    else launch_verify<LogitF16>(*v, t, a, all_greedy);
    return launched("st_verify_drafts", hipGetLastError());
}

}  // extern "C"
