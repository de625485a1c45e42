// The verdict over drafted tokens: the C entry points and the kernels.
//
// A row of target logits is p = softmax(x / T), of draft logits q.  The rows that follow a row are tried in order.  After k of them have failed what is left of p is
//     p_k = max(p - a_k q, 0) / b_k,   a_0 = 0, b_0 = 1,   a_k+1 = a_k + b_k,   b_k+1 = sum max(p - a_k+1 q, 0)
// (where p_k is positive, p_k - q = (p - (a_k + b_k) q) / b_k, and elsewhere both are cut), so that a failure costs one look at p and q and nothing is stored.  A draft
// with token t stays if u q(t) b_k < max(p(t) - a_k q(t), 0).  Without draft logits p_k is p without the failed tokens and b_k what they leave of its sum.
//
// All of it is in 64 bits, the temperatures too: a verdict compares two numbers, and the token that follows is looked for among 150000 sums that lie 1e-5 apart.
//
//   k_verify_sums   largest logit and sum of exponentials of every part of every row          (the whole chip, all logits once)
//   k_verify_rows   the verdict after every row, a wave each; with draft logits, of its first draft
//   k_verify_left   b_k of the rows whose first k drafts have failed, k = 1 .. width - 1        (draft logits and trees only)
//   k_verify_close  the verdicts that wait for them                                            (draft logits and trees only)
//   k_verify_draw   the walk through the rows that stay, by every block alike, and the sum of one part of the row that the next token is drawn from
//   k_verify_pick   the part, and in it the token; a block a sequence
#include <algorithm>
#include <cmath>
#include <new>

#include "checks.h"
#include "st_device.h"

namespace st {

constexpr int kSumPart = 8192, kSumPartSmall = 2048;  // logits of a part of k_verify_sums
constexpr int kDrawPart = 4096;                       // of k_verify_draw and k_verify_left
constexpr int kVerifyRows = 1024;                     // most rows of a sequence
constexpr int kVerifyWidth = 64;                      // most rows that follow one (a lane each)
constexpr int kVerifySpans = ST_KV4_MAX_SPANS;

// Sequences of a call, by value: no copy to the device precedes the kernels, and a captured launch keeps them
struct VerifySpans {
    int32_t n;
    int32_t first[kVerifySpans + 1];  // their first rows among the call's
    double heat[kVerifySpans];
};
// A part of a row: its largest logit and where it is (greedy sequences), or the sum of 2^((x c - base) / 256), c = 256 / (T ln 2), base the whole number nearest to the largest
// x c: products with c are never rounded, and parts of different bases differ by a power of 2^(1/256).  From 2^50 on (logits of 1e13 temperatures, and masks of a type's lowest number)
// a base is the rounded product itself; any other logit of the type is 2^26 units away and more, 2^-24 of such a product, and weighs nothing.  sum: NaN where some logit is, or (T > 0) is +infinity
struct VerifyPart {
    double base, sum;
    float top;
    int32_t at;
};
// A row: its distribution p(x) = 2^((x c - p_base) / 256) / p_sum, q alike, and the verdict over the rows that follow it
struct VerifyRow {
    double p_base, p_sum, q_base, q_sum;
    double a;        // p's weights are max(p - a q, 0) once all drafts have failed
    int32_t stays;   // row of the sequence, -1: none, kOpen: not known yet
    int32_t drafts;  // that follow it, of which as many as may be tried; without draft logits those that failed
    int32_t best;    // greedy: the largest logit's token
    int32_t good;    // it is a distribution
};
constexpr int kOpen = -2;
// A draft after a row
struct VerifyDraft {
    double u, p, q;  // its random number, its probabilities
    int32_t row, token;
};
struct VerifyArgs {
    const int32_t *parent, *tokens;
    const void *target, *draft;
    int64_t target_stride, draft_stride;
    const double *accept, *sample;
    int32_t vocab, sum_parts, draw_parts, rows, width;
    VerifyPart *part;     // [target | draft][rows][sum_parts]
    VerifyRow *row;       // [rows]
    VerifyDraft *drafts;  // [rows][width]
    double *left;         // [width - 1][rows][draw_parts]
    double *weight;       // [sequence][draw_parts]
    int32_t *end;         // [sequence]: the row that the next token is drawn from, -1: none is drawn
    int32_t *path, *accepted, *next;
    int32_t path_stride;
};
struct Verify {
    st_verify_config c;
    int32_t draw_parts;
    VerifyPart *part;
    VerifyRow *row;
    VerifyDraft *drafts;
    double *left, *weight;
    int32_t *end;
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

constexpr int kTable = 256;  // powers of 2 that are tabulated: 2^(i / kTable)

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
__device__ __forceinline__ double units_of(double heat) { return kTable * 1.4426950408889634074 / heat; }  // c: logits to 1/256 of a power of 2
// Whether a base leaves x c - base as it is; else a weight is 1 where the products are the same, and 0 (the difference would be the product's rounding, of any size)
__device__ __forceinline__ bool is_exact(double base) { return fabs(base) < 0x1p50; }
__device__ __forceinline__ double weight_from(float x, double c, double base) { return rint((double)x * c) == base ? 1.0 : 0.0; }
__device__ __forceinline__ double power_of(float x, double c, double base) {
    return is_exact(base) ? exp2_64(fma((double)x, c, -base) * (1.0 / kTable)) : weight_from(x, c, base);
}

// The same for many numbers, off by less than 2.5e-14 of it and not at all at the table's own, in eight instructions of 64 bits and three others: powers of 2^(1/256) from a table in LDS times a third-degree
// polynomial (the series of e^x, |x| <= r = ln 2 / 512, with x^4 replaced by 2 (sqrt 2 - 1) r^2 x^2, which it is nearest to: off by 0.172 r^4 / 24 = 2.4e-14), the exponent added to the
// number's upper half.  (A sum of 1.5 * 2^52 and a number has the rounded number in its low bits.)  A table of 64 needs the fourth degree and one instruction more for
// its index, which is no byte.
struct Exp2Table {
    const uint2 *two;  // as fill_table leaves them
    double c, base, shift;
    __device__ __forceinline__ Exp2Table(const uint2 *table, double units, double b) : two(table), c(units), base(b), shift(6755399441055744.0 - b) {}
    // y and g with y * g = 2^((x c - base) / 256); x c - base is above -256000 and not above 1
    __device__ __forceinline__ double power(float x, double &g) const {
        constexpr double l = 0.69314718055994530942 / kTable, r = l / 2;
        const double v = (double)x, k = fma(v, c, shift), f = fma(v, c, -(k - shift));
        const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, k);
        double p = l * l * l / 6;
        p = fma(p, f, l * l * (0.5 + 0.82842712474619009760 * r * r / 24));
        p = fma(p, f, l);
        g = fma(p, f, 1.0);
        const uint2 half = two[n & (kTable - 1)];
        const uint32_t upper = half.y + (n << 12);
        return __builtin_bit_cast(double, (uint64_t)upper << 32 | half.x);
    }
    __device__ __forceinline__ bool small(float x) const { return !(fma((double)x, c, -base) > -1000.0 * kTable); }
    __device__ __forceinline__ double any(float x) const {  // of any x; 0 below 2^-1000
        if (!exact()) return weight_from(x, c, base);
        if (small(x)) return 0.0;
        double g;
        const double y = power(x, g);
        return y * g;
    }
    __device__ __forceinline__ bool exact() const { return is_exact(base); }
};
// 2^(i / 256) as its halves, the upper one less i << 12: with n << 12 added, n = 256 e + i, it is 2^e times as large
struct Exp2Powers {
    uint2 at[kTable];
};
constexpr Exp2Powers exp2_powers() {
    Exp2Powers t{};
    for (int i = 0; i < kTable; ++i) {
        const double x = i * (0.69314718055994530942 / kTable);
        double p = 1.0;
        for (int k = 24; k; --k) p = 1.0 + p * x / k;  // the series of e^x
        const uint64_t bits = __builtin_bit_cast(uint64_t, p);
        t.at[i].x = (uint32_t)bits, t.at[i].y = (uint32_t)(bits >> 32) - ((uint32_t)i << 12);
    }
    return t;
}
__constant__ constexpr Exp2Powers kPowers = exp2_powers();
__device__ __forceinline__ void fill_table(uint2 *two) {  // followed by a barrier
    if (threadIdx.x < kTable) two[threadIdx.x] = kPowers.at[threadIdx.x];
}

// Sums over a wave by lane moves without LDS (see wave_sum)
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_move64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROW_MASK, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROW_MASK, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum64(double v) {
    v += dpp_move64<0xB1, 0xf>(v);
    v += dpp_move64<0x4E, 0xf>(v);
    v += dpp_move64<0x141, 0xf>(v);
    v += dpp_move64<0x140, 0xf>(v);
    v += dpp_move64<0x142, 0xa>(v);
    v += dpp_move64<0x143, 0xc>(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = __builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_max64(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d, kWave));
    return v;
}
__device__ __forceinline__ double wave_prefix64(double v) {  // inclusive
    v += dpp_move64<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8: within rows of 16
    v += dpp_move64<0x112, 0xf>(v);
    v += dpp_move64<0x114, 0xf>(v);
    v += dpp_move64<0x118, 0xf>(v);
    v += dpp_move64<0x142, 0xa>(v);  // the last lane of row 0 (2) to row 1 (3), of row 1 to rows 2 and 3
    v += dpp_move64<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ double lane64(double v, int lane) {  // of a wave-uniform lane
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int wave_min_int(int v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = min(v, __shfl_xor(v, d, kWave));
    return v;
}
template <int WAVES = 4>
__device__ __forceinline__ double block_sum64(double v, double *sums) {  // sums: a number of LDS for each wave
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    if constexpr (WAVES == 8) v += (sums[4] + sums[5]) + (sums[6] + sums[7]);
    return v;
}
__device__ __forceinline__ int span_of_row(const VerifySpans &t, int row) {
    const int lane = threadIdx.x & 63;
    return __builtin_amdgcn_readfirstlane(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < t.n && t.first[lane] <= row)) - 1);
}

// A part of a row of logits in the registers of 256 threads: vectors i, i + 256, ... of 16 bytes.  Rows may start anywhere: parts are cut at multiples of 16 bytes of the
// address, and vectors that are not wholly in the row are read number by number.
template <class L, int PART>
struct PartOf {
    static constexpr int E = L::kPer16, N = PART / E / 256;
    const typename L::type *p;
    int mis, x0, vocab;  // numbers between the last multiple of 16 bytes and the row; the part's first number (may lie before the row)
    __device__ __forceinline__ PartOf(const void *logits, int64_t stride, int row, int part, int v) {
        p = static_cast<const typename L::type *>(logits) + row * stride;
        mis = (int)(((uintptr_t)p & 15) / sizeof(typename L::type));
        x0 = part * PART - mis, vocab = v;
    }
    __device__ __forceinline__ int first(int i) const { return x0 + (i * 256 + (int)threadIdx.x) * E; }
    __device__ __forceinline__ void load(float (&x)[N][E]) const {  // what is not in the row: -infinity
        if (x0 >= 0 && x0 + PART <= vocab) {
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
//
// The vector pipe bounds it: eight instructions of 64 bits (as fast here as those of 32) and some six others a logit.  256 rows of 152064 bf16 logits and 159 of a draft, 126 MB:
// 42 us, 3.0 TB/s; 336 and 240 rows of 152064 fp32 logits, 350 MB: 61 us, 5.7 TB/s, more than a large copy reaches.  Parts of 4096 logits cost nothing, of
// 2048 20 % (the table is filled in every block); six and eight waves a SIMD spill (+12 and +24 %); a polynomial off by 4e-11 is not near enough (a verdict on what is left of
// a difference goes wrong).
// ---------------------------------------------------------------------------------------
template <class L, int PART>
__global__ __launch_bounds__(256, 4) void k_verify_sums(const VerifySpans t, const VerifyArgs a) {
    const bool is_draft = (int)blockIdx.y >= a.rows;
    const int row = blockIdx.y - (is_draft ? a.rows : 0), part = blockIdx.x, tid = threadIdx.x, wave = tid >> 6;
    const int j = span_of_row(t, row);
    const double heat = t.heat[j];
    if (is_draft && (heat == 0.0 || !has_followers(a.parent, t.first[j], t.first[j + 1] - t.first[j], row - t.first[j]))) return;
    __shared__ float tops[4];
    __shared__ double sums[4];
    __shared__ uint2 two[kTable];
    __shared__ int lowest[4];
    typedef PartOf<L, PART> P;
    const P at = is_draft ? P(a.draft, a.draft_stride, row, part, a.vocab) : P(a.target, a.target_stride, row, part, a.vocab);
    float x[P::N][P::E];
    at.load(x);
    fill_table(two);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < P::N; ++i)
#pragma unroll
        for (int e = 0; e < P::E; ++e) top = __builtin_elementwise_maximum(top, x[i][e]);  // NaN where one is (wave_max passes it over)
    const bool nan = top != top;
    top = wave_max(top);
    if ((tid & 63) == 0) tops[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    double sum = nan ? (double)NAN : 0.0;
    int low = INT32_MAX;
    double base = -1e300;  // of a part without numbers
    if (heat > 0.0) {
        const double c = units_of(heat);
        if (top == INFINITY) {
            sum = (double)NAN;
        } else if (top > -INFINITY) {
            base = rint((double)top * c);
            const Exp2Table ex(two, c, base);
            float low = top;
#pragma unroll
            for (int i = 0; i < P::N; ++i)
#pragma unroll
                for (int e = 0; e < P::E; ++e) low = fminf(low, x[i][e]);
            if (!ex.exact()) {
#pragma unroll
                for (int i = 0; i < P::N; ++i)
#pragma unroll
                    for (int e = 0; e < P::E; ++e) sum += x[i][e] == top ? 1.0 : 0.0;
            } else if (__builtin_amdgcn_ballot_w64(ex.small(low)) == 0) {
#pragma unroll
                for (int i = 0; i < P::N; ++i)
#pragma unroll
                    for (int e = 0; e < P::E; ++e) {
                        double g;
                        const double y = ex.power(x[i][e], g);
                        sum = fma(y, g, sum);
                    }
            } else {  // some are masked, or not in the row
#pragma unroll
                for (int i = 0; i < P::N; ++i)
#pragma unroll
                    for (int e = 0; e < P::E; ++e) {
                        double g;
                        const bool none = ex.small(x[i][e]);
                        const double y = ex.power(none ? top : x[i][e], g);
                        sum = fma(y, none ? 0.0 : g, sum);
                    }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < P::N; ++i)
#pragma unroll
            for (int e = 0; e < P::E; ++e)
                if (x[i][e] == top) low = min(low, at.first(i) + e);
        low = wave_min_int(low);
        if ((tid & 63) == 0) lowest[wave] = low;
    }
    sum = block_sum64(sum, sums);
    if (tid == 0)
        a.part[(size_t)blockIdx.y * a.sum_parts + part] =
            VerifyPart{base, sum, top, heat > 0.0 ? 0 : min(min(lowest[0], lowest[1]), min(lowest[2], lowest[3]))};
}

// A row from its parts, by one wave
struct RowSum {
    double base, sum;
    int at;     // greedy: the largest number's token
    bool good;  // it is a distribution (greedy: it has a largest number)
};
__device__ __forceinline__ RowSum row_sum(const VerifyPart *part, int parts, double heat) {
    const int lane = threadIdx.x & 63;
    constexpr VerifyPart none{-1e300, 0.0, -INFINITY, INT32_MAX};
    const VerifyPart p0 = lane < parts ? part[lane] : none, p1 = lane + 64 < parts ? part[lane + 64] : none;
    float top = fmaxf(p0.top, p1.top);
    double sum = 0.0;
    if (heat == 0.0) {
        for (int i = lane + 128; i < parts; i += 64) top = fmaxf(top, part[i].top);
        top = wave_max(top);
        int at = INT32_MAX;
        auto add = [&](const VerifyPart &p) {
            if (p.top == top) at = min(at, p.at);
            sum += p.sum;  // 0, or NaN
        };
        add(p0), add(p1);
        for (int i = lane + 128; i < parts; i += 64) add(part[i]);
        sum = wave_sum64(sum);
        return RowSum{0.0, sum, wave_min_int(at), sum == sum && top > -INFINITY};
    }
    double base = fmax(p0.base, p1.base);
    for (int i = lane + 128; i < parts; i += 64) base = fmax(base, part[i].base);
    base = wave_max64(base);
    auto add = [&](const VerifyPart &p) { sum += p.sum * exp2_64((p.base - base) * (1.0 / kTable)); };
    add(p0), add(p1);
    for (int i = lane + 128; i < parts; i += 64) add(part[i]);
    sum = wave_sum64(sum);
    return RowSum{base, sum, 0, sum == sum && base > -1e299};
}

// ---------------------------------------------------------------------------------------
// Rows.  A wave is one row: its distribution from the parts, the rows that follow it (a lane each, 64 rows at a time) with their tokens' probabilities, and the verdict -- with
// draft logits, of the first of them.  A chain of dependent loads (parts, tokens, their logits): 5.9 us for 336 rows.
// ---------------------------------------------------------------------------------------
template <class L>
__device__ __forceinline__ VerifyRow row_verdict(const VerifyArgs &a, int first, int rows, int local, double heat) {
    typedef typename L::type X;
    const int row = first + local, lane = threadIdx.x & 63;
    const bool draws = a.draft && heat > 0.0;
    // the first 64 rows behind it, which is where what follows it mostly is: asked for beside the parts
    const X *pr = static_cast<const X *>(a.target) + row * a.target_stride, *qr = static_cast<const X *>(a.draft) + row * a.draft_stride;
    struct Near {
        int token;
        double u;
        float x, y;
        uint64_t follow;
    };
    auto look = [&](int c0) {
        const int child = c0 + lane;
        Near n{-1, 0.0, -INFINITY, -INFINITY, 0};
        const bool follows = child < rows && (a.parent ? a.parent[first + child] == local : child == local + 1);
        n.follow = __builtin_amdgcn_ballot_w64(follows);
        if (follows) {
            n.token = a.tokens[first + child], n.u = a.accept[first + child];
            if (n.token >= 0 && n.token < a.vocab) {
                n.x = L::get(pr[n.token]);
                if (draws) n.y = L::get(qr[n.token]);
            }
        }
        return n;
    };
    Near near = look(local + 1);
    const RowSum p = row_sum(a.part + (size_t)row * a.sum_parts, a.sum_parts, heat);
    RowSum q{0.0, 1.0, 0, true};
    const double c = heat > 0.0 ? units_of(heat) : 0.0;
    int stays = -1, drafts = 0, failed_token = -1;  // lane i: token of draft i that failed
    bool good = p.good, have_q = false;
    double rest = p.sum;  // what the failed tokens leave of the sum, without draft logits
    for (int c0 = local + 1; c0 < rows && good && stays < 0 && drafts < a.width; c0 += 64) {
        if (c0 != local + 1) near = look(c0);
        if (!near.follow) {
            if (!a.parent) break;
            continue;
        }
        if (draws && !have_q) {
            q = row_sum(a.part + (size_t)(a.rows + row) * a.sum_parts, a.sum_parts, heat);
            good = q.good, have_q = true;
            if (!good) break;
        }
        const bool known = near.token >= 0 && near.token < a.vocab;
        double pt = known && heat > 0.0 ? power_of(near.x, c, p.base) : 0.0;
        const double qt = known && draws ? power_of(near.y, c, q.base) / q.sum : 0.0;
        if (draws) pt /= p.sum;
        for (uint64_t bits = near.follow; bits && drafts < a.width && stays < 0; bits &= bits - 1) {
            const int l = __builtin_ctzll(bits), token = __builtin_amdgcn_readlane(near.token, l);
            const bool in = token >= 0 && token < a.vocab;
            if (heat == 0.0) {
                if (in && token == p.at) stays = c0 + l;
            } else if (draws) {
                if (drafts == 0 && in && lane64(near.u, l) * lane64(qt, l) < lane64(pt, l)) stays = c0 + l;
                if (a.width > 1 && lane == l) a.drafts[(size_t)row * a.width + drafts] = VerifyDraft{near.u, pt, qt, c0 + l, near.token};
            } else {
                const bool again = __builtin_amdgcn_ballot_w64(lane < drafts && failed_token == token) != 0;
                const double pl = lane64(pt, l);
                if (in && !again && lane64(near.u, l) * rest < pl) {
                    stays = c0 + l;
                } else {
                    if (lane == drafts) failed_token = token;
                    if (in && !again) rest -= pl;
                    if (rest < p.sum * 0x1p-10) {  // little is left of a difference: summed up instead (once in a thousand failures)
                        rest = 0.0;
                        for (int x = lane; x < a.vocab; x += 64) {
                            bool out = false;
                            for (int f = 0; f <= drafts; ++f) out |= __builtin_amdgcn_readlane(failed_token, f) == x;
                            if (!out) rest += power_of(L::get(pr[x]), c, p.base);
                        }
                        rest = wave_sum64(rest);
                    }
                }
            }
            drafts += stays < 0 || draws;
        }
    }
    if (!draws && heat > 0.0 && lane < drafts) a.drafts[(size_t)row * a.width + lane].token = failed_token;
    return VerifyRow{p.base, p.sum, q.base, q.sum, draws && drafts > 0 && stays < 0 ? 1.0 : 0.0, stays < 0 && good && draws && drafts > 1 ? kOpen : stays, drafts, p.at, good};
}

template <class L>
__global__ __launch_bounds__(64) void k_verify_rows(const VerifySpans t, const VerifyArgs a) {
    const int row = blockIdx.x, j = span_of_row(t, row), first = t.first[j];
    const VerifyRow r = row_verdict<L>(a, first, t.first[j + 1] - first, row - first, t.heat[j]);
    if (threadIdx.x == 0) a.row[row] = r;
}

// max(p - a q, 0), p and q given by factors.  Powers and sums are off by up to 2.5e-14 each, so that p and q of one distribution may differ by 1e-13 of themselves: as much of p
// is left out, or what is left of it less itself would be drawn from their rounding.  (Written as the one fused instruction it is, so that every place that asks gets the same number.)
constexpr double kSure = 1.0 - 0x1p-42;
__device__ __forceinline__ double left_of(double p, double p_of, double q, double q_of) { return fmax(fma(p, p_of, -(q * q_of)), 0.0); }

// The verdict over drafts 1 .. known - 1 of an open row, whose b_k have been summed; by one wave.  a: as they leave it
__device__ __forceinline__ int judge_on(const VerifyArgs &args, int row, int known, double &a) {
    const int lane = threadIdx.x & 63;
    for (int k = 1; k < known; ++k) {
        const VerifyDraft d = args.drafts[(size_t)row * args.width + k];
        const double *part = args.left + ((size_t)(k - 1) * args.rows + row) * args.draw_parts;
        double b = 0.0;
        for (int i = lane; i < args.draw_parts; i += 64) b += part[i];
        b = wave_sum64(b);
        if (d.token >= 0 && d.token < args.vocab && d.u * d.q * b < left_of(d.p, kSure, d.q, a)) return d.row;
        a += b;
    }
    return -1;
}

// The weights of a row: p, or p without tokens that have failed, or max(p - a q, 0); parts of kDrawPart of them, kOwn neighbouring ones to each of 256 threads
constexpr int kOwn = kDrawPart / 256;
template <class L>
struct Weights {
    typedef typename L::type X;
    const X *p, *q;
    const uint2 *two;
    double c, p_base, p_of, q_base, q_of;  // q_of 0: without q
    const VerifyDraft *failed;
    int n_failed, vocab;
    __device__ __forceinline__ Weights(const VerifyArgs &a, int row, const VerifyRow &r, const uint2 *table, double heat, double by, bool plain) {
        p = static_cast<const X *>(a.target) + row * a.target_stride, q = static_cast<const X *>(a.draft) + row * a.draft_stride;
        two = table, c = units_of(heat), p_base = r.p_base, q_base = r.q_base, q_of = plain ? 0.0 : by / r.q_sum, p_of = (q_of > 0.0 ? kSure : 1.0) / r.p_sum;
        failed = a.drafts + (size_t)row * a.width, n_failed = plain || a.draft ? 0 : r.drafts, vocab = a.vocab;
    }
    __device__ __forceinline__ int first(int part) const { return part * kDrawPart + (int)threadIdx.x * kOwn; }  // of this thread
    __device__ __forceinline__ double one(int x) const {  // of any token
        if (x >= vocab) return 0.0;
        for (int f = 0; f < n_failed; ++f)
            if (failed[f].token == x) return 0.0;
        const double w = Exp2Table(two, c, p_base).any(L::get(p[x]));
        return q_of > 0.0 ? left_of(w, p_of, Exp2Table(two, c, q_base).any(L::get(q[x])), q_of) : w * p_of;
    }
    static constexpr int E = L::kPer16, N = kOwn / E;
    template <int N>
    static __device__ __forceinline__ void load(const X *at, int there, float (&x)[N][E]) {  // what is not there: -infinity
        if (there < N * E) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = i * E + e < there ? L::get(at[i * E + e]) : -INFINITY;
        } else if ((uintptr_t)at & 15) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = L::get(at[i * E + e]);
        } else {
            u32x4 v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const u32x4 *>(at + i * E);
#pragma unroll
            for (int i = 0; i < N; ++i) L::spread(v[i], x[i]);
        }
    }
    // The sum of this thread's, from its registers: with two logits a token masked ones (and rows' ends) go vector by vector, since both forms side by side take 144 registers
    // (4 trees of 64 rows 88 us instead of 82); masked they take 108, and 177 token by token.  Parts of 2048 logits: 84 us, 16 trees of 12 rows 62 instead of 64.
    __device__ __forceinline__ double own(int part) const {
        const int x0 = first(part), there = min(vocab - x0, kOwn);
        const Exp2Table ep(two, c, p_base), eq(two, c, q_base);
        double sum = 0.0;
        if (there <= 0) return sum;
        if (!ep.exact() || !eq.exact()) {
            for (int i = 0; i < there; ++i) sum += one(x0 + i);
        } else if (q_of > 0.0) {
            float x[N][E], y[N][E], low = INFINITY, low_q = INFINITY;
            load(p + x0, there, x), load(q + x0, there, y);
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) low = fminf(low, x[i][e]), low_q = fminf(low_q, y[i][e]);
            if (!ep.small(low) && !eq.small(low_q)) {
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        double g, h;
                        const double u = ep.power(x[i][e], g), z = eq.power(y[i][e], h);
                        sum += left_of(u * g, p_of, z * h, q_of);
                    }
            } else {  // some are masked, or not there: vector by vector, for the registers' sake
#pragma unroll 1
                for (int i = 0; i < N; ++i) {
                    float v[1][E], w[1][E];
                    load(p + x0 + i * E, there - i * E, v), load(q + x0 + i * E, there - i * E, w);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        double g, h;
                        const double u = ep.power(v[0][e], g), z = eq.power(w[0][e], h);
                        sum += left_of(ep.small(v[0][e]) ? 0.0 : u * g, p_of, eq.small(w[0][e]) ? 0.0 : z * h, q_of);
                    }
                }
            }
        } else {
            float x[N][E];
            load(p + x0, there, x);
            uint32_t out = 0;  // the thread's tokens that have failed
            for (int f = 0; f < n_failed; ++f) {
                const uint32_t d = (uint32_t)(failed[f].token - x0);
                out |= d < kOwn ? 1u << d : 0u;
            }
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    double g;
                    const double u = ep.power(x[i][e], g);
                    sum += ep.small(x[i][e]) || (out >> (i * E + e) & 1) ? 0.0 : u * p_of * g;
                }
        }
        return sum;
    }
};

// ---------------------------------------------------------------------------------------
// Left: b_k of one part of one row.  Rows whose verdict is known, or that have no more drafts, return.  7.1 us for 256 rows of 152064 bf16 logits, of which those still
// open are read; one after the other for each k, since a_k is known only when b_k-1 is.
// ---------------------------------------------------------------------------------------
template <class L>
__global__ __launch_bounds__(256) void k_verify_left(const VerifySpans t, const VerifyArgs a, int k) {
    const int row = blockIdx.y, part = blockIdx.x;
    const VerifyRow r = a.row[row];
    if (r.stays != kOpen || r.drafts <= k) return;
    __shared__ double sums[4];
    __shared__ uint2 two[kTable];
    fill_table(two);
    double by = r.a;
    if (judge_on(a, row, k, by) >= 0) return;  // (every wave on its own, with the same result)
    __syncthreads();
    const double sum = block_sum64(Weights<L>(a, row, r, two, t.heat[span_of_row(t, row)], by, false).own(part), sums);
    if (threadIdx.x == 0) a.left[((size_t)(k - 1) * a.rows + row) * a.draw_parts + part] = sum;
}

__global__ __launch_bounds__(64) void k_verify_close(const VerifyArgs a) {
    VerifyRow &r = a.row[blockIdx.x];
    if (r.stays != kOpen) return;
    double by = r.a;
    const int stays = judge_on(a, blockIdx.x, r.drafts, by);
    if (threadIdx.x == 0) r.stays = stays, r.a = by;
}

// ---------------------------------------------------------------------------------------
// Draw.  Every block of a sequence walks through the rows that stay (one load, then steps in LDS), and sums up one part of the weights at the end of the walk; the first
// one writes the path.  7.8 us for 16 sequences of 21 rows of 152064 logits, 9.1 with the verdicts of 5 rows: the walk and one part a block, dependent loads.
// ---------------------------------------------------------------------------------------
// FUSED: of few rows the verdicts too, by every block alike, in the place of k_verify_rows.
constexpr int kFusedRows = 8;
template <class L, bool FUSED>
__global__ __launch_bounds__(FUSED ? 64 * kFusedRows : 256) void k_verify_draw(const VerifySpans t, const VerifyArgs a) {
    const int j = blockIdx.y, part = blockIdx.x, tid = threadIdx.x;
    const int first = t.first[j], rows = t.first[j + 1] - first;
    __shared__ int stays[FUSED ? kFusedRows : kVerifyRows], path[FUSED ? kFusedRows : kVerifyRows];
    __shared__ int end_of, count_of;
    __shared__ double sums[FUSED ? kFusedRows : 4];
    __shared__ uint2 two[kTable];
    __shared__ VerifyRow own[FUSED ? kFusedRows : 1];
    if constexpr (FUSED) {
        const int i = tid >> 6;  // a wave a row
        if (i < rows) {
            const VerifyRow r = row_verdict<L>(a, first, rows, i, t.heat[j]);
            if ((tid & 63) == 0) own[i] = r, stays[i] = r.stays;
        }
    } else {
        for (int i = tid; i < rows; i += 256) stays[i] = a.row[first + i].stays;
    }
    fill_table(two);
    __syncthreads();
    if (tid == 0) {
        int at = 0, n = 0;
        for (int next = stays[0]; next >= 0; next = stays[at]) path[n++] = at = next;  // (a row that stays lies behind the row it follows)
        end_of = at, count_of = n;
    }
    __syncthreads();
    const int end = first + end_of, count = count_of;
    const VerifyRow r = FUSED ? own[end_of] : a.row[end];
    const double heat = t.heat[j];
    const bool drawn = heat > 0.0 && r.good;
    if (part == 0) {
        for (int i = tid; i < a.path_stride; i += 256) a.path[(int64_t)j * a.path_stride + i] = i < count ? path[i] : -1;
        if (tid == 0) {
            a.accepted[j] = count, a.end[j] = drawn ? end : -1;
            if (FUSED) a.row[end] = r;  // for k_verify_pick
            if (!drawn) a.next[j] = r.good ? r.best : -1;
        }
    }
    if (!drawn) return;
    double sum = tid < 256 ? Weights<L>(a, end, r, two, heat, r.a, false).own(part) : 0.0;
    sum = block_sum64<FUSED ? kFusedRows : 4>(sum, sums);
    if (tid == 0) a.weight[(size_t)j * a.draw_parts + part] = sum;
}

// ---------------------------------------------------------------------------------------
// Pick: the first token at which the running sum of the weights passes sample * their sum.  The part first, by every wave alike; in it a thread has neighbouring
// tokens, so that the sums run from thread to thread; and of the thread that passes, its tokens, a lane each.  Where rounding lets none pass, the last with a weight.
// 5.5 us for one sequence, 7.5 for 16: three dependent reads and the scans between them.
// ---------------------------------------------------------------------------------------
// The first of 64 lanes at which the running sum of v passes the goal, or the last with a v; -1: there is none.  before: in the sum before the lanes, out before that one
__device__ __forceinline__ int passing_lane(double v, double goal, double &before, bool &passes) {
    const double sum = before + wave_prefix64(v);
    const uint64_t some = __builtin_amdgcn_ballot_w64(v > 0.0), over = __builtin_amdgcn_ballot_w64(sum > goal && v > 0.0);
    passes = over != 0;
    const int l = over ? __builtin_ctzll(over) : some ? 63 - __builtin_clzll(some) : -1;
    before = lane64(sum - v, l < 0 ? 63 : l);
    return l;
}

template <class L>
__global__ __launch_bounds__(256) void k_verify_pick(const VerifySpans t, const VerifyArgs a) {
    const int j = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, end = a.end[j];
    if (end < 0) return;
    double *weights = a.weight + (size_t)j * a.draw_parts;
    __shared__ double sums[4], before_of;
    __shared__ uint2 two[kTable];
    __shared__ int thread_of[4];
    fill_table(two);
    __syncthreads();
    const VerifyRow r = a.row[end];
    double total = 0.0;
    for (int i = lane; i < a.draw_parts; i += 64) total += weights[i];
    total = wave_sum64(total);
    const bool plain = !(total > 0.0);  // rounding has left nothing: p itself (rare)
    const Weights<L> w(a, end, r, two, t.heat[j], r.a, plain);
    if (plain) {
        for (int i = 0; i < a.draw_parts; ++i) {
            const double s = block_sum64(w.own(i), sums);
            if (tid == 0) __hip_atomic_store(weights + i, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            total += s;
            __syncthreads();
        }
    }
    auto weight = [&](int i) {
        if (i >= a.draw_parts) return 0.0;
        return plain ? __hip_atomic_load(weights + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : weights[i];
    };
    const double goal = a.sample[j] * total;
    double before = 0.0, before_it = 0.0;
    int part = -1;  // the part that passes the goal, or the last one with a weight; and the sum before it
    bool passes = false;
    for (int i0 = 0; i0 < a.draw_parts && !passes; i0 += 64) {
        const double v = weight(i0 + lane), all = before + wave_sum64(v);
        const int l = passing_lane(v, goal, before, passes);
        if (l >= 0) part = i0 + l, before_it = before;
        before = all;
    }
    if (part < 0) {  // no weight anywhere: not a distribution after all
        if (tid == 0) a.next[j] = -1;
        return;
    }
    const double own = w.own(part), wave_all = wave_sum64(own);
    __syncthreads();
    if (lane == 0) sums[wave] = wave_all;
    __syncthreads();
    before = before_it;
    for (int v = 0; v < wave; ++v) before += sums[v];
    const int l = passing_lane(own, goal, before, passes);
    if (lane == 0) thread_of[wave] = l < 0 ? -1 : (passes ? 256 : 0) + wave * 64 + l;  // (256 on: it passes)
    __syncthreads();
    int best = -1;
    for (int v = 3; v >= 0; --v)  // the first wave that passes, else the last one with a weight
        if (thread_of[v] >= 256 || (best < 0 && thread_of[v] >= 0)) best = thread_of[v];
    if (best < 0) best = 0;
    if ((best & 255) == tid) before_of = lane64(before, 0);
    __syncthreads();
    if (wave) return;
    before = before_of;
    const int first = part * kDrawPart + (best & 255) * kOwn;
    const int at = passing_lane(lane < kOwn ? w.one(first + lane) : 0.0, goal, before, passes);
    if (lane == 0) a.next[j] = first + (at < 0 ? 0 : at);
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
// (a row's first part may start up to 7 numbers before it)
static int parts_of(int vocab, int part) { return (vocab + 7 + part - 1) / part; }

static void carve(const st_verify_config &c, char *ws, Verify *v, size_t *bytes) {
    size_t off = 0;
    auto take = [&](size_t n) {
        char *p = ws ? ws + off : nullptr;
        off += up256(n);
        return p;
    };
    v->c = c;
    v->draw_parts = (c.vocab + kDrawPart - 1) / kDrawPart;
    const size_t rows = c.max_rows;
    v->part = reinterpret_cast<VerifyPart *>(take(sizeof(VerifyPart) * 2 * rows * parts_of(c.vocab, kSumPartSmall)));
    v->row = reinterpret_cast<VerifyRow *>(take(sizeof(VerifyRow) * rows));
    v->drafts = reinterpret_cast<VerifyDraft *>(take(sizeof(VerifyDraft) * rows * c.max_width));
    v->left = reinterpret_cast<double *>(take(sizeof(double) * (c.max_width - 1) * rows * v->draw_parts));
    v->weight = reinterpret_cast<double *>(take(sizeof(double) * kVerifySpans * v->draw_parts));
    v->end = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * kVerifySpans));
    *bytes = off;
}

template <class L>
static void launch_verify(const Verify &v, const VerifySpans &t, VerifyArgs a, bool all_greedy) {
    const bool draws = a.draft && !all_greedy;
    const int planes = draws ? 2 * a.rows : a.rows, large = parts_of(a.vocab, kSumPart);
    // Smaller parts while larger ones would not give every compute unit two blocks.  us small : large, one sequence of 5 rows, 1024 logits 16.8 : 18.8, 151936 (190 large
    // parts) 18.4 : 19.1, 20 rows (760) 24.8 : 24.0; 4 sequences of 5 rows (760) 22.4 : 22.1, 8 of 8 rows without draft logits (1216) 30.6 : 29.5
    const bool small = (int64_t)planes * large < 512;
    a.sum_parts = small ? parts_of(a.vocab, kSumPartSmall) : large;
    auto *sums = small ? k_verify_sums<L, kSumPartSmall> : k_verify_sums<L, kSumPart>;
    hipLaunchKernelGGL(sums, dim3(a.sum_parts, planes), dim3(256), 0, v.stream, t, a);
    int longest = 0;
    for (int j = 0; j < t.n; ++j) longest = std::max(longest, t.first[j + 1] - t.first[j]);
    const bool looks = draws && a.width > 1;
    // The verdicts by every block of the draw where they are a row a wave and there is a compute unit for every block, instead of a launch of their own.  us fused : not, one
    // sequence of 5 rows, 1024 logits 17.9 : 20.4, 151936 19.2 : 20.4; 16 sequences of 5 rows 42.3 : 41.3, 64 of 4 rows 92.9 : 77.9.
    const bool fused = !looks && longest <= kFusedRows && (int64_t)a.draw_parts * t.n <= 256;
    if (!fused) hipLaunchKernelGGL(k_verify_rows<L>, dim3(a.rows), dim3(64), 0, v.stream, t, a);
    if (looks) {
        for (int k = 1; k < a.width; ++k) hipLaunchKernelGGL(k_verify_left<L>, dim3(a.draw_parts, a.rows), dim3(256), 0, v.stream, t, a, k);
        hipLaunchKernelGGL(k_verify_close, dim3(a.rows), dim3(64), 0, v.stream, a);
    }
    auto *draw = fused ? k_verify_draw<L, true> : k_verify_draw<L, false>;
    hipLaunchKernelGGL(draw, dim3(all_greedy ? 1 : a.draw_parts, t.n), dim3(fused ? 64 * kFusedRows : 256), 0, v.stream, t, a);
    if (!all_greedy) hipLaunchKernelGGL(k_verify_pick<L>, dim3(t.n), dim3(256), 0, v.stream, t, a);
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

int st_verify_drafts64(st_verify *h, const int32_t *rows, int32_t n, const st_draft_tree *tree, const int32_t *tokens, const void *target,
                       int64_t target_stride, const void *draft, int64_t draft_stride, const double *temperature, const double *accept,
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
        if (!(temperature[j] >= 0.0) || std::isinf(temperature[j])) return fail(ST_EINVAL, "sequence %d: bad temperature", j);
        t.first[j] = (int32_t)total;
        t.heat[j] = temperature[j] > 0.0 ? std::max(temperature[j], 0x1p-800) : 0.0;  // (products with 1 / T stay finite; any two logits are far apart by then)
        all_greedy = all_greedy && temperature[j] == 0.0;
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
    const VerifyArgs a{tree ? tree->parent : nullptr, tokens, target, draft, target_stride, draft_stride, accept, sample, v->c.vocab, 0, v->draw_parts,
                       (int32_t)total, tree ? tree->width : 1, v->part, v->row, v->drafts, v->left, v->weight, v->end, path, accepted, next, path_stride};
    if (v->c.dtype == ST_F32) launch_verify<LogitF32>(*v, t, a, all_greedy);
    else if (v->c.dtype == ST_BF16) launch_verify<LogitBf16>(*v, t, a, all_greedy);
    else launch_verify<LogitF16>(*v, t, a, all_greedy);
    return launched("st_verify_drafts", hipGetLastError());
}

int st_verify_drafts(st_verify *h, const int32_t *rows, int32_t n, const st_draft_tree *tree, const int32_t *tokens, const void *target,
                     int64_t target_stride, const void *draft, int64_t draft_stride, const float *temperature, const double *accept,
                     const double *sample, int32_t *path, int32_t path_stride, int32_t *accepted, int32_t *next) {
    double heat[kVerifySpans];
    for (int j = 0; temperature && j < n && j < kVerifySpans; ++j) heat[j] = temperature[j];
    return st_verify_drafts64(h, rows, n, tree, tokens, target, target_stride, draft, draft_stride, temperature ? heat : nullptr, accept, sample, path,
                              path_stride, accepted, next);
}

}  // extern "C"
