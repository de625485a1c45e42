// Attention over the key/value cache in pages: causal, or for drafted rows that each see the context and their own branch.
//
// The query heads of a kv head are folded into columns: column i * G + h is row i of head h.  With S^T = K Q^T (slots x columns) a lane holds one column, so the
// softmax is register arithmetic and P^T is the second product's operand as it stands: O^T = V^T P^T.  Scores, maxima, sums and outputs are fp32; the weights
// enter the second product in 16 bits (the largest so far as 1, in fp16 as 2^15 where numbers 2^-29 of it are still whole), as the framework's other attention does.
//
// What a column sees of a tile is a word of bits: all of the context, of the span's own rows the first i + 1 or those that `sees` names, nothing of a hole and
// nothing past the end.  It is only made where some column does not see all of the tile ("part").  There the values are looked through as well: an infinity or NaN
// times a weight of zero would reach columns that do not see it, so such numbers are multiplied as zeros, and added to the columns that see them.
#include <algorithm>
#include <atomic>
#include <utility>

#include "checks.h"
#include "paged.h"
#include "st_device.h"

namespace st {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Bits of slots key0 .. key0 + 63 that row `row` of a span sees, holes aside
__device__ __forceinline__ uint64_t seen_bits(const uint64_t *__restrict__ sees, int words, int len, int rows, int row0, int row, int key0) {
    const int j0 = key0 - len;  // the span's row in slot key0
    auto below = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1ull; };  // the first n bits
    if (!sees) return below(row + 1 - j0);
    if (j0 <= -64) return ~0ull;
    const uint64_t *w = sees + (int64_t)(row0 + row) * words;
    uint64_t own;
    if (j0 <= 0) {
        own = below(-j0) | w[0] << -j0;
    } else {
        const int i = j0 >> 6, s = j0 & 63;
        own = i < words ? w[i] >> s : 0ull;
        if (s && i + 1 < words) own |= w[i + 1] << (64 - s);
    }
    return own & below(rows - j0);
}

// Weights are 2^(s c - base), c = log2(e) / sqrt(D), base the product of c and the largest score s so far (less kRaise), rounded: one multiply-add each.  What rounding base takes away is the same
// for all weights, and cancels; but from 2^22 on (scores no trained model has) it could be powers of two, from 2^31 on enough for weights of 0 or infinity.  There every
// product is rounded as base is before base is taken from it, so that the largest score's weight is 1 (or 2^kRaise) again, and
// base is 0 from then on.  Asking costs a tile of k_paged_chunk 2 %: 177.4 us without and 181.0 with, 2048 rows on 2048 slots.
__device__ __forceinline__ bool is_far(float base) { return fabsf(base) >= 0x1p22f; }
template <class T>
__device__ __forceinline__ float less_far(float s, float scale, float base) {
#pragma clang fp contract(off)
    const float less = s * scale - base;
    return (less > T::kRaise ? T::kRaise : less) / scale;  // (the largest one's rounding may add to what it is raised by)
}

// One column's query: row of the span and head
struct PagedColumn {
    int row, head;
};
__device__ __forceinline__ PagedColumn paged_column(int col, int G, int kvh) { return PagedColumn{col / G, kvh * G + col % G}; }

// ---------------------------------------------------------------------------------------
// Few columns: single tokens and short runs, bound by reading the cache once.
//
// A wave works on its own, on tiles of 32 slots, with NT tiles of 16 columns and no LDS until the end: S^T by 16x16x32 MFMAs whose A rows are slots 8 (m / 4) + 4 t +
// m % 4, so that lane (column, quarter) ends up with the weights of slots 8 quarter .. + 7 -- the B operand of the second product.  Keys are read as the first
// product wants them, 64 bytes of 16 slots an instruction; of eight slots of values a lane reads the D / 16 channels that make its row m of D / 16 products, whole
// slots an instruction, and puts the slots of a channel together by byte permutes.  The next tile's loads are issued before this tile's work, its pages' numbers (wave-uniform, in
// scalar registers) one tile before that.  A block's four waves take every fourth tile of its range and are joined through LDS; ranges are joined by k_paged_join.
//
// One row of 12 / 2 heads of 128 on 4608 slots: 5.6 us for 4.7 MB in 72 blocks of a tile a wave, which is the latency of queries, page numbers, tiles and the join of the
// waves one after the other.  16 sequences of 4 rows of 40 / 8 heads on 3000 slots: 41 us for 197 MB, 4.8 TB/s, memory.  Columns by 32 are 16 to 30 % longer than
// blocks of 128 once a call has more than 32 of them (see the plan), since every group of columns reads the cache again.
// ---------------------------------------------------------------------------------------
constexpr int kFewTile = 32, kFewWaves = 4;

template <class T, int D, int NT, int CAP>
__global__ __launch_bounds__(256, NT == 1 ? 2 : 1) void k_paged_few(const Kv4Spans<CAP> t, const PagedView view, const uint64_t *__restrict__ sees, int words,
                                                      const uint16_t *__restrict__ q, int64_t q_stride, uint16_t *__restrict__ out, int64_t out_stride,
                                                      float *__restrict__ part_o, float *__restrict__ part_ml) {
    constexpr int KS = D / 32, DPL = D / 16, VW = DPL / 2;  // VW: words of values of a slot and lane
    typedef typename T::vec8 vec8;
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, qd = lane >> 4;
    const int nkv = view.nkv, G = view.nq / nkv;
    const int cols = sp.rows * G, n_cb = (cols + 16 * NT - 1) / (16 * NT), local = blockIdx.x - sp.blk0;
    const int kvh = local % nkv, z = local / nkv / n_cb, c0 = local / nkv % n_cb * (16 * NT);  // c0: the block's first column
    const int n_keys = sees ? sp.len + sp.rows : sp.len + min(c0 + 16 * NT - 1, cols - 1) / G + 1, last = n_keys - 1;
    const int n_tiles = (n_keys + kFewTile - 1) / kFewTile;
    const int t_begin = z * sp.per, t_end = min(n_tiles, t_begin + sp.per);
    const int32_t *__restrict__ pages = view.table + (int64_t)sp.seq * view.max_pages;
    const int mask = (1 << view.shift) - 1;
    const int all_see = sees ? sp.len - 1 : sp.len + c0 / G;  // last slot that all of its columns see
    const float scale = 1.4426950408889634f / sqrtf((float)D);

    vec8 qf[NT][KS];
    int row[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const PagedColumn w = paged_column(min(c0 + 16 * c + m16, cols - 1), G, kvh);
        row[c] = w.row;
        const uint16_t *src = q + (int64_t)(sp.row0 + w.row) * q_stride + w.head * D + qd * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[c][s] = __builtin_bit_cast(vec8, *reinterpret_cast<const u32x4 *>(src + 32 * s));
    }
    f32x4 o[NT][DPL];
    float m_i[NT], l_i[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        m_i[c] = -INFINITY, l_i[c] = 0.f;
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[c][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    struct Pages {  // of slots 0-15 and 16-31 of a tile
        int a, b;
    };
    struct Tile {
        u32x4 k[2][KS];
        uint32_t v[8][VW];
        Pages at;
    };
    auto look_up = [&](int tile) {
        const int key0 = tile * kFewTile;
        return Pages{page_of(pages, view.n_pages, min(key0, last) >> view.shift), page_of(pages, view.n_pages, min(key0 + 16, last) >> view.shift)};
    };
    auto load = [&](Tile &x, int tile, Pages at) {
        const int key0 = tile * kFewTile;
        x.at = at;
        const size_t a = ((size_t)max(at.a, 0) * nkv + kvh) << view.shift, b = ((size_t)max(at.b, 0) * nkv + kvh) << view.shift;
        const uint16_t *kp = view.k + (m16 >= 8 ? b : a) * D + qd * 8, *vp = view.v + (qd >= 2 ? b : a) * D + m16 * DPL;
        const bool whole = key0 + kFewTile <= n_keys;
        // (slots past the last one are read as the last, so that no address past it is formed)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int slot = min(key0 + 8 * (m16 >> 2) + 4 * u + (m16 & 3), last) & mask;
#pragma unroll
            for (int s = 0; s < KS; ++s) x.k[u][s] = *reinterpret_cast<const u32x4 *>(kp + slot * D + 32 * s);
        }
        auto value = [&](int j, int slot) {
            if constexpr (VW == 4) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(vp + slot * D);
                x.v[j][0] = w.x, x.v[j][1] = w.y, x.v[j][2] = w.z, x.v[j][3] = w.w;
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(vp + slot * D);
                x.v[j][0] = w.x, x.v[j][1] = w.y;
            }
        };
        if (whole) {
            const int first = (key0 + 8 * qd) & mask;
#pragma unroll
            for (int j = 0; j < 8; ++j) value(j, first + j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) value(j, min(key0 + 8 * qd + j, last) & mask);
        }
    };
    auto work = [&](Tile &x, int tile) {
        const int key0 = tile * kFewTile;
        f32x4 sc[NT][2];
#pragma unroll
        for (int c = 0; c < NT; ++c) sc[c][0] = sc[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int c = 0; c < NT; ++c) sc[c][u] = T::mfma16(__builtin_bit_cast(vec8, x.k[u][s]), qf[c][s], sc[c][u]);
        const bool part = key0 + kFewTile - 1 > all_see || (x.at.a | x.at.b) < 0;
        uint32_t seen[NT];
        bool spoiled = false;
        if (part) {
            const uint32_t held = (x.at.a < 0 ? 0u : 0xffffu) | (x.at.b < 0 ? 0u : 0xffff0000u);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                seen[c] = (uint32_t)seen_bits(sees, words, sp.len, sp.rows, sp.row0, row[c], key0) & held;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!(seen[c] >> (8 * qd + 4 * u + r) & 1)) sc[c][u][r] = -INFINITY;
            }
            uint32_t bad = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) bad |= not_finite<T>(x.v[j][w]);
            spoiled = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
            if (spoiled)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int w = 0; w < VW; ++w) x.v[j][w] &= ~halves_of(not_finite<T>(x.v[j][w]));
        }
        vec8 pf[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            float mx = sc[c][0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[c][u][r]);
            float a, b;
            with_xor16(mx, a, b);
            mx = max_xor32(fmaxf(a, b));
            const float cand = fmaf(mx, scale, -T::kRaise);
            const bool raise = cand > m_i[c];
            const float m_new = raise ? cand : m_i[c];
            float base = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet
            if (__builtin_amdgcn_ballot_w64(raise)) {
                const float corr = raise ? __builtin_amdgcn_exp2f(m_i[c] - base) : 1.0f;
                l_i[c] *= corr;
#pragma unroll
                for (int d = 0; d < DPL; ++d) o[c][d] *= corr;
            }
            m_i[c] = m_new;
            const bool far = is_far(base);
            if (__builtin_amdgcn_ballot_w64(far)) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sc[c][u][r] = far ? less_far<T>(sc[c][u][r], scale, base) : sc[c][u][r];
                base = far ? 0.f : base;
            }
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(fmaf(sc[c][j >> 2][j & 3], scale, -base));
                l_i[c] += p[j];
            }
            pf[c] = __builtin_bit_cast(vec8, u32x4{T::pack(p[0], p[1]), T::pack(p[2], p[3]), T::pack(p[4], p[5]), T::pack(p[6], p[7])});
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            const u32x4 even = {low_halves(x.v[0][w], x.v[1][w]), low_halves(x.v[2][w], x.v[3][w]), low_halves(x.v[4][w], x.v[5][w]), low_halves(x.v[6][w], x.v[7][w])};
            const u32x4 odd = {high_halves(x.v[0][w], x.v[1][w]), high_halves(x.v[2][w], x.v[3][w]), high_halves(x.v[4][w], x.v[5][w]), high_halves(x.v[6][w], x.v[7][w])};
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                o[c][2 * w] = T::mfma16(__builtin_bit_cast(vec8, even), pf[c], o[c][2 * w]);
                o[c][2 * w + 1] = T::mfma16(__builtin_bit_cast(vec8, odd), pf[c], o[c][2 * w + 1]);
            }
        }
        if (spoiled)  // this lane's channels are (4 qd + r) DPL + d
            for (int j = 0; j < kFewTile && key0 + j < n_keys; ++j) {
                const int page = j < 16 ? x.at.a : x.at.b;
                if (page < 0) continue;
                const uint16_t *src = view.v + ((((size_t)page * nkv + kvh) << view.shift) + ((key0 + j) & mask)) * D + 4 * qd * DPL;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int d = 0; d < DPL; d += 2) {
                        const uint32_t w = *reinterpret_cast<const uint32_t *>(src + r * DPL + d), b = not_finite<T>(w);
#pragma unroll
                        for (int c = 0; c < NT; ++c) {
                            if ((b & 0x8000u) && (seen[c] >> j & 1)) o[c][d][r] += T::lo(w);
                            if ((b >> 31) && (seen[c] >> j & 1)) o[c][d + 1][r] += T::hi(w);
                        }
                    }
            }
    };
    Tile a, b;
    int i = t_begin + wave;
    if (i < t_end) {
        load(a, i, look_up(i));
        Pages next = look_up(min(i + kFewWaves, t_end - 1));
        while (true) {
            if (i + kFewWaves < t_end) {
                load(b, i + kFewWaves, next);
                next = look_up(min(i + 2 * kFewWaves, t_end - 1));
            }
            work(a, i);
            i += kFewWaves;
            if (i >= t_end) break;
            if (i + kFewWaves < t_end) {
                load(a, i + kFewWaves, next);
                next = look_up(min(i + 2 * kFewWaves, t_end - 1));
            }
            work(b, i);
            i += kFewWaves;
            if (i >= t_end) break;
        }
    }

    // the four waves' results, one tile of columns after another
    constexpr int LD = D + 4;
    __shared__ __align__(16) float so[kFewWaves][16][LD];
    __shared__ float sm[kFewWaves][16], sl[kFewWaves][16];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const float l = sum_xor32(sum_xor16(l_i[c]));
        if (c) __syncthreads();
        if (qd == 0) sm[wave][m16] = m_i[c], sl[wave][m16] = l;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int d = 0; d < DPL; d += 4)
                *reinterpret_cast<float4 *>(&so[wave][m16][(4 * qd + r) * DPL + d]) =
                    make_float4(o[c][d][r], o[c][d + 1][r], o[c][d + 2][r], o[c][d + 3][r]);
        __syncthreads();
        const int col = c0 + 16 * c + (threadIdx.x >> 4), n = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * DPL;
        if (col >= cols) continue;
        float M = sm[0][n], L = 0.f;
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) M = fmaxf(M, sm[v][n]);
        float x[DPL];
#pragma unroll
        for (int e = 0; e < DPL; ++e) x[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) {
            if (sl[v][n] == 0.f) continue;  // a wave that saw nothing
            const float w = __builtin_amdgcn_exp2f(sm[v][n] - M);
            L += w * sl[v][n];
#pragma unroll
            for (int e = 0; e < DPL; ++e) x[e] = fmaf(w, so[v][n][d0 + e], x[e]);
        }
        const PagedColumn where = paged_column(col, G, kvh);
        if (sp.splits == 1) {
            const float inv = L == 0.f ? 0.f : 1.0f / L;
            uint16_t *dst = out + (int64_t)(sp.row0 + where.row) * out_stride + where.head * D + d0;
            if constexpr (DPL == 8)
                *reinterpret_cast<u32x4 *>(dst) = u32x4{T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv), T::pack(x[4] * inv, x[5] * inv),
                                                        T::pack(x[6] * inv, x[7] * inv)};
            else
                *reinterpret_cast<u32x2 *>(dst) = u32x2{T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv)};
        } else {
            const size_t pr = (size_t)sp.part0 + ((size_t)z * sp.rows + where.row) * view.nq + where.head;
#pragma unroll
            for (int e = 0; e < DPL; e += 4)
                *reinterpret_cast<float4 *>(part_o + pr * D + d0 + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
            if (d0 == 0) *reinterpret_cast<float2 *>(part_ml + pr * 2) = make_float2(M, L);
        }
    }
}

// ---------------------------------------------------------------------------------------
// Many columns: trees and chunks.  A block is 128 columns of one kv head, 32 to a wave, on a range of tiles of 64 slots.  Keys and values go from memory to LDS
// directly (a wave loads 16 slots of a tile, which lie in one page), a tile ahead, 16-byte chunks swapped by the slot so that neither the reads of S^T
// fragments nor the transposing reads of V^T meet in a bank.  S^T rows: fragment row m of 32 slots is slot m with bits 2 and 3 exchanged: registers 0-7 and
// 8-15 of a lane are then eight consecutive slots each, as the second product wants them.
//
// Matrix and vector pipe bound it, one after the other: with 2048 rows of 40 / 8 heads behind 2048 slots (129 GFLOP, 0.72 PFLOP/s, 180 us) the matrix pipe is busy for 33 %
// of the cycles and the vector pipe for 43 %, and 640 blocks on 512 places leave a sixth of the chip without work at the end.  A tile costs a block 2.2 us beside
// another block on its compute unit, the call some 10 us beside its tiles.  Two blocks of four waves a compute unit are what 256 registers a lane and 66 KB of LDS allow.
// Measured against it: products and softmax of 32-slot steps interleaved in one wave 220 us, eight waves in halves that take turns 196, fragments read 6 and 8
// ahead 0, three blocks a compute unit not possible without spilling 40 registers.  16 sequences of 21 rows on 500 to 6000 slots: 54.6 us in 488 blocks.
// ---------------------------------------------------------------------------------------
constexpr int kChunkTile = 64, kChunkCols = kPagedColumns;
template <int D>
constexpr int kChunkTileBytes = kChunkTile * D * 2;
template <int D>
constexpr int kChunkLds = 4 * kChunkTileBytes<D> + 64;  // two tiles of keys, two of values, and eight words: whether a wave's values were not finite

// 64 lanes x 16 bytes from a wave-uniform base and an offset per lane to 1 KB of LDS starting at lds_off (wave-uniform)
__device__ __forceinline__ void to_lds16(const void *base, uint32_t off, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds_off)) : "memory");
}
template <int N>
using step = std::integral_constant<int, N>;
template <int... I, class F>
__device__ __forceinline__ void steps_of(std::integer_sequence<int, I...>, F f) {
    (f(step<I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void steps(F f) {  // f(0), ..., f(N - 1), each as a type
    steps_of(std::make_integer_sequence<int, N>{}, f);
}
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <class T, int D, int CAP>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(const Kv4Spans<CAP> t, const PagedView view, const uint64_t *__restrict__ sees, int words,
                                                        const uint16_t *__restrict__ q, int64_t q_stride, uint16_t *__restrict__ out, int64_t out_stride,
                                                        float *__restrict__ part_o, float *__restrict__ part_ml) {
    constexpr int ST = D / 16, TT = D / 32, RB = D * 2, CPR = RB / 16, SPI = 64 / CPR;  // RB: bytes of a slot, CPR: its chunks, SPI: slots a load instruction fills
    typedef typename T::vec8 vec8;
    extern __shared__ __align__(1024) unsigned char smem[];
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int nkv = view.nkv, G = view.nq / nkv, cols = sp.rows * G, n_cb = (cols + kChunkCols - 1) / kChunkCols;
    const int local = blockIdx.x - sp.blk0, kvh = local % nkv, z = local / nkv / n_cb;
    const int cb = n_cb - 1 - local / nkv % n_cb;  // the blocks with the most slots first
    const int c0 = cb * kChunkCols + wave * 32, col = min(c0 + l32, cols - 1);
    const bool active = c0 < cols;
    const PagedColumn where = paged_column(col, G, kvh);
    // the last slot that all columns of the block (wave) see, and the last that some column of the wave does
    const int block_all = sees ? sp.len - 1 : sp.len + cb * kChunkCols / G;
    const int wave_all = sees ? sp.len - 1 : sp.len + min(c0, cols - 1) / G;
    const int wave_last = sees ? sp.len + sp.rows - 1 : sp.len + min(c0 + 31, cols - 1) / G;
    const int n_keys = sees ? sp.len + sp.rows : sp.len + min(cb * kChunkCols + kChunkCols - 1, cols - 1) / G + 1, last = n_keys - 1;
    const int n_tiles = (n_keys + kChunkTile - 1) / kChunkTile;
    const int t_begin = z * sp.per, t_end = min(n_tiles, t_begin + sp.per);
    const int32_t *__restrict__ pages = view.table + (int64_t)sp.seq * view.max_pages;
    const int mask = (1 << view.shift) - 1;
    const float scale = 1.4426950408889634f / sqrtf((float)D);

    vec8 qf[ST];
    {
        const uint16_t *src = q + (int64_t)(sp.row0 + where.row) * q_stride + where.head * D + 8 * hf;
#pragma unroll
        for (int s = 0; s < ST; ++s) qf[s] = __builtin_bit_cast(vec8, *reinterpret_cast<const u32x4 *>(src + 16 * s));
    }
    f32x16 o[TT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[tt][r] = 0.f;
    float m_i = -INFINITY, l_i = 0.f;

    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    typedef __attribute__((address_space(3))) uint32_t lds_u32;
    typedef __attribute__((address_space(3))) unsigned char lds_u8;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8 *)smem;
    auto k_at = [&](int i) { return lds0 + (i & 1) * kChunkTileBytes<D>; };
    auto v_at = [&](int i) { return lds0 + (2 + (i & 1)) * kChunkTileBytes<D>; };
    auto flags_at = [&](int i) { return lds0 + 4 * kChunkTileBytes<D> + (i & 1) * 16; };
    // Chunk c of slot r lies at position c ^ swap(r).  D 128: the 16 slots of an S^T read take 16 different positions, and so do the (slot, chunk) pairs of a
    // transposing read.  D 64: slots of 128 bytes, two to a row of banks: every other slot of a read takes every position.
    auto swap = [](int r) { return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (r >> 1) & 7; };
    // Pages of the tile's four runs of 16 slots: lane i % 4 looks up run i.  Nothing is done with them until they are used: that would wait for every load before them.
    auto look_up = [&](int tile) { return pages[min(tile * kChunkTile + 16 * (lane & 3), last) >> view.shift]; };
    auto held_runs = [&](int at) { return (uint32_t)__builtin_amdgcn_ballot_w64((uint32_t)at < (uint32_t)view.n_pages) & 15u; };
    const uint32_t lane_off = lane / CPR * RB + (((lane % CPR) ^ swap(lane / CPR)) << 4);  // of a lane in its run; of the e-th instruction: ^ swap(e SPI) << 4, e SPI slots on
    const size_t head_at = ((size_t)kvh << view.shift) * D, page_stride = ((size_t)nkv << view.shift) * D;
    const uint16_t *const k_head = view.k + head_at, *const v_head = view.v + head_at;
    auto load = [&](int tile, int at) {
        const int run0 = tile * kChunkTile + 16 * wave, found = __builtin_amdgcn_readlane(at, wave);
        const uint32_t page = (uint32_t)found < (uint32_t)view.n_pages ? found : 0;
        size_t first = page * page_stride;
        uint32_t off[16 / SPI];
        if (run0 + 15 <= last) {
            first += (uint32_t)(run0 & mask) * D;
#pragma unroll
            for (int e = 0; e < 16 / SPI; ++e) off[e] = (lane_off ^ (swap(e * SPI) << 4)) + e * SPI * RB;
        } else {  // (slots past the last one: the last)
#pragma unroll
            for (int e = 0; e < 16 / SPI; ++e) off[e] = (min(run0 + e * SPI + lane / CPR, last) & mask) * RB + ((lane_off ^ (swap(e * SPI) << 4)) & (RB - 1));
        }
        const uint16_t *kp = k_head + first, *vp = v_head + first;
        uint32_t into = k_at(tile) + 16 * wave * RB;
        asm volatile("" : "+s"(into));  // (else every sum below is kept in a register of its own from one tile to the next)
#pragma unroll
        for (int e = 0; e < 16 / SPI; ++e) to_lds16(kp, off[e], into + e * SPI * RB);
#pragma unroll
        for (int e = 0; e < 16 / SPI; ++e) to_lds16(vp, off[e], into + 2 * kChunkTileBytes<D> + e * SPI * RB);
    };
    const int part_from = (block_all + 1) / kChunkTile, masked_from = (wave_all + 1) / kChunkTile, own_to = active ? wave_last / kChunkTile : -1;  // first, first and last tile
    auto is_part = [&](int tile, uint32_t held) { return tile >= part_from || held != 15u; };
    // Looks through the values this wave has loaded: what is not finite becomes zero, and is noted
    auto look_through = [&](int tile) {
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 16 * RB / 1024; ++e) {
            lds_u32x4 *p = (lds_u32x4 *)(uintptr_t)(v_at(tile) + 16 * wave * RB + e * 1024 + lane * 16);
            u32x4 w = *p;
            uint32_t bad = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t b = not_finite<T>(w[x]);
                bad |= b;
                w[x] &= ~halves_of(b);
            }
            if (bad) *p = w;
            any |= bad;
        }
        const bool spoiled = __builtin_amdgcn_ballot_w64(any != 0) != 0;
        if (lane == 0) *((lds_u32 *)(uintptr_t)(flags_at(tile) + 4 * wave)) = spoiled;
    };
    // S^T: lane i of a 32-slot fragment reads slot swap23(i);  V^T: lane 4 r + x of a group of 16 reads four channels of slot r.  Fragment n of a product is read while
    // fragment n - kAhead is multiplied; what differs between fragments is an exclusive or of the lane's address, or a constant added to it.
    constexpr int kAhead = 4, NS = 2 * ST, NV = 4 * TT;
    const int krow = (l32 & 19) | ((l32 & 4) << 1) | ((l32 & 8) >> 1), vr = (lane & 15) >> 2, vx = lane & 3, vg = (lane >> 4) & 1;
    const uint32_t k_lane = krow * RB + ((hf ^ swap(krow)) << 4);                                           // chunk 2 s + hf: ^ (s << 5)
    const uint32_t v_lane = (8 * hf + vr) * RB + (((2 * vg + (vx >> 1)) ^ swap(8 * hf + vr)) << 4) + (vx & 1) * 8;  // chunk 4 tt + ..: ^ (tt << 6); four slots on: ^ swap(4)
    vec8 kf[kAhead], vf[kAhead];
    uint32_t kt, vt;
    auto k_read = [&](auto n_c) {  // fragment n: 32 slots u = n % 2, 16 channels n / 2
        constexpr int n = decltype(n_c)::value;
        kf[n % kAhead] = __builtin_bit_cast(vec8, *((const lds_u32x4 *)(uintptr_t)((kt ^ (n / 2 << 5)) + n % 2 * 32 * RB)));
    };
    auto v_read = [&](auto n_c) {  // fragment n: 32 channels n % TT, 16 slots n / TT; two reads of four slots
        constexpr int n = decltype(n_c)::value, tt = n % TT, s = n / TT;
        constexpr uint32_t four = D == 128 ? 1 << 4 : 2 << 4;  // swap(4)
        const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((vt ^ (tt << 6)) + 16 * s * RB)));
        const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)((vt ^ (tt << 6) ^ four) + (16 * s + 4) * RB)));
        vf[n % kAhead] = __builtin_bit_cast(vec8, u32x4{x.x, x.y, y.x, y.y});
    };
    auto compute = [&](int tile, uint32_t held, bool part) {
        const int key0 = tile * kChunkTile;
        f32x16 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[u][r] = 0.f;
        kt = k_at(tile) + k_lane, vt = v_at(tile) + v_lane;
        steps<kAhead>([&](auto n_c) { k_read(n_c); });
        __builtin_amdgcn_sched_barrier(0);
        steps<NS>([&](auto n_c) {
            constexpr int n = decltype(n_c)::value;
            sc[n % 2] = T::mfma32(kf[n % kAhead], qf[n / 2], sc[n % 2]);
            if constexpr (n + kAhead < NS) k_read(step<n + kAhead>{});
            else v_read(step<n + kAhead - NS>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        uint64_t seen = ~0ull;
        if (tile >= masked_from || held != 15u) {
            seen = seen_bits(sees, words, sp.len, sp.rows, sp.row0, where.row, key0);
#pragma unroll
            for (int run = 0; run < 4; ++run)
                if (!(held >> run & 1)) seen &= ~(0xffffull << (16 * run));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t bits = (uint32_t)(seen >> (32 * u)) >> (8 * hf);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(bits >> (16 * (r >> 3) + (r & 7)) & 1)) sc[u][r] = -INFINITY;
            }
        }
        float mx = sc[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[u][r]);
        mx = max_xor32(mx);
        const float cand = fmaf(mx, scale, -T::kRaise);
        const bool raise = cand > m_i;
        const float m_new = raise ? cand : m_i;
        float base = m_new == -INFINITY ? 0.f : m_new;  // a row may have seen no slot yet
        if (__builtin_amdgcn_ballot_w64(raise)) {
            const float corr = raise ? __builtin_amdgcn_exp2f(m_i - base) : 1.0f;
            l_i *= corr;
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[tt][r] *= corr;
        }
        m_i = m_new;
        const bool far = is_far(base);
        if (__builtin_amdgcn_ballot_w64(far)) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[u][r] = far ? less_far<T>(sc[u][r], scale, base) : sc[u][r];
            base = far ? 0.f : base;
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[u][r], scale, -base));
                sc[u][r] = p;
                sum[r & 3] += p;
            }
        l_i += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        vec8 pf[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int u = s >> 1, b = 8 * (s & 1);
            pf[s] = __builtin_bit_cast(vec8, u32x4{T::pack(sc[u][b], sc[u][b + 1]), T::pack(sc[u][b + 2], sc[u][b + 3]), T::pack(sc[u][b + 4], sc[u][b + 5]),
                                                   T::pack(sc[u][b + 6], sc[u][b + 7])});
        }
        steps<NV>([&](auto n_c) {
            constexpr int n = decltype(n_c)::value;
            o[n % TT] = T::mfma32(vf[n % kAhead], pf[n / TT], o[n % TT]);
            if constexpr (n + kAhead < NV) v_read(step<n + kAhead>{});
            __builtin_amdgcn_sched_barrier(0);
        });
        if (part) {
            const u32x4 f = *((const lds_u32x4 *)(uintptr_t)flags_at(tile));
            if (f.x | f.y | f.z | f.w)  // register r of tile tt is channel 32 tt + r % 4 + 8 (r / 4) + 4 hf
                for (int j = 0; j < kChunkTile && key0 + j < n_keys; ++j) {
                    const int page = page_of(pages, view.n_pages, (key0 + j) >> view.shift);
                    if (page < 0 || !(seen >> j & 1)) continue;
                    const uint16_t *src = view.v + ((((size_t)page * nkv + kvh) << view.shift) + ((key0 + j) & mask)) * D + 4 * hf;
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                        for (int r = 0; r < 16; r += 2) {
                            const uint32_t w = *reinterpret_cast<const uint32_t *>(src + 32 * tt + (r & 3) + 8 * (r >> 2)), b = not_finite<T>(w);
                            if (b & 0x8000u) o[tt][r] += T::lo(w);
                            if (b >> 31) o[tt][r + 1] += T::hi(w);
                        }
                }
        }
    };
    if (t_begin < t_end) {
        int at = look_up(t_begin), next = look_up(min(t_begin + 1, t_end - 1));
        load(t_begin, at);
        for (int i = t_begin; i < t_end; ++i) {
            const uint32_t held = held_runs(at);
            const bool part = is_part(i, held);
            wait_for_loads();
            if (part) look_through(i);
            __syncthreads();  // tile i is whole, and tile i - 1 has been read by every wave
            if (i + 1 < t_end) {
                at = next;
                next = look_up(min(i + 2, t_end - 1));
                load(i + 1, at);
            }
            if (i <= own_to) compute(i, held, part);
        }
    }
    l_i = sum_xor32(l_i);
    if (!active || c0 + l32 >= cols) return;
    if (sp.splits == 1) {
        const float inv = l_i == 0.f ? 0.f : 1.0f / l_i;
        uint16_t *dst = out + (int64_t)(sp.row0 + where.row) * out_stride + where.head * D + 4 * hf;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<u32x2 *>(dst + 32 * tt + 2 * r) = u32x2{T::pack(o[tt][r] * inv, o[tt][r + 1] * inv), T::pack(o[tt][r + 2] * inv, o[tt][r + 3] * inv)};
    } else {
        const size_t pr = (size_t)sp.part0 + ((size_t)z * sp.rows + where.row) * view.nq + where.head;
        float *dst = part_o + pr * D + 4 * hf;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(dst + 32 * tt + 2 * r) = make_float4(o[tt][r], o[tt][r + 1], o[tt][r + 2], o[tt][r + 3]);
        if (hf == 0) *reinterpret_cast<float2 *>(part_ml + pr * 2) = make_float2(m_i, l_i);
    }
}

// ---------------------------------------------------------------------------------------
// Joins the key ranges of one row and head (a unit).  A range of which the row sees nothing has sum 0 and an unused output.
// Few units: four waves each.  A lane takes the (max, sum) of one range, so that all of them are fetched at once; then D / 4 lanes add a range's output, four channels each,
// 1024 / D ranges at a time.  3.7 us with 12 units of 36 ranges: the launch and two dependent reads.
// ---------------------------------------------------------------------------------------
template <class T, int D, int CAP>
__global__ __launch_bounds__(256) void k_paged_join_wide(const Kv4Spans<CAP> t, int nq, const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                         uint16_t *__restrict__ out, int64_t out_stride) {
    constexpr int TPR = D / 4, PAR = 256 / TPR, kBatch = 8;  // lanes of a range, ranges at a time
    __shared__ float4 red[(PAR - 1) * TPR];
    const Kv4Span sp = t.s[blockIdx.y];
    const int unit = blockIdx.x;
    if (sp.splits == 1 || unit >= sp.rows * nq) return;
    const int tid = threadIdx.x, lane = tid & 63, e = tid % TPR, g = tid / TPR;
    const size_t step = (size_t)sp.rows * nq, pr = (size_t)sp.part0 + unit;
    const float2 ml = lane < sp.splits ? reinterpret_cast<const float2 *>(part_ml)[pr + lane * step] : make_float2(-INFINITY, 0.f);
    const float4 *po = reinterpret_cast<const float4 *>(part_o) + pr * TPR + e;
    float4 v[kBatch];
    auto fetch = [&](int z0) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) v[u] = z0 + u * PAR < sp.splits ? po[(z0 + u * PAR) * step * TPR] : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    fetch(g);
    const float M = wave_max(ml.x);
    const float w = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    const float L = wave_sum(ml.y == 0.f ? 0.f : w * ml.y);
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z0 = g; z0 - g < sp.splits; z0 += kBatch * PAR) {
        if (z0 != g) fetch(z0);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int z = z0 + u * PAR;
            const float wz = __shfl(w, z & 63, kWave), lz = __shfl(ml.y, z & 63, kWave);
            if (z < sp.splits && lz != 0.f) A.x = fmaf(wz, v[u].x, A.x), A.y = fmaf(wz, v[u].y, A.y), A.z = fmaf(wz, v[u].z, A.z), A.w = fmaf(wz, v[u].w, A.w);
        }
    }
    if (g) red[(g - 1) * TPR + e] = A;  // the PAR sums, in order
    __syncthreads();
    if (g) return;
#pragma unroll
    for (int i = 1; i < PAR; ++i) {
        const float4 x = red[(i - 1) * TPR + e];
        A.x += x.x, A.y += x.y, A.z += x.z, A.w += x.w;
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    *reinterpret_cast<u32x2 *>(out + (int64_t)(sp.row0 + unit / nq) * out_stride + unit % nq * D + 4 * e) = u32x2{T::pack(A.x * inv, A.y * inv), T::pack(A.z * inv, A.w * inv)};
}
// Many units: D / 4 lanes each, four channels a lane, which reads every (max, sum) itself; nothing passes between lanes.  2560 units of 21 ranges: 6.6 us for 27 MB that the
// blocks before have just written, 4.1 TB/s.
template <class T, int D, int CAP>
__global__ __launch_bounds__(256) void k_paged_join(const Kv4Spans<CAP> t, int nq, const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                    uint16_t *__restrict__ out, int64_t out_stride) {
    constexpr int TPU = D / 4, UPB = 256 / TPU, kBatch = 8;
    const Kv4Span sp = t.s[blockIdx.y];
    if (sp.splits == 1) return;
    const int unit = blockIdx.x * UPB + threadIdx.x / TPU, e = threadIdx.x % TPU;
    if (unit >= sp.rows * nq) return;
    const size_t step = (size_t)sp.rows * nq, pr = (size_t)sp.part0 + unit;
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + pr;
    const float4 *po = reinterpret_cast<const float4 *>(part_o) + pr * TPU + e;
    float M = -INFINITY, L = 0.f;
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z0 = 0; z0 < sp.splits; z0 += kBatch) {
        float2 m[kBatch];
        float4 v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const bool there = z0 + u < sp.splits;
            m[u] = there ? ml[(z0 + u) * step] : make_float2(-INFINITY, 0.f);
            v[u] = there ? po[(z0 + u) * step * TPU] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float top = M;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) top = fmaxf(top, m[u].x);
        const float corr = L == 0.f ? 0.f : __builtin_amdgcn_exp2f(M - top);  // (0 where there is nothing yet: A and L are 0)
        L *= corr, A.x *= corr, A.y *= corr, A.z *= corr, A.w *= corr;
        M = top;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (m[u].y != 0.f) {
                const float w = __builtin_amdgcn_exp2f(m[u].x - M);
                L = fmaf(w, m[u].y, L), A.x = fmaf(w, v[u].x, A.x), A.y = fmaf(w, v[u].y, A.y), A.z = fmaf(w, v[u].z, A.z), A.w = fmaf(w, v[u].w, A.w);
            }
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    *reinterpret_cast<u32x2 *>(out + (int64_t)(sp.row0 + unit / nq) * out_stride + unit % nq * D + 4 * e) = u32x2{T::pack(A.x * inv, A.y * inv), T::pack(A.z * inv, A.w * inv)};
}

// ---------------------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------------------
PagedAttendPlan plan_paged_attend(const Paged &k, Kv4Table &t) {
    const int nkv = k.c.n_kv_heads, G = k.c.n_q_heads / nkv;
    int64_t most = 0, longest = 0;
    for (int j = 0; j < t.n; ++j) {
        if (!t.s[j].rows) continue;
        most = std::max<int64_t>(most, (int64_t)t.s[j].rows * G);
        longest = std::max<int64_t>(longest, (int64_t)t.s[j].len + t.s[j].rows);
    }
    // us with columns by 32 : by 128, 40 / 8 heads, one sequence of 8 rows on 1000 slots 12.0 : 11.9, on 4000 18.1 : 13.1, of 64 rows on 4000 34.5 : 26.2; 16 of 8 rows on
    // 3000 slots 51.1 : 44.2; 12 / 2 heads, 16 rows on 2000 slots 11.3 : 11.2, 40 rows 13.0 : 14.1
    PagedAttendPlan p{most <= 16 ? 16 : most <= 32 ? 32 : kChunkCols, 0, 0};
    const bool few = p.cols < kChunkCols;
    const int tile = few ? kFewTile : kChunkTile, step = few ? kFewWaves : 1;
    auto groups = [&](const Kv4Span &s) { return (int64_t)nkv * (((int64_t)s.rows * G + p.cols - 1) / p.cols); };
    auto tiles = [&](const Kv4Span &s) { return ((int64_t)s.len + s.rows + tile - 1) / tile; };
    int64_t work = 0;
    for (int j = 0; j < t.n; ++j)
        if (t.s[j].rows) work += groups(t.s[j]) * tiles(t.s[j]);
    // Ranges of one length for all spans: the call's work in kPagedBlocks parts, so that long spans are cut however many short ones stand beside them; a little longer
    // where that leaves no more blocks than the chip holds at a time, as one block more lasts as long as all of them.
    auto up = [&](int64_t x) { return std::max<int64_t>((x + step - 1) / step * step, 1); };
    auto blocks_of = [&](int64_t x) {
        int64_t blocks = 0;
        for (int j = 0; j < t.n; ++j)
            if (t.s[j].rows) blocks += groups(t.s[j]) * ((tiles(t.s[j]) + x - 1) / x);
        return blocks;
    };
    auto parts_of = [&](int64_t want) { return up(std::max((work + want - 1) / want, ((longest + tile - 1) / tile + kPagedRanges - 1) / kPagedRanges)); };
    // Ranges of less than eight tiles of 64 slots are made twice as long, for one block a compute unit: what such a block saves at its tiles costs as much again in
    // partial results.  us with 512 : 256 blocks, 40 / 8 heads, 64 rows on 1000 slots 24.4 : 19.1, on 4000 28.8 : 26.3, on 16000 44.8 : 50.1; 16 rows on 4000 20.7 : 16.4;
    // 16 sequences of 21 rows on 500 to 6000 67.0 : 77.6; 12 of 10 to 60 rows on 128 to 1500, 28 / 4 heads, 27.8 : 26.9.
    int64_t want = kPagedBlocks, per = parts_of(want);
    if (!few && per < 8) want = kPagedBlocks / 2, per = parts_of(want);
    // up to 512 slots in one range, without a join: 12 / 2 heads, one row, 300 slots 7.4 us : 9.1 in ranges, 500 slots 8.6 : 9.2; 4 of 300 slots with 40 / 8 heads 7.6 : 9.2
    if (few && longest <= 512) per = std::max<int64_t>(per, 512 / tile);
    if (blocks_of(per) > want && blocks_of(2 * per) <= want) {  // (longer ranges are never more blocks: the shortest ones that are few enough, by halving)
        int64_t low = per, high = 2 * per;  // too many blocks, few enough
        while (high - low > step) {
            const int64_t middle = up((low + high) / 2);
            if (middle == high) break;
            (blocks_of(middle) <= want ? high : low) = middle;
        }
        per = high;
    }
    int64_t part = 0;
    for (int j = 0; j < t.n; ++j) {
        Kv4Span &s = t.s[j];
        s.blk0 = (int32_t)std::min<int64_t>(p.blocks, INT32_MAX);
        s.per = (int32_t)per, s.splits = 1, s.part0 = (int32_t)part;
        if (!s.rows) continue;
        s.splits = (int32_t)((tiles(s) + per - 1) / per);
        p.blocks += groups(s) * s.splits;
        if (s.splits > 1) {
            part += (int64_t)s.splits * s.rows * k.c.n_q_heads;
            p.join = std::max(p.join, s.rows);
        }
    }
    return p;
}

// More LDS than a kernel has without asking: allowed once per kernel and GPU
template <class T, int D, int CAP>
static hipError_t allow_chunk_lds() {
    if (kChunkLds<D> <= 65536) return hipSuccess;
    static std::atomic<uint64_t> allowed{0};  // a bit per GPU; those past 64 are asked every time
    int gpu = 0;
    hipError_t e = hipGetDevice(&gpu);
    if (e != hipSuccess) return e;
    const uint64_t bit = gpu >= 0 && gpu < 64 ? 1ull << gpu : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_paged_chunk<T, D, CAP>), hipFuncAttributeMaxDynamicSharedMemorySize, kChunkLds<D>);
    if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <class T, int D>
static hipError_t attend_in(const Paged &k, int layer, const Kv4Table &t, const PagedAttendPlan &p, const uint64_t *sees, int words, const uint16_t *q,
                            int64_t q_stride, uint16_t *out, int64_t out_stride) {
    hipError_t e = hipSuccess;
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        const dim3 grid(p.blocks);
        const PagedView view = k.view(layer);
        if (p.cols == 16)
            hipLaunchKernelGGL((k_paged_few<T, D, 1, CAP>), grid, dim3(256), 0, k.stream, tab, view, sees, words, q, q_stride, out, out_stride, k.part_o, k.part_ml);
        else if (p.cols == 32)
            hipLaunchKernelGGL((k_paged_few<T, D, 2, CAP>), grid, dim3(256), 0, k.stream, tab, view, sees, words, q, q_stride, out, out_stride, k.part_o, k.part_ml);
        else {
            e = allow_chunk_lds<T, D, CAP>();
            if (e != hipSuccess) return;
            hipLaunchKernelGGL((k_paged_chunk<T, D, CAP>), grid, dim3(256), kChunkLds<D>, k.stream, tab, view, sees, words, q, q_stride, out, out_stride, k.part_o,
                               k.part_ml);
        }
        if (p.join) {
            // Four waves a unit while there are fewer units than would fill the chip otherwise.  us with four waves : without, 40 / 8 heads, one sequence, 1 row on 4000
            // slots 9.3 : 11.4, on 2000 8 rows 12.0 : 14.3, 22 rows 18.2 : 19.7, 30 rows 17.6 : 17.6, 64 rows 22.6 : 21.3; 16 of 8 rows on 3000 slots 43.2 : 39.1
            const int64_t units = (int64_t)p.join * k.c.n_q_heads;
            const bool wide = units * t.n < 1024;
            auto *kern = wide ? k_paged_join_wide<T, D, CAP> : k_paged_join<T, D, CAP>;
            constexpr int per_block = 1024 / D;
            hipLaunchKernelGGL(kern, dim3(wide ? units : (units + per_block - 1) / per_block, t.n), dim3(256), 0, k.stream, tab, k.c.n_q_heads, k.part_o, k.part_ml, out, out_stride);
        }
        e = hipGetLastError();
    });
    return e;
}

int launch_paged_attend(const Paged &k, int layer, Kv4Table &t, const uint64_t *sees, int words, const uint16_t *q, int64_t q_stride, uint16_t *out,
                        int64_t out_stride) {
    const PagedAttendPlan p = plan_paged_attend(k, t);
    // a launch has at most 2^32 - 1 threads a direction (asked before anything is launched)
    if (p.blocks >= 1 << 24) return fail(ST_ERANGE, "%lld blocks of work, 2^24 or more", (long long)p.blocks);
    const bool f16 = k.c.dtype == ST_F16;
    const hipError_t e = k.c.head_dim == 128 ? (f16 ? attend_in<Fp16, 128>(k, layer, t, p, sees, words, q, q_stride, out, out_stride)
                                                    : attend_in<Bf16, 128>(k, layer, t, p, sees, words, q, q_stride, out, out_stride))
                                             : (f16 ? attend_in<Fp16, 64>(k, layer, t, p, sees, words, q, q_stride, out, out_stride)
                                                    : attend_in<Bf16, 64>(k, layer, t, p, sees, words, q, q_stride, out, out_stride));
    return launched("st_paged_attend", e);
}

}  // namespace st
