// Attention over the 4-bit key/value cache, and the attention weight each of its slots receives.
//
// Row i of a span (seq, len, rows) sees slots [0, len + i].  The query heads of a kv head are folded into columns: column i * G
// + h is row i of head h.  With S^T = K Q^T (slots x columns) a lane holds one column, so the softmax is register arithmetic
// and P^T is the second product's operand as it stands: O^T = V^T P^T.  Codes become bf16 in registers
// (v_cvt_scalef32_pk_bf16_fp4, two values an instruction, exact); keys give eight channels of a slot to a lane, which is what
// the first product wants, values come as channel pairs of one slot and are put together with the neighbouring slot's by a byte
// permute. Scores, maxima, sums and outputs are fp32; the weights enter the second product as bf16 (rounded just below the
// running maximum's 1, where that costs least), as the model's own attention does.
//
// A value group that held an infinity or NaN reads as NaN, and reaches exactly the rows that see it: in tiles that some row
// sees only in part such groups are multiplied as zeros and the rows that see them marked.
#include <utility>

#include "kv4.h"
#include "st_device.h"

namespace st {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));  // scales: rows of two or four bytes
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ u32x4 keys8(uint32_t w, float unit) {  // eight channels of one slot
    return u32x4{kv4_pair<0>(w, unit), kv4_pair<1>(w, unit), kv4_pair<2>(w, unit), kv4_pair<3>(w, unit)};
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Eight slots of V as a lane loads them: NB bytes of codes (2 NB channels of one scale group) of slot j in c[j], and the scale
// bytes of all groups, not taken apart until they are used, so that nothing waits for the load where it is issued.
template <int D, int NB>
struct Values8 {
    uint32_t c[8], s[D / 16];
    // bits of the scale of slot j (byte << 23); shift: 8 * group
    __device__ __forceinline__ uint32_t unit(int j, int shift) const {
        return __builtin_amdgcn_ubfe(D == 128 ? s[j] : s[j >> 1], shift + (D == 128 ? 0 : 16 * (j & 1)), 8) << 23;
    }
};
// Slots key .. key + 7 of one kv head: NB bytes of codes at byte `at` of each.  TAIL: slots past `last` are read as `last` (no
// address past it is formed).
template <int D, int NB, bool TAIL>
__device__ __forceinline__ void load_values(Values8<D, NB> &v, const uint8_t *codes, const uint8_t *scales, int key, int last, int at) {
    constexpr int CB = D / 2, SB = D / 32;
    auto code = [&](int slot) -> uint32_t {
        const uint8_t *p = codes + (uint32_t)slot * CB + at;
        if constexpr (NB == 4) return *reinterpret_cast<const uint32_t *>(p);
        if constexpr (NB == 2) return *reinterpret_cast<const uint16_t *>(p);
        return *p;
    };
    if constexpr (TAIL) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int slot = min(key + j, last);
            v.c[j] = code(slot);
            if constexpr (SB == 4) {
                v.s[j] = *reinterpret_cast<const uint32_t *>(scales + (uint32_t)slot * SB);
            } else {
                const uint32_t w = *reinterpret_cast<const uint16_t *>(scales + (uint32_t)slot * SB);
                v.s[j >> 1] = j & 1 ? v.s[j >> 1] | w << 16 : w;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v.c[j] = code(key + j);
        const u32x4_a2 *p = reinterpret_cast<const u32x4_a2 *>(scales + (uint32_t)key * SB);
#pragma unroll
        for (int h = 0; h < D / 64; ++h) {
            const u32x4 a = p[h];
#pragma unroll
            for (int j = 0; j < 4; ++j) v.s[4 * h + j] = a[j];
        }
    }
}
// The scales of eight slots, ready for use.  A NaN's (255 << 23) is an infinity, and infinity times its zero codes a NaN.
struct Units8 {
    uint32_t f[8];
    template <int D, int NB>
    __device__ __forceinline__ Units8(const Values8<D, NB> &v, int shift) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v.unit(j, shift);
    }
    __device__ __forceinline__ bool any_nan() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, f[j]);
        return m == (uint32_t)kKv4Nan << 23;
    }
    __device__ __forceinline__ void nan_to_zero() {  // (their codes are zeros: any finite scale does)
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = min(f[j], 0x7f000000u);
    }
};
// channels 2 B and 2 B + 1 of the eight slots, slots in order
template <int B, int D, int NB>
__device__ __forceinline__ void value_pairs(const Values8<D, NB> &v, const Units8 &u, u32x4 &even, u32x4 &odd) {
    uint32_t p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = kv4_pair<B>(v.c[j], __uint_as_float(u.f[j]));
    even = u32x4{low_halves(p[0], p[1]), low_halves(p[2], p[3]), low_halves(p[4], p[5]), low_halves(p[6], p[7])};
    odd = u32x4{high_halves(p[0], p[1]), high_halves(p[2], p[3]), high_halves(p[4], p[5]), high_halves(p[6], p[7])};
}

// Where a column's query is
struct Column {
    int row, head;  // row of the span, query head
};
__device__ __forceinline__ Column column_of(int col, int G, int kvh) { return Column{col / G, kvh * G + col % G}; }

// ---------------------------------------------------------------------------------------
// Few columns: single tokens and short runs.  With one group of columns bound by memory (the cache is read once): 16 tokens of
// 40 / 8 heads on 500 to 6000 slots 17.0 us, 3.4 TB/s, one of 12 / 2 heads on 4608 slots 4.6 us, all latency.  With more by the
// vector pipe and latency: 350 vector and 32 matrix instructions a tile of 32 columns, 86 rows of 40 / 8 heads on 4096 slots 24 us.
// With one wave a SIMD a tile takes 2900 cycles; of the waves' cycles 60 % issue (52 % vector instructions), 29 % wait for loads
// and results, 11 % for their turn.  (Twice the blocks on half the slots each take as long.)
//
// A wave works on its own, on tiles of 32 slots, with NT tiles of 16 columns and no LDS until the end (four tiles no longer fit
// the registers without moves: 36 us for 86 rows of 40 / 8 heads on 4096 slots, against 28 with two): S^T by 16x16x32 MFMAs
// whose A rows are slots 8 (m / 4) + 4 t + m % 4, so that lane (column, quarter) ends up with the weights of slots 8 quarter ..
// + 7 -- the B operand of the second product.  A lane reads 16 bytes (one scale group) of each of its two keys and, of eight
// value slots, the D / 16 channels that make its row m of D / 16 products.  The next tile's loads are issued before this tile's
// work.  A block's four waves take every fourth tile of its range and are joined through LDS; ranges are joined by k_kv4_join.
// ---------------------------------------------------------------------------------------
constexpr int kFewTile = 32, kFewWaves = 4;

template <int D, int NT, int CAP>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void k_kv4_few(const Kv4Spans<CAP> t, const Kv4View view, const bf16_t *__restrict__ q,
                                                 int64_t q_stride, bf16_t *__restrict__ out, int64_t out_stride,
                                                 float *__restrict__ part_o, float *__restrict__ part_ml,
                                                 float *__restrict__ lse, float *__restrict__ scores, int64_t score_stride) {
    constexpr int KS = D / 32, DPL = D / 16, NB = D / 32, CB = D / 2, SB = D / 32;
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, qd = lane >> 4;
    const int nkv = view.nkv, G = view.nq / nkv;
    const int cols = sp.rows * G, n_cb = (cols + 16 * NT - 1) / (16 * NT), local = blockIdx.x - sp.blk0;
    const int kvh = local % nkv, z = local / nkv / n_cb, c0 = local / nkv % n_cb * (16 * NT);  // c0: the block's first column
    const int n_keys = sp.len + sp.rows, last = n_keys - 1, n_tiles = (n_keys + kFewTile - 1) / kFewTile;
    const int t_begin = z * sp.per, t_end = min(n_tiles, t_begin + sp.per);
    const size_t head0 = ((size_t)sp.seq * nkv + kvh) * view.max_seq;
    const uint8_t *kc = view.k + head0 * CB, *vc = view.v + head0 * CB, *ks = view.ks + head0 * SB, *vs = view.vs + head0 * SB;
    const int sees_all = sp.len + c0 / G;  // last slot that all of its columns see
    const float scale = 1.4426950408889634f / sqrtf((float)D);

    bf16x8 qf[NT][KS];
    int lim[NT];  // last slot the column sees
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const Column w = column_of(min(c0 + 16 * c + m16, cols - 1), G, kvh);
        lim[c] = sp.len + w.row;
        const bf16_t *src = q + (int64_t)(sp.row0 + w.row) * q_stride + w.head * D + qd * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[c][s] = as_bf16x8(*reinterpret_cast<const u32x4 *>(src + 8 * s));
    }
    f32x4 o[NT][DPL];
    float m_i[NT], l_i[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        m_i[c] = -INFINITY, l_i[c] = 0.f;
#pragma unroll
        for (int T = 0; T < DPL; ++T) o[c][T] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    struct Tile {
        uint32_t k[2][KS], kb[2];
        Values8<D, NB> v;
    };
    auto load = [&](Tile &x, int tile) {
        const int key0 = tile * kFewTile;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t slot = min(key0 + 8 * (m16 >> 2) + 4 * u + (m16 & 3), last);
            if constexpr (D == 128) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(kc + slot * CB + qd * 16);
                x.k[u][0] = w.x, x.k[u][1] = w.y, x.k[u][2] = w.z, x.k[u][3] = w.w;
                x.kb[u] = ks[slot * SB + qd];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(kc + slot * CB + qd * 8);
                x.k[u][0] = w.x, x.k[u][1] = w.y;
                x.kb[u] = ks[slot * SB + (qd >> 1)];
            }
        }
        const int at = m16 * NB;
        if (key0 + kFewTile <= n_keys)
            load_values<D, NB, false>(x.v, vc, vs, key0 + 8 * qd, last, at);
        else
            load_values<D, NB, true>(x.v, vc, vs, key0 + 8 * qd, last, at);
    };
    auto work = [&](Tile &x, int tile) {
        const int key0 = tile * kFewTile;
        f32x4 sc[NT][2];
#pragma unroll
        for (int c = 0; c < NT; ++c) sc[c][0] = sc[c][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 kf = as_bf16x8(keys8(x.k[u][s], kv4_scale(x.kb[u])));
#pragma unroll
                for (int c = 0; c < NT; ++c) sc[c][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][s], sc[c][u], 0, 0, 0);
            }
        Units8 unit(x.v, 8 * (m16 * DPL / 32));
        const bool part = key0 + kFewTile - 1 > sees_all;  // some row does not see all of the tile
        uint32_t poison = 0;                              // columns (bit c) that see a NaN among this lane's output channels
        if (part) {
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (key0 + 8 * qd + 4 * u + r > lim[c]) sc[c][u][r] = -INFINITY;
            if (__builtin_amdgcn_ballot_w64(unit.any_nan())) {
                unit.nan_to_zero();
                for (int slot = key0; slot < min(key0 + kFewTile, n_keys); ++slot)
                    if (vs[(uint32_t)slot * SB + qd * SB / 4] == kKv4Nan)
#pragma unroll
                        for (int c = 0; c < NT; ++c)
                            if (slot <= lim[c]) poison |= 1u << c;
            }
        }
        if constexpr (NT == 1)
            if (scores && c0 + m16 < cols) {
                const Column w = column_of(c0 + m16, G, kvh);
                float4 *dst = reinterpret_cast<float4 *>(scores + ((int64_t)(sp.row0 + w.row) * view.nq + w.head) * score_stride + key0 + 8 * qd);
                dst[0] = make_float4(sc[0][0][0], sc[0][0][1], sc[0][0][2], sc[0][0][3]);
                dst[1] = make_float4(sc[0][1][0], sc[0][1][1], sc[0][1][2], sc[0][1][3]);
            }
        bf16x8 pf[NT];
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
            const float cand = mx * scale;
            const bool raise = cand > m_i[c];
            const float m_new = raise ? cand : m_i[c];
            const float base = m_new == -INFINITY ? 0.f : m_new;  // nothing seen yet
            if (__builtin_amdgcn_ballot_w64(raise)) {
                const float corr = raise ? __builtin_amdgcn_exp2f(m_i[c] - base) : 1.0f;
                l_i[c] *= corr;
#pragma unroll
                for (int T = 0; T < DPL; ++T) o[c][T] *= corr;
            }
            m_i[c] = m_new;
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = __builtin_amdgcn_exp2f(fmaf(sc[c][j >> 2][j & 3], scale, -base));
                l_i[c] += p[j];
            }
            pf[c] = as_bf16x8(u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])});
        }
        auto multiply = [&](auto b_c) {
            constexpr int B = decltype(b_c)::value;
            u32x4 even, odd;
            value_pairs<B>(x.v, unit, even, odd);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                o[c][2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), pf[c], o[c][2 * B], 0, 0, 0);
                o[c][2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), pf[c], o[c][2 * B + 1], 0, 0, 0);
            }
        };
        multiply(std::integral_constant<int, 0>{});
        multiply(std::integral_constant<int, 1>{});
        if constexpr (NB == 4) {
            multiply(std::integral_constant<int, 2>{});
            multiply(std::integral_constant<int, 3>{});
        }
        if (__builtin_amdgcn_ballot_w64(poison != 0)) {
#pragma unroll
            for (int c = 0; c < NT; ++c)
                if (poison >> c & 1)
#pragma unroll
                    for (int T = 0; T < DPL; ++T) o[c][T] = f32x4{NAN, NAN, NAN, NAN};
        }
    };
    Tile a, b;
    int i = t_begin + wave;
    if (i < t_end) load(a, i);
    while (i < t_end) {
        if (i + kFewWaves < t_end) load(b, i + kFewWaves);
        work(a, i);
        i += kFewWaves;
        if (i >= t_end) break;
        if (i + kFewWaves < t_end) load(a, i + kFewWaves);
        work(b, i);
        i += kFewWaves;
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
            for (int T = 0; T < DPL; T += 4)
                *reinterpret_cast<float4 *>(&so[wave][m16][(4 * qd + r) * DPL + T]) =
                    make_float4(o[c][T][r], o[c][T + 1][r], o[c][T + 2][r], o[c][T + 3][r]);
        __syncthreads();
        const int col = c0 + 16 * c + (threadIdx.x >> 4), n = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * DPL;
        if (col >= cols) continue;
        float M = sm[0][n], w[kFewWaves], L = 0.f;
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) M = fmaxf(M, sm[v][n]);
        float x[DPL];
#pragma unroll
        for (int e = 0; e < DPL; ++e) x[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) {
            w[v] = sm[v][n] == -INFINITY && !(sl[v][n] != sl[v][n]) ? 0.f : __builtin_amdgcn_exp2f(sm[v][n] - M);
            L += w[v] * sl[v][n];
#pragma unroll
            for (int e = 0; e < DPL; ++e) x[e] = fmaf(w[v], so[v][n][d0 + e], x[e]);
        }
        const Column where = column_of(col, G, kvh);
        if (sp.splits == 1) {
            const float inv = 1.0f / L;
            bf16_t *dst = out + (int64_t)(sp.row0 + where.row) * out_stride + where.head * D + d0;
            if constexpr (DPL == 8)
                *reinterpret_cast<u32x4 *>(dst) = u32x4{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv),
                                                        pack_bf16x2(x[4] * inv, x[5] * inv), pack_bf16x2(x[6] * inv, x[7] * inv)};
            else
                *reinterpret_cast<u32x2 *>(dst) = u32x2{pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv)};
            if (lse && d0 == 0) lse[(size_t)(sp.row0 + where.row) * view.nq + where.head] = M + __builtin_amdgcn_logf(L);
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
// Chunks, bound by the matrix pipe and, in turn with it, the vector pipe: 4096 rows of 40 / 8 heads on 4096 slots 520 us, 1.0
// PFLOP/s (measured at 515: staging left out 448 us, exponentials left out 497).  A block is 128 columns of one kv head (four waves
// of 32) on a range of tiles of 128 slots.  The tile's codes are loaded one tile ahead into registers, turned into bf16 once for
// all four waves and put into LDS as the MFMA operands that the waves read: 1 KB fragments, 16 bytes a lane (bank conflicts take
// 14 % of the LDS cycles).  Two blocks share a compute unit, so that one has work for either pipe while the other waits: the
// matrix pipe is busy for 42 % of the cycles and the vector pipe for 53 %, so little of them overlaps.
//   K: a thread has one scale group (32 channels) of one or two slots;  V: eight slots x eight channels.
//   S^T rows: fragment row m of 32 slots is slot swap(m) (bits 2 and 3 exchanged): registers 0-7 and 8-15 of a lane are then eight
//   consecutive slots each, as the second product wants them.
// ---------------------------------------------------------------------------------------
constexpr int kTileKeys = 128, kTileCols = kKv4Columns;

__device__ __forceinline__ int swap23(int m) { return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1); }

template <int D, int CAP>
__global__ __launch_bounds__(256, 2) void k_kv4_chunk(const Kv4Spans<CAP> t, const Kv4View view, const bf16_t *__restrict__ q,
                                                      int64_t q_stride, bf16_t *__restrict__ out, int64_t out_stride,
                                                      float *__restrict__ part_o, float *__restrict__ part_ml,
                                                      float *__restrict__ lse) {
    constexpr int CB = D / 2, SB = D / 32, ST = D / 16, TT = D / 32, NO = D / 8, PT = 32 / NO;  // PT: channels of an octet per tile
    constexpr int KG = D / 64;  // scale groups of K per thread
    __shared__ __align__(16) u32x4 kt[4 * ST * 64], vt[TT * 8 * 64];
    __shared__ uint32_t nan_seen[4];
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hf = lane >> 5;
    const int nkv = view.nkv, G = view.nq / nkv, cols = sp.rows * G, n_cb = (cols + kTileCols - 1) / kTileCols;
    const int local = blockIdx.x - sp.blk0, kvh = local % nkv, z = local / nkv / n_cb;
    const int cb = n_cb - 1 - local / nkv % n_cb;  // the blocks with the most slots first
    const int c0 = cb * kTileCols + wave * 32, col = min(c0 + l32, cols - 1);
    const bool active = c0 < cols;
    const Column where = column_of(col, G, kvh);
    const int lim = sp.len + where.row;
    const int wave_first = sp.len + min(c0, cols - 1) / G, wave_last = sp.len + min(c0 + 31, cols - 1) / G;
    const int n_keys = sp.len + min(cb * kTileCols + kTileCols - 1, cols - 1) / G + 1, last = n_keys - 1;
    const int n_tiles = (n_keys + kTileKeys - 1) / kTileKeys;
    const int t_begin = z * sp.per, t_end = min(n_tiles, t_begin + sp.per);
    const size_t head0 = ((size_t)sp.seq * nkv + kvh) * view.max_seq;
    const uint8_t *kc = view.k + head0 * CB, *vc = view.v + head0 * CB, *ks = view.ks + head0 * SB, *vs = view.vs + head0 * SB;
    const float scale = 1.4426950408889634f / sqrtf((float)D);

    bf16x8 qf[ST];
    {
        const bf16_t *src = q + (int64_t)(sp.row0 + where.row) * q_stride + where.head * D + 8 * hf;
#pragma unroll
        for (int s = 0; s < ST; ++s) qf[s] = as_bf16x8(*reinterpret_cast<const u32x4 *>(src + 16 * s));
    }
    f32x16 o[TT];
#pragma unroll
    for (int tt = 0; tt < TT; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[tt][r] = 0.f;
    float m_i = -INFINITY, l_i = 0.f;

    // this thread's part of a tile
    const int k_slot = tid & 127, k_group = tid >> 7;                     // K: groups k_group and k_group + 2
    const int v_oct = tid % NO, v_kb = tid / NO;                          // V: channels 8 v_oct .. + 7 of slots 8 v_kb .. + 7
    const bool has_v = v_kb < 16;
    u32x4 kw[KG];
    uint32_t kb[KG];
    Values8<D, 4> vw;
    auto load = [&](int tile) {
        const int key0 = tile * kTileKeys;
        const uint32_t slot = min(key0 + k_slot, last);
#pragma unroll
        for (int e = 0; e < KG; ++e) {
            kw[e] = *reinterpret_cast<const u32x4 *>(kc + slot * CB + (k_group + 2 * e) * 16);
            kb[e] = ks[slot * SB + k_group + 2 * e];
        }
        if (!has_v) return;
        if (key0 + kTileKeys <= n_keys)
            load_values<D, 4, false>(vw, vc, vs, key0 + 8 * v_kb, last, 4 * v_oct);
        else
            load_values<D, 4, true>(vw, vc, vs, key0 + 8 * v_kb, last, 4 * v_oct);
    };
    auto stage = [&]() {
        const int u = k_slot >> 5, m = swap23(k_slot & 31);
#pragma unroll
        for (int e = 0; e < KG; ++e) {
            const float k_unit = kv4_scale(kb[e]);
#pragma unroll
            for (int c = 0; c < 4; ++c)  // channels 32 group + 8 c
                kt[(u * ST + 2 * (k_group + 2 * e) + (c >> 1)) * 64 + (c & 1) * 32 + m] = keys8(kw[e][c], k_unit);
        }
        Units8 unit(vw, 8 * (v_oct >> 2));
        const bool bad = has_v && unit.any_nan();
        if (bad) unit.nan_to_zero();
        const uint64_t any = __builtin_amdgcn_ballot_w64(bad);
        if (lane == 0) nan_seen[wave] = any != 0;
        if (!has_v) return;
        u32x4 *dst = &vt[(v_kb >> 1) * 64 + (v_kb & 1) * 32 + v_oct];  // channel 8 v_oct + e: tile e / PT, row v_oct + NO (e % PT)
        auto put = [&](auto b_c) {
            constexpr int B = decltype(b_c)::value;
            u32x4 even, odd;
            value_pairs<B>(vw, unit, even, odd);
            dst[(2 * B) / PT * 512 + NO * ((2 * B) % PT)] = even;
            dst[(2 * B + 1) / PT * 512 + NO * ((2 * B + 1) % PT)] = odd;
        };
        put(std::integral_constant<int, 0>{});
        put(std::integral_constant<int, 1>{});
        put(std::integral_constant<int, 2>{});
        put(std::integral_constant<int, 3>{});
    };
    auto half_tile = [&](int key0, auto h_c) {  // 64 slots
        constexpr int H = decltype(h_c)::value;
        f32x16 sc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[u][r] = 0.f;
#pragma unroll
        for (int s = 0; s < ST; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kt[((2 * H + u) * ST + s) * 64 + lane]), qf[s], sc[u], 0, 0, 0);
        if (key0 + 63 > wave_first) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key0 + 32 * u + 16 * (r >> 3) + 8 * hf + (r & 7) > lim) sc[u][r] = -INFINITY;
        }
        float mx = sc[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[u][r]);
        mx = max_xor32(mx);
        const float cand = mx * scale;
        const bool raise = cand > m_i;
        const float m_new = raise ? cand : m_i;
        const float base = m_new == -INFINITY ? 0.f : m_new;  // a row may see no slot of this range
        if (__builtin_amdgcn_ballot_w64(raise)) {
            const float corr = raise ? __builtin_amdgcn_exp2f(m_i - base) : 1.0f;
            l_i *= corr;
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[tt][r] *= corr;
        }
        m_i = m_new;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[u][r], scale, -base));
                sc[u][r] = p;
                l_i += p;
            }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int u = s >> 1, b = 8 * (s & 1);
            const bf16x8 pf = as_bf16x8(u32x4{pack_bf16x2(sc[u][b], sc[u][b + 1]), pack_bf16x2(sc[u][b + 2], sc[u][b + 3]),
                                              pack_bf16x2(sc[u][b + 4], sc[u][b + 5]), pack_bf16x2(sc[u][b + 6], sc[u][b + 7])});
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
                o[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(vt[(tt * 8 + 4 * H + s) * 64 + lane]), pf, o[tt], 0, 0, 0);
        }
    };
    if (t_begin < t_end) load(t_begin);
    for (int i = t_begin; i < t_end; ++i) {
        if (i > t_begin) __syncthreads();  // every wave is done with the tile before
        stage();
        __syncthreads();
        if (i + 1 < t_end) load(i + 1);
        const int key0 = i * kTileKeys;
        if (!active || key0 > wave_last) continue;
        half_tile(key0, std::integral_constant<int, 0>{});
        if (key0 + 64 <= wave_last) half_tile(key0 + 64, std::integral_constant<int, 1>{});
        if (nan_seen[0] | nan_seen[1] | nan_seen[2] | nan_seen[3]) {  // rows that see a group without numbers
            uint32_t groups = 0;
            for (int slot = key0; slot <= min(key0 + kTileKeys - 1, lim); ++slot)
#pragma unroll
                for (int g = 0; g < SB; ++g)
                    if (vs[(uint32_t)slot * SB + g] == kKv4Nan) groups |= 1u << g;
#pragma unroll
            for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int oct = ((r & 3) + 8 * (r >> 2) + 4 * hf) % NO;
                    if (groups >> (oct >> 2) & 1) o[tt][r] = NAN;
                }
        }
    }
    l_i = sum_xor32(l_i);
    if (!active || c0 + l32 >= cols) return;
    // register r of tile tt is channel 8 oct + tt PT + (m / NO), m = r % 4 + 8 (r / 4) + 4 hf, oct = m % NO: each octet's eight
    // channels are in this lane
    auto channel = [&](int oct_r, int e) -> float {  // oct_r: register that holds channel 0 of the octet (in tile 0)
        const int tt = e / PT, step = (e % PT) * NO;  // row m + step
        return o[tt][oct_r + step / 2];
    };
    if (sp.splits == 1) {
        const float inv = 1.0f / l_i;
        bf16_t *dst = out + (int64_t)(sp.row0 + where.row) * out_stride + where.head * D;
#pragma unroll
        for (int r = 0; r < NO / 2; ++r) {
            const int oct = (r & 3) + 8 * (r >> 2) + 4 * hf;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = channel(r, e) * inv;
            *reinterpret_cast<u32x4 *>(dst + 8 * oct) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        }
        if (lse && hf == 0) lse[(size_t)(sp.row0 + where.row) * view.nq + where.head] = m_i + __builtin_amdgcn_logf(l_i);
    } else {
        const size_t pr = (size_t)sp.part0 + ((size_t)z * sp.rows + where.row) * view.nq + where.head;
        float *dst = part_o + pr * D;
#pragma unroll
        for (int r = 0; r < NO / 2; ++r) {
            const int oct = (r & 3) + 8 * (r >> 2) + 4 * hf;
#pragma unroll
            for (int e = 0; e < 8; e += 4)
                *reinterpret_cast<float4 *>(dst + 8 * oct + e) = make_float4(channel(r, e), channel(r, e + 1), channel(r, e + 2), channel(r, e + 3));
        }
        if (hf == 0) *reinterpret_cast<float2 *>(part_ml + pr * 2) = make_float2(m_i, l_i);
    }
}

// ---------------------------------------------------------------------------------------
// Joins the key ranges of one row and head (a unit): WPU waves.  A lane takes the (max, sum) of one range, so that all of them
// are fetched at once; then D / 4 lanes add a range's output, four channels each, 64 WPU / (D / 4) ranges at a time.  A range
// whose slots the row does not see has sum 0 and an unused output.  Latency: 3 to 4.7 us; 4096 rows of 4 heads 9.2 us.
// ---------------------------------------------------------------------------------------
template <int D, int WPU>
__device__ __forceinline__ void join_unit(const Kv4Span &sp, int unit, bool live, int nq, const float *__restrict__ part_o,
                                          const float *__restrict__ part_ml, bf16_t *__restrict__ out, int64_t out_stride,
                                          float *__restrict__ lse, float4 *red) {
    constexpr int TPR = D / 4, PAR = 64 * WPU / TPR, kBatch = 8;  // PAR ranges at a time
    const int lane = threadIdx.x & 63, tid = threadIdx.x & (64 * WPU - 1), e = tid % TPR, g = tid / TPR;
    const size_t step = (size_t)sp.rows * nq, pr = (size_t)sp.part0 + unit;
    const float2 ml = live && lane < sp.splits ? reinterpret_cast<const float2 *>(part_ml)[pr + lane * step] : make_float2(-INFINITY, 0.f);
    const float4 *po = reinterpret_cast<const float4 *>(part_o) + pr * TPR + e;
    float4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = live && g + u * PAR < sp.splits ? po[(g + u * PAR) * step * TPR] : make_float4(0.f, 0.f, 0.f, 0.f);
    const float M = wave_max(ml.x);
    const float w = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    const float L = wave_sum(w == 0.f && ml.y == ml.y ? 0.f : w * ml.y);
    float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z0 = g; z0 - g < sp.splits; z0 += kBatch * PAR) {
        if (z0 != g)
#pragma unroll
            for (int u = 0; u < kBatch; ++u) v[u] = live && z0 + u * PAR < sp.splits ? po[(z0 + u * PAR) * step * TPR] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int z = z0 + u * PAR;
            const float wz = __shfl(w, z & 63, kWave), lz = __shfl(ml.y, z & 63, kWave);
            if (z < sp.splits && lz != 0.f)
                A.x = fmaf(wz, v[u].x, A.x), A.y = fmaf(wz, v[u].y, A.y), A.z = fmaf(wz, v[u].z, A.z), A.w = fmaf(wz, v[u].w, A.w);
        }
    }
    // the PAR sums, in order
    if (PAR > 1) {
        if (g) red[(g - 1) * TPR + e] = A;
        __syncthreads();
        if (g == 0)
#pragma unroll
            for (int i = 1; i < PAR; ++i) {
                const float4 x = red[(i - 1) * TPR + e];
                A.x += x.x, A.y += x.y, A.z += x.z, A.w += x.w;
            }
    }
    if (!live || g) return;
    const float inv = 1.0f / L;
    const int row = sp.row0 + unit / nq, head = unit % nq;
    *reinterpret_cast<u32x2 *>(out + (int64_t)row * out_stride + head * D + 4 * e) =
        u32x2{pack_bf16x2(A.x * inv, A.y * inv), pack_bf16x2(A.z * inv, A.w * inv)};
    if (lse && e == 0) lse[(size_t)row * nq + head] = M + __builtin_amdgcn_logf(L);
}

template <int D, int WPU, int CAP>
__global__ __launch_bounds__(256) void k_kv4_join(const Kv4Spans<CAP> t, int nq, const float *__restrict__ part_o,
                                                  const float *__restrict__ part_ml, bf16_t *__restrict__ out, int64_t out_stride,
                                                  float *__restrict__ lse) {
    constexpr int UPB = 4 / WPU, RED = (64 * WPU / (D / 4) - 1) * (D / 4);
    __shared__ float4 red[UPB][RED];
    const Kv4Span sp = t.s[blockIdx.y];
    if (sp.splits == 1 || (int)blockIdx.x * UPB >= sp.rows * nq) return;
    const int unit = blockIdx.x * UPB + threadIdx.x / (64 * WPU);
    join_unit<D, WPU>(sp, unit, unit < sp.rows * nq, nq, part_o, part_ml, out, out_stride, lse, red[threadIdx.x / (64 * WPU)]);
}

// ---------------------------------------------------------------------------------------
// Few columns: the weight each slot received, and the ranges' join beside it in the same launch.  Up to kScoreCols columns have
// left their scores in the workspace (STORED; four bytes a column and slot, where the keys would be 68), and a thread sums up a
// slot: 6 us for 16 tokens of 40 / 8 heads on 500 to 6000 slots, 10 from the keys.  For more, scores are formed once more from
// the keys (half of what the first kernel read, and mostly still in the last-level cache), as S = Q K^T: a lane then has one
// slot and four columns of each tile of 16, and the sum over the columns is three additions and two exchanges.  One lane owns a
// slot's sum: no atomics. A block works on the range of slots that the same block of k_kv4_few had; blocks past those join one
// unit each.
// ---------------------------------------------------------------------------------------
constexpr int kScoreCols = 8;

template <int D, int NT, bool STORED, int CAP>
__global__ __launch_bounds__(256) void k_kv4_few_weights(const Kv4Spans<CAP> t, const Kv4View view, const bf16_t *__restrict__ q,
                                                         int64_t q_stride, const float *__restrict__ part_o,
                                                         const float *__restrict__ part_ml, const float *__restrict__ lse,
                                                         int blocks, int join_rows, bf16_t *__restrict__ out, int64_t out_stride,
                                                         float *__restrict__ weights, const float *__restrict__ scores, int64_t score_stride) {
    constexpr int KS = D / 32, CB = D / 2, SB = D / 32;
    __shared__ float4 red[(256 / (D / 4) - 1) * (D / 4)];
    __shared__ float base_s[NT * 16];
    if ((int)blockIdx.x >= blocks) {
        const int x = blockIdx.x - blocks, per_span = join_rows * view.nq;
        const Kv4Span sp = t.s[x / per_span];
        const int unit = x % per_span;
        if (sp.splits == 1 || unit >= sp.rows * view.nq) return;
        join_unit<D, 4>(sp, unit, true, view.nq, part_o, part_ml, out, out_stride, nullptr, red);
        return;
    }
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, qd = lane >> 4, nkv = view.nkv, G = view.nq / nkv;
    const int kvh = (blockIdx.x - sp.blk0) % nkv, z = (blockIdx.x - sp.blk0) / nkv;
    const int n_keys = sp.len + sp.rows, last = n_keys - 1, n_tiles = (n_keys + kFewTile - 1) / kFewTile;
    const int t_begin = z * sp.per, t_end = min(n_tiles, t_begin + sp.per);
    const size_t head0 = ((size_t)sp.seq * nkv + kvh) * view.max_seq;
    const uint8_t *kc = view.k + head0 * CB, *ks = view.ks + head0 * SB;
    const int cols = sp.rows * G;
    const float scale = 1.4426950408889634f / sqrtf((float)D);
    bf16x8 qf[NT][KS];
    if constexpr (!STORED)
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const Column w = column_of(min(16 * c + m16, cols - 1), G, kvh);
            const bf16_t *src = q + (int64_t)(sp.row0 + w.row) * q_stride + w.head * D + qd * (D / 4);
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[c][s] = as_bf16x8(*reinterpret_cast<const u32x4 *>(src + 8 * s));
        }
    // log2 of the columns' softmax sums: wave c makes those of tile c, four lanes a column
    if (wave < NT) {
        const int col = min(16 * wave + m16, cols - 1);
        const Column w = column_of(col, G, kvh);
        float b;
        if (sp.splits == 1) {
            b = lse[(size_t)(sp.row0 + w.row) * view.nq + w.head];
        } else {
            const size_t step = (size_t)sp.rows * view.nq;
            const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + (size_t)sp.part0 + (size_t)w.row * view.nq + w.head;
            float2 r[kKv4Ranges / 4];
#pragma unroll
            for (int i = 0; i < kKv4Ranges / 4; ++i) r[i] = 4 * i + qd < sp.splits ? ml[(4 * i + qd) * step] : make_float2(-INFINITY, 0.f);
            float M = -INFINITY, L = 0.f, x, y;
#pragma unroll
            for (int i = 0; i < kKv4Ranges / 4; ++i) M = fmaxf(M, r[i].x);
            with_xor16(M, x, y);
            M = max_xor32(fmaxf(x, y));
#pragma unroll
            for (int i = 0; i < kKv4Ranges / 4; ++i)
                if (r[i].y != 0.f) L = fmaf(__builtin_amdgcn_exp2f(r[i].x - M), r[i].y, L);
            L = sum_xor32(sum_xor16(L));
            b = M + __builtin_amdgcn_logf(L);
        }
        if (qd == 0) base_s[16 * wave + m16] = b;
    }
    __syncthreads();
    float *dst = weights + head0;
    if constexpr (STORED) {
        const float *col[kScoreCols];
        int lim[kScoreCols];  // last slot the column sees
#pragma unroll
        for (int c = 0; c < kScoreCols; ++c) {
            const Column w = column_of(min(c, cols - 1), G, kvh);
            lim[c] = c < cols ? sp.len + w.row : -1;
            col[c] = scores + ((int64_t)(sp.row0 + w.row) * view.nq + w.head) * score_stride;
        }
        for (int key = t_begin * kFewTile + threadIdx.x; key < min(t_end * kFewTile, n_keys); key += 256) {
            float v[kScoreCols], sum = 0.f;
            const float was = dst[key];
#pragma unroll
            for (int c = 0; c < kScoreCols; ++c) v[c] = col[c][key];
#pragma unroll
            for (int c = 0; c < kScoreCols; ++c) {  // (selected, as a row without numbers has none for the slots it does not see either)
                const float p = __builtin_amdgcn_exp2f(fmaf(v[c], scale, -base_s[c]));
                sum += key <= lim[c] ? p : 0.f;
            }
            dst[key] = was + sum;
        }
        return;
    }
    float base[NT][4];
    int lim[NT][4];
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int col = 16 * c + 4 * qd + r;
            base[c][r] = base_s[col], lim[c][r] = col < cols ? sp.len + col / G : -1;
        }
    for (int tile = t_begin + wave; tile < t_end; tile += kFewWaves) {
        const int key0 = tile * kFewTile;
        const int key = key0 + 16 * (qd & 1) + m16;  // the slot whose sum lanes of quarters 0 and 1 write
        float was = 0.f;
        if (qd < 2 && key < n_keys) was = dst[key];
        float sum[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t slot = min(key0 + 16 * u + m16, last);
            f32x4 sc[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c) sc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
            uint32_t w[KS];
            float unit;
            if constexpr (D == 128) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(kc + slot * CB + qd * 16);
                w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
                unit = kv4_scale(ks[slot * SB + qd]);
            } else {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(kc + slot * CB + qd * 8);
                w[0] = x.x, w[1] = x.y;
                unit = kv4_scale(ks[slot * SB + (qd >> 1)]);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 kf = as_bf16x8(keys8(w[s], unit));
#pragma unroll
                for (int c = 0; c < NT; ++c) sc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[c][s], kf, sc[c], 0, 0, 0);
            }
            sum[u] = 0.f;
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(sc[c][r], scale, -base[c][r]));
                    sum[u] += key0 + 16 * u + m16 <= lim[c][r] ? p : 0.f;
                }
            sum[u] = sum_xor32(sum_xor16(sum[u]));
        }
        if (qd < 2 && key < n_keys) dst[key] = was + (qd ? sum[1] : sum[0]);
    }
}

// ---------------------------------------------------------------------------------------
// Chunks: the weight each slot received, sum over the columns that see it of exp2(score - lse), the scores formed once more (K
// only).  A block is 64 slots, its keys in registers as bf16; its W waves take every W-th tile of 32 columns, S = Q K^T, so
// that a lane has one slot and the sum over the columns stays in the lane.  One block owns a slot's sum: no atomics, the same
// order in every run.  2048 rows of 40 / 8 heads on 4096 slots 202 us, 0.53 PFLOP/s (the products alone at a large product's rate:
// 78); 86 rows 13.2 us.  The vector pipe is busy for 54 % of the cycles (an exponential and two more operations a score), the matrix
// pipe for 23 %; a wave waits 41 % of its own for its turn and 18 % for loads and LDS, as each stages its columns by itself.
// ---------------------------------------------------------------------------------------
constexpr int kWeightKeys = 64;

template <int D, int W, int CAP>
__global__ __launch_bounds__(64 * W, W == 4 ? 3 : 2) void k_kv4_weights(const Kv4Spans<CAP> t, const Kv4View view, const bf16_t *__restrict__ q,
                                                        int64_t q_stride, const float *__restrict__ lse, float *__restrict__ weights) {
    constexpr int CB = D / 2, SB = D / 32, ST = D / 16;
    constexpr int LPR = D / 8, RPL = 64 / LPR, LD = LPR + 1;  // lanes of a column's 2 D bytes, columns of a load, 16-byte words of a column in LDS
    __shared__ float sums[W][kWeightKeys];
    __shared__ u32x4 qs[W][32 * LD];
    __shared__ float4 base_s[W][8];
    __shared__ int4 lim_s[W][8];
    const Kv4Span sp = t.s[kv4_span_of(t, blockIdx.x)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, hf = lane >> 5, nkv = view.nkv, G = view.nq / nkv, cols = sp.rows * G;
    const int kvh = (blockIdx.x - sp.blk0) % nkv, key0 = (blockIdx.x - sp.blk0) / nkv * kWeightKeys;
    const int last = sp.len + sp.rows - 1;
    const size_t head0 = ((size_t)sp.seq * nkv + kvh) * view.max_seq;
    const uint8_t *kc = view.k + head0 * CB, *ks = view.ks + head0 * SB;
    const float scale = 1.4426950408889634f / sqrtf((float)D);
    const uint32_t inverse = (uint32_t)((0x100000000ull + G - 1) / G);  // col / G for col < 2^24, G of 2 to 16
    auto column = [&](int col) {
        const int row = G == 1 ? col : (int)__umulhi((uint32_t)col, inverse);
        return Column{row, kvh * G + col - row * G};
    };
    int ct = max(0, key0 - sp.len) * G / 32 + wave;  // the columns before see none of the block
    u32x4 qw[32 / RPL];
    float base;
    int lim;
    // A load is whole columns, side by side (a lane's own column would be a line of its own for each lane); LDS brings them
    // into the operand's order.
    auto load = [&]() {
        const Column own = column(min(ct * 32 + l32, cols - 1));
        lim = ct * 32 + l32 < cols ? sp.len + own.row : -1;
        base = lse[(size_t)(sp.row0 + own.row) * view.nq + own.head];
#pragma unroll
        for (int i = 0; i < 32 / RPL; ++i) {
            const Column w = column(min(ct * 32 + i * RPL + lane / LPR, cols - 1));
            qw[i] = *reinterpret_cast<const u32x4 *>(q + (int64_t)(sp.row0 + w.row) * q_stride + w.head * D + lane % LPR * 8);
        }
    };
    if (ct * 32 < cols) load();
    const bool owns = threadIdx.x < kWeightKeys && key0 + (int)threadIdx.x <= last;
    float *dst = weights + head0 + key0 + threadIdx.x;
    const float was = owns ? *dst : 0.f;
    bf16x8 kf[2][ST];  // slot key0 + 32 u + l32, channels hf D / 2 + 8 s
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint32_t slot = min(key0 + 32 * u + l32, last);
#pragma unroll
        for (int g = 0; g < D / 64; ++g) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(kc + slot * CB + hf * (CB / 2) + 16 * g);
            const float unit = kv4_scale(ks[slot * SB + hf * (SB / 2) + g]);
#pragma unroll
            for (int c = 0; c < 4; ++c) kf[u][4 * g + c] = as_bf16x8(keys8(w[c], unit));
        }
    }
    float acc[2] = {0.f, 0.f};
    while (ct * 32 < cols) {
        const bool all = ct * 32 + 31 < cols && sp.len + ct * 32 / G >= key0 + kWeightKeys - 1;  // every column sees every slot
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 32 / RPL; ++i) qs[wave][(i * RPL + lane / LPR) * LD + lane % LPR] = qw[i];
        if (hf == 0) {
            reinterpret_cast<float *>(base_s[wave])[l32] = base;
            reinterpret_cast<int *>(lim_s[wave])[l32] = lim;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        f32x16 sc[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[0][r] = sc[1][r] = 0.f;
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            const bf16x8 qf = as_bf16x8(qs[wave][l32 * LD + hf * (LPR / 2) + s]);
#pragma unroll
            for (int u = 0; u < 2; ++u) sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[u][s], sc[u], 0, 0, 0);
        }
        ct += W;
        if (ct * 32 < cols) load();  // beside the exponentials
        // register r is column (r & 3) + 8 (r >> 2) + 4 hf
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 b4 = base_s[wave][2 * i + hf];
            const float b[4] = {b4.x, b4.y, b4.z, b4.w};
            if (all) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[u] += __builtin_amdgcn_exp2f(fmaf(sc[u][4 * i + r], scale, -b[r]));
            } else {
                const int4 l4 = lim_s[wave][2 * i + hf];
                const int l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(sc[u][4 * i + r], scale, -b[r]));
                        acc[u] += key0 + 32 * u + l32 <= l[r] ? p : 0.f;
                    }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float v = sum_xor32(acc[u]);
        if (hf == 0) sums[wave][32 * u + l32] = v;
    }
    __syncthreads();
    if (owns) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += sums[w][threadIdx.x];
        *dst = was + v;
    }
}

// ---------------------------------------------------------------------------------------
// launcher
// ---------------------------------------------------------------------------------------
// Cuts the spans' tiles of `tile` slots into ranges of Kv4Span::per tiles (a multiple of `step`, at least `whole` of them if no
// span has more), as short as leaves at most `want` blocks, kKv4Ranges ranges and the partial results within their buffer;
// returns the blocks.  blocks_of(span): blocks of one range.  (Steps grow with the range: a long context with few rows tries
// some dozen lengths, not thousands.)
template <class F>
static int cut_ranges(const Kv4 &k, Kv4Table &t, int tile, int step, int whole, int want, F blocks_of) {
    const int64_t nq = k.c.n_q_heads;
    int64_t work = 0;
    int most = 1;
    for (int j = 0; j < t.n; ++j) {
        if (!t.s[j].rows) continue;
        const int tiles = (t.s[j].len + t.s[j].rows + tile - 1) / tile;
        work += (int64_t)blocks_of(t.s[j]) * tiles;
        most = tiles > most ? tiles : most;
    }
    const int64_t least = (most + kKv4Ranges - 1) / kKv4Ranges, even = work / want;
    int64_t per = ((even > least ? even : least) + step - 1) / step * step;
    if (most <= whole && per < whole) per = whole;
    for (per = per ? per : step;; per += (per / 16 + step) / step * step) {
        int64_t blk = 0, part = 0;
        for (int j = 0; j < t.n; ++j) {
            Kv4Span &s = t.s[j];
            const int tiles = s.rows ? (s.len + s.rows + tile - 1) / tile : 0;
            s.splits = s.rows ? (int)((tiles + per - 1) / per) : 1;
            s.blk0 = (int)blk, s.part0 = (int)part, s.per = (int)per;
            if (s.rows) blk += (int64_t)blocks_of(s) * s.splits;
            if (s.splits > 1) part += (int64_t)s.splits * s.rows * nq;
        }
        if ((blk <= want && part <= (int64_t)k.part_rows) || per >= most) return (int)blk;
    }
}

Kv4AttendPlan plan_kv4_attend(const Kv4 &k, Kv4Table &t, bool weights) {
    const int nkv = k.c.n_kv_heads, G = k.c.n_q_heads / nkv;
    int64_t most = 0, few_tiles = 0, chunk_tiles = 0;
    for (int j = 0; j < t.n; ++j) {
        if (!t.s[j].rows) continue;
        const int64_t cols = (int64_t)t.s[j].rows * G, held = t.s[j].len + t.s[j].rows;
        most = cols > most ? cols : most;
        few_tiles += (cols + 31) / 32 * nkv * ((held + kFewTile - 1) / kFewTile);
        chunk_tiles += (cols + kTileCols - 1) / kTileCols * nkv * ((held + kTileKeys - 1) / kTileKeys);
    }
    // k_kv4_chunk takes longer to get going and to join its larger partial results, k_kv4_few dequantises for 32 columns at a
    // time: a line between them over the tiles of 32 x 32 and of 128 x 128 that each has, fitted to 96 shapes of 1 to 32
    // sequences (0.8 % lost to the better form in the mean).  40 / 8 heads on 4096 slots, few against chunk: 20 rows 15.2 :
    // 21.5 us, 86 rows 26.6 : 31.7, 200 rows 35.9 : 44.5, 300 rows 55.6 : 53.2, 500 rows 83.6 : 74.8; 12 sequences with 150 to
    // 300 rows on 128 to 1500 slots 110 : 76.
    const bool few = most <= 16 || few_tiles <= 10000 + 116 * chunk_tiles / 10;
    // The weights of up to 64 columns beside the join, in one launch; of more than 32 only while that launch is short.  Rows of
    // 40 / 8 heads, one launch against two: 4 sequences x 12 rows on 500 to 4000 slots 22.6 : 23.7 us, 16 x 12 rows 69.2 :
    // 57.4, 16 x 6 rows 32.8 : 45.6.
    const bool fused = weights && few && (most <= 32 || (most <= 64 && few_tiles <= 6000));
    Kv4AttendPlan p{most <= 16 ? 16 : few ? 32 : kTileCols, 0, 0, most, fused, 0, 0};
    auto groups = [&](const Kv4Span &s) { return nkv * ((s.rows * G + p.cols - 1) / p.cols); };
    // A call that fills `want` blocks as it is stays uncut, so it lasts as long as its longest span: 40 / 8 heads, a single token on
    // 16001 slots beside 32 on 201 slots 13.5 us (32 ranges), beside 63 of them, which are 512 blocks, 93 (one range).  256 blocks
    // of 32 columns were measured on single spans.
    // Up to 512 slots stay in one range where a join would be a launch of its own: one row of 12 / 2 heads on 128 slots 4.1 us
    // against 6.5, on 512 6.2 against 6.7; 16 rows of 40 / 8 heads on 512 slots each 6.7 against 9.6.  (On 1024 slots 8.7
    // against 6.7.)
    const int whole = few && !p.fused ? 512 / kFewTile : 0;
    p.blocks = cut_ranges(k, t, few ? kFewTile : kTileKeys, few ? kFewWaves : 1, whole, p.cols == 32 ? 256 : kKv4Blocks, groups);
    int64_t rows = 0, longest = 0, parts = 0;
    for (int j = 0; j < t.n; ++j) {
        const Kv4Span &s = t.s[j];
        if (!s.rows) continue;
        rows += s.rows;
        longest = s.len + s.rows > longest ? s.len + s.rows : longest;
        if (s.splits > 1) {
            parts += (int64_t)s.splits * s.rows * k.c.n_q_heads;
            p.join = s.rows > p.join ? s.rows : p.join;
        }
    }
    // Scores are kept behind the partial outputs where there is room: 16 single tokens of 40 / 8 heads on 500 to 6000 slots
    // 21.6 us with them, 24.2 without; 64 on 500 to 1500 slots 25.9 against 30.3.
    const int64_t stride = (longest + kFewTile - 1) / kFewTile * kFewTile, at = parts * k.c.head_dim;
    if (p.fused && most <= kScoreCols && at + rows * k.c.n_q_heads * stride <= (int64_t)k.part_floats) p.score_at = at, p.score_stride = stride;
    return p;
}

int launch_kv4_attend(const Kv4 &k, int layer, Kv4Table &t, const bf16_t *q, int64_t q_stride, bf16_t *out, int64_t out_stride,
                      float *weights) {
    const int nkv = k.c.n_kv_heads, D = k.c.head_dim;
    const Kv4View view = k.view(layer);
    float *lse = weights ? k.lse : nullptr;
    const Kv4AttendPlan plan = plan_kv4_attend(k, t, weights);
    const bool few = plan.cols < kTileCols, fused = plan.fused;
    const int blocks = plan.blocks, join = plan.join;
    const int64_t most = plan.most, score_stride = plan.score_stride;
    float *scores = score_stride ? k.part_o + plan.score_at : nullptr;
    int64_t weight_blocks = 0;  // of k_kv4_weights
    if (weights && !fused)
        for (int j = 0; j < t.n; ++j)
            if (t.s[j].rows) weight_blocks += (int64_t)nkv * ((t.s[j].len + t.s[j].rows + kWeightKeys - 1) / kWeightKeys);
    // a launch has at most 2^32 - 1 threads a direction (asked before anything is launched)
    if (weight_blocks >= 1 << 24) return fail(ST_ERANGE, "weights of 2^30 slots or more, over all spans and kv heads");
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        const int nq = k.c.n_q_heads, units = join * nq;
#define ST_FEW(DV, NTV)                                                                                                                  \
    hipLaunchKernelGGL((k_kv4_few<DV, NTV, CAP>), dim3(blocks), dim3(256), 0, k.stream, tab, view, q, q_stride, out, out_stride, k.part_o, \
                       k.part_ml, lse, scores, score_stride)
        if (few && most <= 16) {
            if (D == 128) ST_FEW(128, 1);
            else ST_FEW(64, 1);
        } else if (few) {
            if (D == 128) ST_FEW(128, 2);
            else ST_FEW(64, 2);
        } else {
            auto *kern = D == 128 ? k_kv4_chunk<128, CAP> : k_kv4_chunk<64, CAP>;
            hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, k.stream, tab, view, q, q_stride, out, out_stride, k.part_o, k.part_ml, lse);
        }
#undef ST_FEW
        if (fused) {
            int blk = 0;  // one block for all columns of a range
            for (int j = 0; j < tab.n; ++j) {
                tab.s[j].blk0 = blk;
                if (tab.s[j].rows) blk += nkv * tab.s[j].splits;
            }
#define ST_FEW_WEIGHTS(DV, NTV, STORED)                                                                                                   \
    hipLaunchKernelGGL((k_kv4_few_weights<DV, NTV, STORED, CAP>), dim3(blk + units * tab.n), dim3(256), 0, k.stream, tab, view, q, q_stride, k.part_o, \
                       k.part_ml, lse, blk, join, out, out_stride, weights, scores, score_stride)
            if (D == 128) {
                if (scores) ST_FEW_WEIGHTS(128, 1, true);
                else if (most <= 16) ST_FEW_WEIGHTS(128, 1, false);
                else if (most <= 32) ST_FEW_WEIGHTS(128, 2, false);
                else ST_FEW_WEIGHTS(128, 4, false);
            } else {
                if (scores) ST_FEW_WEIGHTS(64, 1, true);
                else if (most <= 16) ST_FEW_WEIGHTS(64, 1, false);
                else if (most <= 32) ST_FEW_WEIGHTS(64, 2, false);
                else ST_FEW_WEIGHTS(64, 4, false);
            }
#undef ST_FEW_WEIGHTS
        }
        if (join && !fused) {
            // four waves a unit while there are fewer units than would fill the chip with one each
            const bool wide = units * t.n < 1024;
            auto *kern = D == 128 ? (wide ? k_kv4_join<128, 4, CAP> : k_kv4_join<128, 1, CAP>) : (wide ? k_kv4_join<64, 4, CAP> : k_kv4_join<64, 1, CAP>);
            hipLaunchKernelGGL(kern, dim3(wide ? units : (units + 3) / 4, t.n), dim3(256), 0, k.stream, tab, nq, k.part_o, k.part_ml,
                               out, out_stride, lse);
        }
    });
    if (weights && !fused) {
        int blk = 0;
        for (int j = 0; j < t.n; ++j) {
            t.s[j].blk0 = blk;
            if (t.s[j].rows) blk += nkv * ((t.s[j].len + t.s[j].rows + kWeightKeys - 1) / kWeightKeys);
        }
        with_table(t, [&](auto tab) {
            constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
            // Eight waves share a block's columns while there is at most one block a compute unit: 125 rows of 12 / 2 heads on
            // 3000 slots 23.6 us with the attention against 26.4, 86 rows of 40 / 8 heads on 4096 (528 blocks) 44.6 against
            // 40.4.
            const bool wide = weight_blocks <= 256;
            auto *kern = D == 128 ? (wide ? k_kv4_weights<128, 8, CAP> : k_kv4_weights<128, 4, CAP>) : (wide ? k_kv4_weights<64, 8, CAP> : k_kv4_weights<64, 4, CAP>);
            hipLaunchKernelGGL(kern, dim3(weight_blocks), dim3(wide ? 512 : 256), 0, k.stream, tab, view, q, q_stride, lse, weights);
        });
    }
    return ST_OK;
}

}  // namespace st
