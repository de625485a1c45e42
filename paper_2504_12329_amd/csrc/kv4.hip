// A key/value cache held in 4 bits: the C entry points, and the two kernels that write and read single slots (append with the
// norms of queries and keys and the rotation, and read).
//
// Format.  32 neighbouring channels of a head form a group with one scale 2^s, held as the byte s + 127, and 4-bit codes: sign
// and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6.  s is the least with max |x| <= 7 * 2^s: the largest value is then clipped by less
// than the rounding of its neighbours costs (mean error on normal data 19.0 dB below the data, against 18.75 with max |x| <= 6
// * 2^s).  A slot is head_dim / 2 bytes of codes and head_dim / 32 of scales, in planes of their own, so that a wave reads
// whole lines of codes.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "checks.h"
#include "kv4.h"
#include "st_device.h"

namespace st {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------
// Append.  D/8 threads per head; a thread owns four neighbouring channels of each half of the head, i.e. four rotation pairs,
// so that norm, rotation and quantisation need no exchange but the group's maximum (8 lanes) and the norm's sum.  Bound by
// memory: 2 bytes per channel in, 2 out for the queries, 4.25 bits for keys and values.  4096 rows of 40 / 8 heads, 105 MB and 2
// of the rotation table, 20.9 us, 5.1 TB/s (a large copy: 5.1); 16 rows 3.5 us.  64 channels, 4096 rows of 4 / 2 heads: 4.4 us.
//
// Every product and sum is rounded to fp32 by itself (no contraction) and the sum of squares adds neighbours first, so the
// codes are a function of the inputs alone: no choice of the kernel's shape shows in them.
// ---------------------------------------------------------------------------------------
// sum / largest over the lanes of a group of 8 (16): quad swaps, then the mirrors, as every lane of a quad then holds the same
__device__ __forceinline__ float sum_of_4(float v) {
    v += dpp_move<0xB1, 0xf>(0.f, v);
    return v + dpp_move<0x4E, 0xf>(0.f, v);
}
__device__ __forceinline__ uint32_t max_over_8(uint32_t v) {
    auto step = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));
    v = step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));
    return step(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));
}

// Scale byte of a group whose largest |x| has the bits `top`
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7f800000u) return kKv4Nan;
    // top = f * 2^e, 1 <= f < 2: s = e - 2 while f <= 7/4, else e - 1
    const int s = (int)(top >> 23) - 127 - ((top & 0x7fffffu) <= 0x600000u ? 2 : 1);
    return (uint32_t)(min(max(s, -100), 125) + 127);
}

template <int D, int CAP>
__global__ __launch_bounds__(256) void k_kv4_append(const Kv4Spans<CAP> t, const Kv4View view, const bf16_t *__restrict__ qkv,
                                                    int64_t qkv_stride, const bf16_t *__restrict__ q_norm,
                                                    const bf16_t *__restrict__ k_norm, float eps,
                                                    const float *__restrict__ rope, bf16_t *__restrict__ q_out,
                                                    int64_t q_stride, float *__restrict__ weights,
                                                    int32_t *__restrict__ positions) {
#pragma clang fp contract(off)
    constexpr int TPH = D / 8, HPB = 256 / TPH;
    const int nq = view.nq, nkv = view.nkv, row = blockIdx.x;
    const Kv4Span sp = t.s[kv4_span_of(t, row)];
    const int i = row - sp.row0, head = blockIdx.y * HPB + threadIdx.x / TPH, l = threadIdx.x % TPH;
    if (head >= nq + 2 * nkv) return;
    const bf16_t *src = qkv + row * qkv_stride + head * D + 4 * l;
    const u32x2 wl = *reinterpret_cast<const u32x2 *>(src), wh = *reinterpret_cast<const u32x2 *>(src + D / 2);
    float lo[4] = {bf16_lo(wl.x), bf16_hi(wl.x), bf16_lo(wl.y), bf16_hi(wl.y)};
    float hi[4] = {bf16_lo(wh.x), bf16_hi(wh.x), bf16_lo(wh.y), bf16_hi(wh.y)};
    if (head < nq + nkv) {
        const float4 *at = reinterpret_cast<const float4 *>(rope + ((size_t)(sp.pos + i) * (D / 2) + 4 * l) * 2);
        const float4 a01 = at[0], a23 = at[1];
        const bf16_t *norm = head < nq ? q_norm : k_norm;
        if (norm) {
            const u32x2 nl = *reinterpret_cast<const u32x2 *>(norm + 4 * l), nh = *reinterpret_cast<const u32x2 *>(norm + D / 2 + 4 * l);
            const float gl[4] = {bf16_lo(nl.x), bf16_hi(nl.x), bf16_lo(nl.y), bf16_hi(nl.y)};
            const float gh[4] = {bf16_lo(nh.x), bf16_hi(nh.x), bf16_lo(nh.y), bf16_hi(nh.y)};
            auto half_sum = [](const float *x) {  // of the half's channels, neighbours first
                float v = (x[0] * x[0] + x[1] * x[1]) + (x[2] * x[2] + x[3] * x[3]);
                v = sum_of_4(v);
                v += dpp_move<0x141, 0xf>(0.f, v);
                if constexpr (D == 128) v += dpp_move<0x140, 0xf>(0.f, v);
                return v;
            };
            const float sum = half_sum(lo) + half_sum(hi);
            const float r = 1.0f / sqrtf(sum / D + eps);
#pragma unroll
            for (int e = 0; e < 4; ++e) lo[e] = lo[e] * r * gl[e], hi[e] = hi[e] * r * gh[e];
        }
        const float cx[4] = {a01.x, a01.z, a23.x, a23.z}, sy[4] = {a01.y, a01.w, a23.y, a23.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = lo[e] * cx[e] - hi[e] * sy[e];
            hi[e] = hi[e] * cx[e] + lo[e] * sy[e];
            lo[e] = a;
        }
    }
    if (head < nq) {
        bf16_t *dst = q_out + row * q_stride + head * D + 4 * l;
        *reinterpret_cast<u32x2 *>(dst) = u32x2{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3])};
        *reinterpret_cast<u32x2 *>(dst + D / 2) = u32x2{pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
        return;
    }
    const bool is_k = head < nq + nkv;
    const size_t at = ((size_t)sp.seq * nkv + (head - nq - (is_k ? 0 : nkv))) * view.max_seq + sp.len + i;
    uint8_t *codes = (is_k ? view.k : view.v) + at * (D / 2), *scales = (is_k ? view.ks : view.vs) + at * (D / 32);
    auto quantise = [&](const float *x, int half) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        const uint32_t byte = scale_byte(max_over_8(top));
        uint32_t w = 0;
        if (byte != kKv4Nan) {
            const float unit = kv4_scale(byte);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
        }
        *reinterpret_cast<uint16_t *>(codes + half * (D / 4) + 2 * l) = (uint16_t)w;
        if ((l & 7) == 0) scales[half * (D / 64) + (l >> 3)] = (uint8_t)byte;
    };
    quantise(lo, 0);
    quantise(hi, 1);
    if (positions && is_k && l == 0) {
        positions[at] = sp.pos + i;
        weights[at] = 0.f;
    }
}

// ---------------------------------------------------------------------------------------
// Read: slots [len, len + rows) of every span as the bf16 numbers they stand for (each is one exactly).  A thread turns four
// bytes of codes into 16 of output; 1 << shift waves have RPW rows, so that heads too few for a block share it with other rows.
// Bound by memory.
// ---------------------------------------------------------------------------------------
template <int D, int RPW, int CAP>
__global__ __launch_bounds__(256) void k_kv4_read(const Kv4Spans<CAP> t, Kv4View view, size_t k_layer, size_t s_layer, int rows, int shift,
                                                  bf16_t *__restrict__ k_out, bf16_t *__restrict__ v_out) {
    constexpr int TPH = D / 8;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), layer = blockIdx.y;
    const int first = (((blockIdx.x << 2) + wave) >> shift) * RPW;
    size_t slot[RPW];
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
        const int row = min(first + r, rows - 1);
        const Kv4Span sp = t.s[kv4_span_of(t, row)];
        slot[r] = (size_t)sp.seq * view.nkv * view.max_seq + sp.len + (row - sp.row0);
    }
    for (int u = (wave & ((1 << shift) - 1)) * 64 + (threadIdx.x & 63); u < 2 * view.nkv * TPH; u += 64 << shift) {
        const bool is_k = u < view.nkv * TPH;
        const int x = is_k ? u : u - view.nkv * TPH, head = x / TPH, l = x % TPH;
        const uint8_t *codes = (is_k ? view.k : view.v) + layer * k_layer + 4 * l;
        const uint8_t *scales = (is_k ? view.ks : view.vs) + layer * s_layer + (l >> 2);
        bf16_t *out = (is_k ? k_out : v_out) + ((size_t)layer * rows + first) * view.nkv * D + head * D + 8 * l;
        uint32_t w[RPW], byte[RPW];
#pragma unroll
        for (int r = 0; r < RPW; ++r) {
            const size_t at = slot[r] + (size_t)head * view.max_seq;
            w[r] = *reinterpret_cast<const uint32_t *>(codes + at * (D / 2));
            byte[r] = scales[at * (D / 32)];
        }
#pragma unroll
        for (int r = 0; r < RPW; ++r) {
            if (first + r >= rows) break;
            const float unit = kv4_scale(byte[r]);
            u32x4 o = {kv4_pair<0>(w[r], unit), kv4_pair<1>(w[r], unit), kv4_pair<2>(w[r], unit), kv4_pair<3>(w[r], unit)};
            if (byte[r] == kKv4Nan) o = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
            *reinterpret_cast<u32x4 *>(out + (size_t)r * view.nkv * D) = o;
        }
    }
}

template <class T>
static void by_rows(T &t) {  // block = row
    for (int j = 0; j < t.n; ++j) t.s[j].blk0 = t.s[j].row0;
}

void launch_kv4_append(const Kv4 &k, int layer, const Kv4Table &t, int rows, const bf16_t *qkv, int64_t qkv_stride,
                       const bf16_t *q_norm, const bf16_t *k_norm, bf16_t *q_out, int64_t q_stride, float *weights,
                       int32_t *positions) {
    const int per_block = 256 / (k.c.head_dim / 8), heads = k.c.n_q_heads + 2 * k.c.n_kv_heads;
    const dim3 grid(rows, (heads + per_block - 1) / per_block);
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        auto *kern = k.c.head_dim == 128 ? k_kv4_append<128, CAP> : k_kv4_append<64, CAP>;
        by_rows(tab);
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, k.stream, tab, k.view(layer), qkv, qkv_stride, q_norm, k_norm, k.c.rms_eps,
                           k.rope, q_out, q_stride, weights, positions);
    });
}

void launch_kv4_read(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int rows, bf16_t *k_out, bf16_t *v_out) {
    const int units = 2 * k.c.n_kv_heads * (k.c.head_dim / 8), shift = units > 128 ? 2 : units > 64 ? 1 : 0, layers = layer_hi - layer_lo;
    // Two rows a wave once that leaves the chip full: 16 x 1024 rows of 8 heads 16.8 us against 19.8 (5.1 TB/s), 28 x 512 of 2
    // heads 5.8 against 6.2; 12 x 35 of 4 heads 2.8 against 2.5.
    const bool many = (int64_t)rows * layers << shift >= 12288;
    const int groups = many ? (rows + 1) / 2 : rows;
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        auto *kern = k.c.head_dim == 128 ? (many ? k_kv4_read<128, 2, CAP> : k_kv4_read<128, 1, CAP>) : (many ? k_kv4_read<64, 2, CAP> : k_kv4_read<64, 1, CAP>);
        by_rows(tab);
        hipLaunchKernelGGL(kern, dim3((((int64_t)groups << shift) + 3) / 4, layers), dim3(256), 0, k.stream, tab, k.view(layer_lo), k.per_layer[0],
                           k.per_layer[2], rows, shift, k_out, v_out);
    });
}

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
static int check_config(const st_kv4_config *c) {
    if (!c) return fail(ST_EINVAL, "config is NULL");
    if (c->n_layers <= 0 || c->n_seq <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->max_seq <= 0 || c->max_rows <= 0 ||
        c->max_pos <= 0)
        return fail(ST_EINVAL, "config has a non-positive dimension");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(ST_EINVAL, "head_dim must be 64 or 128");
    if (c->n_q_heads % c->n_kv_heads) return fail(ST_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
    if (c->n_q_heads / c->n_kv_heads > 16) return fail(ST_EINVAL, "at most 16 query heads per kv head");
    if (c->n_q_heads > 4096) return fail(ST_EINVAL, "at most 4096 query heads");
    if (c->n_layers > 65535) return fail(ST_EINVAL, "at most 65535 layers");
    if (c->max_seq > 1 << 24 || c->max_rows > 1 << 20) return fail(ST_EINVAL, "max_seq must be <= 2^24 and max_rows <= 2^20");
    if (!(c->rms_eps >= 0.f) || std::isinf(c->rms_eps)) return fail(ST_EINVAL, "bad rms_eps");
    // 2^46 bytes is far more than any device has, and every size below then fits 64 bits
    if ((double)c->n_layers * c->n_seq * c->n_kv_heads * c->max_seq * c->head_dim > 0x1p46)
        return fail(ST_EINVAL, "the cache would be larger than 2^46 bytes");
    return ST_OK;
}

// The planes and the workspace; with cache / ws == nullptr the record only has sizes that matter.
static void carve(const st_kv4_config &c, char *cache, char *ws, Kv4 *k, size_t *cache_bytes, size_t *ws_bytes) {
    size_t off = 0;
    const size_t slots = (size_t)c.n_seq * c.n_kv_heads * c.max_seq;
    for (int p = 0; p < 4; ++p) {
        k->per_layer[p] = slots * (c.head_dim / (p < 2 ? 2 : 32));
        k->plane[p] = reinterpret_cast<uint8_t *>(cache ? cache + off : nullptr);
        off += up256(k->per_layer[p] * c.n_layers);
    }
    *cache_bytes = off;
    off = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? ws + off : nullptr;
        off += up256(bytes);
        return p;
    };
    // A launch that cuts ranges has at most 512 blocks, of at most 128 columns each, and at most 64 ranges of a row.
    const size_t columns = (size_t)c.max_rows * c.n_q_heads * kKv4Ranges, blocks = (size_t)kKv4Blocks * kKv4Columns;
    k->part_rows = columns < blocks ? columns : blocks;
    k->lse = reinterpret_cast<float *>(take(sizeof(float) * c.max_rows * (size_t)c.n_q_heads));
    k->part_ml = reinterpret_cast<float *>(take(sizeof(float) * 2 * k->part_rows));
    // (and scores: of single rows over all slots, as far as the largest partial results' room goes)
    const size_t score_rows = (size_t)(c.max_rows < ST_KV4_MAX_SPANS ? c.max_rows : ST_KV4_MAX_SPANS) * c.n_q_heads;
    const size_t wanted = k->part_rows * c.head_dim + score_rows * (((size_t)c.max_seq + 31) & ~(size_t)31), most = blocks * 128;
    k->part_floats = std::max(k->part_rows * c.head_dim, std::min(wanted, most));
    k->part_o = reinterpret_cast<float *>(take(sizeof(float) * k->part_floats));
    k->kept_words = ((size_t)c.max_seq + 63) / 64;
    const size_t spans = c.n_seq < ST_KV4_MAX_SPANS ? c.n_seq : ST_KV4_MAX_SPANS;
    k->kept = reinterpret_cast<uint64_t *>(take(sizeof(uint64_t) * c.n_layers * spans * c.n_kv_heads * k->kept_words));
    *ws_bytes = off;
}

// Checks the spans and deals the rows to them.  With `positions` they must lie in the rotation table.
static int take_spans(const Kv4 &k, const st_kv4_span *spans, int32_t n, bool positions, Kv4Table *t, int *rows) {
    const st_kv4_config &c = k.c;
    if (n < 0 || n > ST_KV4_MAX_SPANS) return fail(ST_EINVAL, "%d spans, 0 to %d are supported", n, ST_KV4_MAX_SPANS);
    if (n && !spans) return fail(ST_EINVAL, "spans is NULL");
    int64_t total = 0;
    for (int j = 0; j < n; ++j) {
        const st_kv4_span &s = spans[j];
        if (s.seq < 0 || s.seq >= c.n_seq) return fail(ST_ERANGE, "span %d: sequence %d outside [0, %d)", j, s.seq, c.n_seq);
        if (s.len < 0 || s.rows < 0 || (int64_t)s.len + s.rows > c.max_seq)
            return fail(ST_ERANGE, "span %d: %d slots + %d rows, capacity %d", j, s.len, s.rows, c.max_seq);
        if (s.pos < 0 || (positions && (int64_t)s.pos + s.rows > c.max_pos))
            return fail(ST_ERANGE, "span %d: positions from %d, %d rows, table of %d", j, s.pos, s.rows, c.max_pos);
        for (int i = 0; i < j; ++i)
            if (spans[i].seq == s.seq) return fail(ST_EINVAL, "spans %d and %d are both sequence %d", i, j, s.seq);
        t->s[j] = Kv4Span{s.seq, s.len, s.pos, s.rows, (int32_t)total, 0, 1, 0, 0};
        total += s.rows;
        if (total >= 1 << 24) return fail(ST_ERANGE, "2^24 rows or more");  // a launch has at most 2^32 - 1 threads a direction
    }
    t->n = n;
    *rows = (int)total;
    return ST_OK;
}
static int check_rows(const Kv4 &k, int rows) {
    return rows > k.c.max_rows ? fail(ST_ERANGE, "%d rows, max_rows is %d", rows, k.c.max_rows) : ST_OK;
}
static int check_layers(const Kv4 &k, int lo, int hi) {
    return lo < 0 || hi > k.c.n_layers || lo > hi ? fail(ST_ERANGE, "layers [%d, %d) outside [0, %d)", lo, hi, k.c.n_layers) : ST_OK;
}
static int check_layer(const Kv4 &k, int layer) {
    return layer < 0 || layer >= k.c.n_layers ? fail(ST_ERANGE, "layer %d outside [0, %d)", layer, k.c.n_layers) : ST_OK;
}
static int check_ledger(const st_kv4_ledger *l, const char *name) {
    if (!l->weights || !l->positions) return fail(ST_EINVAL, "%s: weights or positions is NULL", name);
    if (((uintptr_t)l->weights | (uintptr_t)l->positions) & 3) return fail(ST_EINVAL, "%s is not aligned to 4 bytes", name);
    return ST_OK;
}
}  // namespace st

using namespace st;

extern "C" {

int st_kv4_query_sizes(const st_kv4_config *cfg, size_t *cache_bytes, size_t *workspace_bytes) {
    if (int rc = check_config(cfg)) return rc;
    Kv4 k;
    size_t cb, wb;
    carve(*cfg, nullptr, nullptr, &k, &cb, &wb);
    if (cache_bytes) *cache_bytes = cb;
    if (workspace_bytes) *workspace_bytes = wb;
    return ST_OK;
}

int st_kv4_create(const st_kv4_config *cfg, const float *rope, void *cache, size_t cache_bytes, void *workspace,
                  size_t workspace_bytes, void *stream, st_kv4 **out) {
    if (!out) return fail(ST_EINVAL, "out is NULL");
    *out = nullptr;
    if (int rc = check_config(cfg)) return rc;
    if (!rope || !cache || !workspace) return fail(ST_EINVAL, "rope, cache or workspace is NULL");
    if (((uintptr_t)cache | (uintptr_t)workspace) & 255) return fail(ST_EINVAL, "cache and workspace must be 256-byte aligned");
    if ((uintptr_t)rope & 15) return fail(ST_EINVAL, "rope is not aligned to 16 bytes");
    Kv4 *k = new (std::nothrow) Kv4();
    if (!k) return fail(ST_ENOMEM, "out of host memory");
    size_t cb, wb;
    carve(*cfg, (char *)cache, (char *)workspace, k, &cb, &wb);
    if (cache_bytes < cb || workspace_bytes < wb) {
        delete k;
        return cache_bytes < cb ? fail(ST_ENOMEM, "cache has %zu bytes, %zu needed", cache_bytes, cb)
                                : fail(ST_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, wb);
    }
    k->c = *cfg, k->rope = rope, k->stream = (hipStream_t)stream;
    *out = reinterpret_cast<st_kv4 *>(k);
    return ST_OK;
}

void st_kv4_destroy(st_kv4 *h) { delete reinterpret_cast<Kv4 *>(h); }

int st_kv4_append(st_kv4 *h, int32_t layer, const st_kv4_span *spans, int32_t n, const void *qkv, int64_t qkv_stride,
                  const void *q_norm, const void *k_norm, void *q_out, int64_t q_stride, const st_kv4_ledger *ledger) {
    const Kv4 *k = reinterpret_cast<const Kv4 *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    const int64_t d = k->c.head_dim;
    Kv4Table t;
    int rows;
    if (int rc = check_layer(*k, layer)) return rc;
    if (int rc = take_spans(*k, spans, n, true, &t, &rows)) return rc;
    if (int rc = check_rows(*k, rows)) return rc;
    if (int rc = check_matrix("qkv", qkv, qkv_stride, (k->c.n_q_heads + 2 * k->c.n_kv_heads) * d)) return rc;
    if (int rc = check_matrix("q_out", q_out, q_stride, k->c.n_q_heads * d)) return rc;
    if (int rc = check_apart("qkv", qkv, qkv_stride, (k->c.n_q_heads + 2 * k->c.n_kv_heads) * d, "q_out", q_out, q_stride, k->c.n_q_heads * d, rows)) return rc;
    if (!q_norm != !k_norm) return fail(ST_EINVAL, "q_norm and k_norm are given together or not at all");
    if (((uintptr_t)q_norm | (uintptr_t)k_norm) & 7) return fail(ST_EINVAL, "the norms are not aligned to 8 bytes");
    if (ledger)
        if (int rc = check_ledger(ledger, "ledger")) return rc;
    if (!rows) return ST_OK;
    const size_t base = (size_t)layer * k->c.n_seq * k->c.n_kv_heads * k->c.max_seq;
    launch_kv4_append(*k, layer, t, rows, (const bf16_t *)qkv, qkv_stride, (const bf16_t *)q_norm, (const bf16_t *)k_norm,
                      (bf16_t *)q_out, q_stride, ledger ? ledger->weights + base : nullptr,
                      ledger ? ledger->positions + base : nullptr);
    return launched("st_kv4_append", hipGetLastError());
}

int st_kv4_attend(st_kv4 *h, int32_t layer, const st_kv4_span *spans, int32_t n, const void *q, int64_t q_stride, void *out,
                  int64_t out_stride, const st_kv4_ledger *ledger) {
    const Kv4 *k = reinterpret_cast<const Kv4 *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    const int64_t width = (int64_t)k->c.n_q_heads * k->c.head_dim;
    Kv4Table t;
    int rows;
    if (int rc = check_layer(*k, layer)) return rc;
    if (int rc = take_spans(*k, spans, n, false, &t, &rows)) return rc;
    if (int rc = check_rows(*k, rows)) return rc;
    if (int rc = check_matrix("q", q, q_stride, width)) return rc;
    if (int rc = check_matrix("out", out, out_stride, width)) return rc;
    if (int rc = check_apart("q", q, q_stride, width, "out", out, out_stride, width, rows)) return rc;
    if (ledger)
        if (int rc = check_ledger(ledger, "ledger")) return rc;
    if (!rows) return ST_OK;
    const size_t base = (size_t)layer * k->c.n_seq * k->c.n_kv_heads * k->c.max_seq;
    if (int rc = launch_kv4_attend(*k, layer, t, (const bf16_t *)q, q_stride, (bf16_t *)out, out_stride,
                                   ledger ? ledger->weights + base : nullptr))
        return rc;
    return launched("st_kv4_attend", hipGetLastError());
}

int st_kv4_attend_plan(const st_kv4_config *cfg, const st_kv4_span *spans, int32_t n, int32_t with_ledger, int32_t *columns, int32_t *blocks,
                       int32_t *ranges) {
    if (int rc = check_config(cfg)) return rc;
    Kv4 k{};
    size_t cb, wb;
    Kv4Table t;
    int rows;
    k.c = *cfg;
    carve(*cfg, nullptr, nullptr, &k, &cb, &wb);
    if (int rc = take_spans(k, spans, n, false, &t, &rows)) return rc;
    if (int rc = check_rows(k, rows)) return rc;
    const Kv4AttendPlan p = plan_kv4_attend(k, t, with_ledger != 0);
    if (columns) *columns = rows ? p.cols : 0;
    if (blocks) *blocks = rows ? p.blocks : 0;
    for (int j = 0; ranges && j < n; ++j) ranges[j] = t.s[j].rows ? t.s[j].splits : 0;
    return ST_OK;
}

int st_kv4_evict(st_kv4 *h, int32_t layer_lo, int32_t layer_hi, const st_kv4_span *spans, int32_t n, int32_t keep,
                 int32_t recent, const st_kv4_ledger *ledger, const st_kv4_ledger *into) {
    const Kv4 *k = reinterpret_cast<const Kv4 *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    Kv4Table t;
    int rows;
    if (int rc = check_layers(*k, layer_lo, layer_hi)) return rc;
    if (int rc = take_spans(*k, spans, n, false, &t, &rows)) return rc;
    for (int j = 0; j < n; ++j)
        if (spans[j].rows) return fail(ST_EINVAL, "span %d: rows must be 0", j);
    if (keep <= 0 || recent < 0 || recent > keep) return fail(ST_EINVAL, "keep %d and recent %d: 0 <= recent <= keep, keep > 0", keep, recent);
    if (!ledger) return fail(ST_EINVAL, "ledger is NULL");
    if (int rc = check_ledger(ledger, "ledger")) return rc;
    if (!into) into = ledger;
    if (int rc = check_ledger(into, "into")) return rc;
    if ((into->weights == ledger->weights) != (into->positions == ledger->positions))
        return fail(ST_EINVAL, "into shares one array with ledger and not the other");
    const size_t bytes = 4 * (size_t)k->c.n_layers * k->c.n_seq * k->c.n_kv_heads * k->c.max_seq;
    auto overlap = [&](const void *a, const void *b) {
        const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
        return (x < y ? y - x : x - y) < bytes;
    };
    if (into->weights != ledger->weights &&
        (overlap(into->weights, ledger->weights) || overlap(into->positions, ledger->positions) || overlap(into->weights, ledger->positions) ||
         overlap(into->positions, ledger->weights) || overlap(into->weights, into->positions)))
        return fail(ST_EINVAL, "into and ledger overlap");
    if (!n || layer_lo == layer_hi) return ST_OK;
    return launched("st_kv4_evict", launch_kv4_evict(*k, layer_lo, layer_hi, t, keep, recent, ledger->weights, ledger->positions, into->weights, into->positions));
}

int st_kv4_read(st_kv4 *h, int32_t layer_lo, int32_t layer_hi, const st_kv4_span *spans, int32_t n, void *k_out, void *v_out) {
    const Kv4 *k = reinterpret_cast<const Kv4 *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    Kv4Table t;
    int rows;
    if (int rc = check_layers(*k, layer_lo, layer_hi)) return rc;
    if (int rc = take_spans(*k, spans, n, false, &t, &rows)) return rc;
    if (!k_out || !v_out) return fail(ST_EINVAL, "k_out or v_out is NULL");
    if (((uintptr_t)k_out | (uintptr_t)v_out) & 15) return fail(ST_EINVAL, "k_out or v_out is not aligned to 16 bytes");
    if (!rows || layer_lo == layer_hi) return ST_OK;
    launch_kv4_read(*k, layer_lo, layer_hi, t, rows, (bf16_t *)k_out, (bf16_t *)v_out);
    return launched("st_kv4_read", hipGetLastError());
}

}  // extern "C"
