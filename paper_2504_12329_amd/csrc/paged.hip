// A key/value cache in pages: the C entry points, and the kernels that write rows (append with the norms of queries and keys and the rotation) and
// move them (keep).
//
// A page holds page_size slots of every kv head, a head's slots one after the other, so that attention reads whole lines of 256 (128) bytes a slot and
// a run of 16 slots and more without a gap.  Which page a run is in is one 4-byte read per 16 slots.
#include <algorithm>
#include <cmath>
#include <new>

#include "checks.h"
#include "paged.h"
#include "st_device.h"

namespace st {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------
// Append.  D / 8 threads per head; a thread owns two groups of four neighbouring channels.  Where pairs are halves of the rotating part the groups lie half of
// it apart, else side by side, and either way the thread has its four pairs whole: pairs 4 l .. 4 l + 3 of the table.  Channels behind the rotating part
// are passed on.  The norm's sum is an exchange over the head's 8 or 16 lanes.
//
// Memory bounds it: every number is read and written once, 8 bytes an instruction and lane so that a thread has whole pairs of either order without exchanges.  4096
// rows of 40 / 8 heads of 128 with norms and rotation take 21.0 us, 119 MB at 5.7 TB/s (a copy of 2 GiB reaches 4.9; the rotation table comes from L2); a single row 2.1 us.
// ---------------------------------------------------------------------------------------
template <class T, int D, int CAP>
__global__ __launch_bounds__(256) void k_paged_append(const Kv4Spans<CAP> t, const PagedView view, const int32_t *__restrict__ depth,
                                                      const uint16_t *__restrict__ qkv, int64_t qkv_stride, const uint16_t *__restrict__ q_norm,
                                                      const uint16_t *__restrict__ k_norm, float eps, const float *__restrict__ rope, int rot, int halves,
                                                      int max_pos, uint16_t *__restrict__ q_out, int64_t q_stride) {
    constexpr int TPH = D / 8, HPB = 256 / TPH;
    const int nq = view.nq, nkv = view.nkv, row = blockIdx.x;
    const Kv4Span sp = t.s[kv4_span_of(t, row)];
    const int i = row - sp.row0, head = blockIdx.y * HPB + threadIdx.x / TPH, l = threadIdx.x % TPH;
    const int slot = sp.len + i;
    const int page = page_of(view.table + (int64_t)sp.seq * view.max_pages, view.n_pages, slot >> view.shift);
    const uint32_t pos = min((uint32_t)sp.pos + (uint32_t)(depth ? max(depth[row], 0) : i), (uint32_t)max_pos - 1u);
    if (head >= nq + 2 * nkv) return;
    const bool turns = head < nq + nkv && 8 * l < rot;
    const int at_a = turns && halves ? 4 * l : 8 * l, at_b = turns && halves ? rot / 2 + 4 * l : 8 * l + 4;
    const uint16_t *src = qkv + row * qkv_stride + head * D;
    const u32x2 wa = *reinterpret_cast<const u32x2 *>(src + at_a), wb = *reinterpret_cast<const u32x2 *>(src + at_b);
    u32x2 oa = wa, ob = wb;
    if (head < nq + nkv) {
        float a[4] = {T::lo(wa.x), T::hi(wa.x), T::lo(wa.y), T::hi(wa.y)};
        float b[4] = {T::lo(wb.x), T::hi(wb.x), T::lo(wb.y), T::hi(wb.y)};
        float4 t01 = make_float4(1.f, 0.f, 1.f, 0.f), t23 = t01;
        if (turns) {
            const float4 *at = reinterpret_cast<const float4 *>(rope + ((size_t)pos * (rot / 2) + 4 * l) * 2);
            t01 = at[0], t23 = at[1];
        }
        const uint16_t *norm = head < nq ? q_norm : k_norm;
        if (norm) {
            const u32x2 na = *reinterpret_cast<const u32x2 *>(norm + at_a), nb = *reinterpret_cast<const u32x2 *>(norm + at_b);
            const float ga[4] = {T::lo(na.x), T::hi(na.x), T::lo(na.y), T::hi(na.y)};
            const float gb[4] = {T::lo(nb.x), T::hi(nb.x), T::lo(nb.y), T::hi(nb.y)};
            float v = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v = fmaf(a[e], a[e], fmaf(b[e], b[e], v));
            v += dpp_move<0xB1, 0xf>(0.f, v);   // quad swaps, then the mirrors: over 8 lanes, over 16
            v += dpp_move<0x4E, 0xf>(0.f, v);
            v += dpp_move<0x141, 0xf>(0.f, v);
            if constexpr (D == 128) v += dpp_move<0x140, 0xf>(0.f, v);
            const float r = 1.0f / sqrtf(v / D + eps);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = a[e] * r * ga[e], b[e] = b[e] * r * gb[e];
        }
        const float cx[4] = {t01.x, t01.z, t23.x, t23.z}, sy[4] = {t01.y, t01.w, t23.y, t23.w};
        if (turns) {
            if (halves) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = a[e] * cx[e] - b[e] * sy[e];
                    b[e] = b[e] * cx[e] + a[e] * sy[e];
                    a[e] = x;
                }
            } else {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const float x = a[2 * p] * cx[p] - a[2 * p + 1] * sy[p], y = b[2 * p] * cx[2 + p] - b[2 * p + 1] * sy[2 + p];
                    a[2 * p + 1] = a[2 * p + 1] * cx[p] + a[2 * p] * sy[p], b[2 * p + 1] = b[2 * p + 1] * cx[2 + p] + b[2 * p] * sy[2 + p];
                    a[2 * p] = x, b[2 * p] = y;
                }
            }
        }
        if (turns || norm) oa = u32x2{T::pack(a[0], a[1]), T::pack(a[2], a[3])}, ob = u32x2{T::pack(b[0], b[1]), T::pack(b[2], b[3])};
    }
    uint16_t *dst;
    if (head < nq) {
        dst = q_out + row * q_stride + head * D;
    } else {
        if (page < 0) return;
        const bool is_k = head < nq + nkv;
        dst = (is_k ? view.k : view.v) + ((((size_t)page * nkv + (head - nq - (is_k ? 0 : nkv))) << view.shift) + (slot & ((1 << view.shift) - 1))) * D;
    }
    *reinterpret_cast<u32x2 *>(dst + at_a) = oa;
    *reinterpret_cast<u32x2 *>(dst + at_b) = ob;
}

// ---------------------------------------------------------------------------------------
// Keep.  A thread owns 16 bytes of a slot in one layer, plane and kv head, and moves them down the branch: every source lies behind its destination and behind all
// destinations before, so sources that are read before their batch's first write are as they were.  A chain of four dependent loads (count, path, table, row) and
// a batch of rows in flight: latency.  8 sequences of 21 rows in 64 layers of 8 heads of 128 take 7.2 us, one sequence in 28 layers of 2 heads 4.0 us.
// ---------------------------------------------------------------------------------------
constexpr int kKeepBatch = 8;

template <int CAP>
__global__ __launch_bounds__(256) void k_paged_keep(const Kv4Spans<CAP> t, PagedView view, size_t per_layer, int units, int D, const int32_t *__restrict__ path,
                                                    int path_stride, const int32_t *__restrict__ accepted) {
    const Kv4Span sp = t.s[blockIdx.y];
    const int u = blockIdx.x * 256 + threadIdx.x, per_head = D / 8, mask = (1 << view.shift) - 1;
    const int n = min(min(accepted[blockIdx.y], path_stride), sp.rows - 1);
    const int32_t *rows = path + (int64_t)blockIdx.y * path_stride, *pages = view.table + (int64_t)sp.seq * view.max_pages;
    if (u >= units) return;
    const bool is_k = u < units / 2;
    const int x = is_k ? u : u - units / 2, head = x / per_head;
    uint16_t *plane = (is_k ? view.k : view.v) + blockIdx.z * per_layer + (x % per_head) * 8;
    auto place = [&](int page, int slot) {
        return reinterpret_cast<u32x4 *>(plane + ((((size_t)page * view.nkv + head) << view.shift) + (slot & mask)) * D);
    };
    int before = 0;
    for (int i0 = 0; i0 < n; i0 += kKeepBatch) {
        // (all of a batch's numbers are asked for before any is looked at: rows past the end are read as the last, and their table entries as the first row's)
        int r[kKeepBatch], from[kKeepBatch], into[kKeepBatch];
#pragma unroll
        for (int e = 0; e < kKeepBatch; ++e) r[e] = rows[min(i0 + e, n - 1)];
        bool whole = true;
#pragma unroll
        for (int e = 0; e < kKeepBatch; ++e) {
            whole = whole && i0 + e < n && r[e] > before && r[e] < sp.rows;
            before = whole ? r[e] : before;
            r[e] = whole ? r[e] : 0;  // (0: nothing moves)
        }
#pragma unroll
        for (int e = 0; e < kKeepBatch; ++e) {
            from[e] = pages[(sp.len + r[e]) >> view.shift];
            into[e] = pages[(sp.len + (r[e] ? 1 + i0 + e : 0)) >> view.shift];
        }
        u32x4 v[kKeepBatch];
        bool moves[kKeepBatch];
#pragma unroll
        for (int e = 0; e < kKeepBatch; ++e) {
            moves[e] = r[e] > 1 + i0 + e && (uint32_t)from[e] < (uint32_t)view.n_pages && (uint32_t)into[e] < (uint32_t)view.n_pages;
            if (moves[e]) v[e] = *place(from[e], sp.len + r[e]);
        }
#pragma unroll
        for (int e = 0; e < kKeepBatch; ++e)
            if (moves[e]) *place(into[e], sp.len + 1 + i0 + e) = v[e];
        if (!whole) return;
    }
}

void launch_paged_append(const Paged &k, int layer, const Kv4Table &t, int rows, const int32_t *depth, const uint16_t *qkv, int64_t qkv_stride,
                         const uint16_t *q_norm, const uint16_t *k_norm, uint16_t *q_out, int64_t q_stride) {
    const int per_block = 256 / (k.c.head_dim / 8), heads = k.c.n_q_heads + 2 * k.c.n_kv_heads;
    const dim3 grid(rows, (heads + per_block - 1) / per_block);
    const bool f16 = k.c.dtype == ST_F16;
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        auto *kern = k.c.head_dim == 128 ? (f16 ? k_paged_append<Fp16, 128, CAP> : k_paged_append<Bf16, 128, CAP>)
                                         : (f16 ? k_paged_append<Fp16, 64, CAP> : k_paged_append<Bf16, 64, CAP>);
        for (int j = 0; j < tab.n; ++j) tab.s[j].blk0 = tab.s[j].row0;  // block = row
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, k.stream, tab, k.view(layer), depth, qkv, qkv_stride, q_norm, k_norm, k.c.rms_eps, k.rope,
                           k.c.rot_dim, (int)(k.c.rot_pairs == ST_PAIRS_HALVES), k.c.max_pos, q_out, q_stride);
    });
}

void launch_paged_keep(const Paged &k, int layer_lo, int layer_hi, const Kv4Table &t, const int32_t *path, int path_stride, const int32_t *accepted) {
    const int units = 2 * k.c.n_kv_heads * (k.c.head_dim / 8);
    const dim3 grid((units + 255) / 256, t.n, layer_hi - layer_lo);
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
        hipLaunchKernelGGL(k_paged_keep<CAP>, grid, dim3(256), 0, k.stream, tab, k.view(layer_lo), k.per_layer, units, k.c.head_dim, path, path_stride, accepted);
    });
}

// ---------------------------------------------------------------------------------------
// C entry points
// ---------------------------------------------------------------------------------------
static int check_config(const st_paged_config *c) {
    if (!c) return fail(ST_EINVAL, "config is NULL");
    if (c->n_layers <= 0 || c->n_seq <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_pages <= 0 || c->max_pages <= 0 || c->max_rows <= 0 ||
        c->max_pos <= 0)
        return fail(ST_EINVAL, "config has a non-positive dimension");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(ST_EINVAL, "head_dim must be 64 or 128");
    if (c->n_q_heads % c->n_kv_heads) return fail(ST_EINVAL, "n_q_heads must be a multiple of n_kv_heads");
    if (c->n_q_heads / c->n_kv_heads > 16) return fail(ST_EINVAL, "at most 16 query heads per kv head");
    if (c->n_q_heads > 4096) return fail(ST_EINVAL, "at most 4096 query heads");
    if (c->n_layers > 65535) return fail(ST_EINVAL, "at most 65535 layers");
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return fail(ST_EINVAL, "page_size must be a power of two from 16 to 1024");
    if ((int64_t)c->page_size * c->max_pages > 1 << 24 || c->max_rows > 1 << 20)
        return fail(ST_EINVAL, "page_size * max_pages must be <= 2^24 and max_rows <= 2^20");
    if (c->dtype != ST_BF16 && c->dtype != ST_F16) return fail(ST_EINVAL, "dtype must be ST_BF16 or ST_F16");
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 16) return fail(ST_EINVAL, "rot_dim must be a multiple of 16 up to head_dim");
    if (c->rot_pairs != ST_PAIRS_HALVES && c->rot_pairs != ST_PAIRS_NEIGHBOURS) return fail(ST_EINVAL, "bad rot_pairs");
    if (!(c->rms_eps >= 0.f) || std::isinf(c->rms_eps)) return fail(ST_EINVAL, "bad rms_eps");
    // 2^46 numbers are far more than any device has, and every size below then fits 64 bits
    if ((double)c->n_layers * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim > 0x1p46)
        return fail(ST_EINVAL, "the cache would be larger than 2^46 numbers");
    return ST_OK;
}

// The planes and the workspace; with cache / ws == nullptr the record only has sizes that matter.
static void carve(const st_paged_config &c, char *cache, char *ws, Paged *k, size_t *cache_bytes, size_t *ws_bytes) {
    k->c = c;
    k->shift = __builtin_ctz(c.page_size);
    k->per_layer = (size_t)c.n_pages * c.n_kv_heads * c.page_size * c.head_dim;
    k->plane[0] = reinterpret_cast<uint16_t *>(cache);
    k->plane[1] = cache ? k->plane[0] + c.n_layers * k->per_layer : nullptr;  // (a page is a multiple of 2 KB)
    *cache_bytes = 4 * k->per_layer * c.n_layers;
    // Where slots are cut into ranges, a range is at least the call's tiles, over all groups of columns, in kPagedBlocks parts: the ranges of the spans that
    // are cut are then at most twice that many blocks.  And a row has at most kPagedRanges of them.
    k->part_rows = std::min((size_t)c.max_rows * c.n_q_heads * kPagedRanges, (size_t)2 * kPagedBlocks * kPagedColumns);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? ws + off : nullptr;
        off += up256(bytes);
        return reinterpret_cast<float *>(p);
    };
    k->part_ml = take(sizeof(float) * 2 * k->part_rows);
    k->part_o = take(sizeof(float) * k->part_rows * c.head_dim);
    *ws_bytes = off;
}

// Checks the spans and deals the rows to them.  With `positions` theirs must lie in the rotation table: all rows', or with `depth` those of rows of depth 0.
static int take_spans(const Paged &k, const st_kv4_span *spans, int32_t n, bool positions, bool depth, Kv4Table *t, int *rows) {
    const st_paged_config &c = k.c;
    const int64_t capacity = (int64_t)c.page_size * c.max_pages;
    if (n < 0 || n > ST_KV4_MAX_SPANS) return fail(ST_EINVAL, "%d spans, 0 to %d are supported", n, ST_KV4_MAX_SPANS);
    if (n && !spans) return fail(ST_EINVAL, "spans is NULL");
    int64_t total = 0;
    for (int j = 0; j < n; ++j) {
        const st_kv4_span &s = spans[j];
        if (s.seq < 0 || s.seq >= c.n_seq) return fail(ST_ERANGE, "span %d: sequence %d outside [0, %d)", j, s.seq, c.n_seq);
        if (s.len < 0 || s.rows < 0 || (int64_t)s.len + s.rows > capacity)
            return fail(ST_ERANGE, "span %d: %d slots + %d rows, the table holds %lld", j, s.len, s.rows, (long long)capacity);
        if (s.pos < 0 || (positions && (int64_t)s.pos + (depth ? s.rows > 0 : s.rows) > c.max_pos))
            return fail(ST_ERANGE, "span %d: positions from %d, %d rows, table of %d", j, s.pos, s.rows, c.max_pos);
        for (int i = 0; i < j; ++i)
            if (spans[i].seq == s.seq) return fail(ST_EINVAL, "spans %d and %d are both sequence %d", i, j, s.seq);
        t->s[j] = Kv4Span{s.seq, s.len, s.pos, s.rows, (int32_t)total, 0, 1, 0, 0};
        total += s.rows;
        if (total > c.max_rows) return fail(ST_ERANGE, "%lld rows or more, max_rows is %d", (long long)total, c.max_rows);
    }
    t->n = n;
    *rows = (int)total;
    return ST_OK;
}
static int check_layer(const Paged &k, int layer) {
    return layer < 0 || layer >= k.c.n_layers ? fail(ST_ERANGE, "layer %d outside [0, %d)", layer, k.c.n_layers) : ST_OK;
}

}  // namespace st

using namespace st;

extern "C" {

int st_paged_query_sizes(const st_paged_config *cfg, size_t *cache_bytes, size_t *workspace_bytes) {
    if (int rc = check_config(cfg)) return rc;
    Paged k;
    size_t cb, wb;
    carve(*cfg, nullptr, nullptr, &k, &cb, &wb);
    if (cache_bytes) *cache_bytes = cb;
    if (workspace_bytes) *workspace_bytes = wb;
    return ST_OK;
}

int st_paged_create(const st_paged_config *cfg, const float *rope, const int32_t *table, void *cache, size_t cache_bytes, void *workspace,
                    size_t workspace_bytes, void *stream, st_paged **out) {
    if (!out) return fail(ST_EINVAL, "out is NULL");
    *out = nullptr;
    if (int rc = check_config(cfg)) return rc;
    if ((!rope && cfg->rot_dim) || !table || !cache || !workspace) return fail(ST_EINVAL, "rope, table, cache or workspace is NULL");
    if (((uintptr_t)cache | (uintptr_t)workspace) & 255) return fail(ST_EINVAL, "cache and workspace must be 256-byte aligned");
    if ((uintptr_t)rope & 15) return fail(ST_EINVAL, "rope is not aligned to 16 bytes");
    if ((uintptr_t)table & 3) return fail(ST_EINVAL, "table is not aligned to 4 bytes");
    Paged *k = new (std::nothrow) Paged();
    if (!k) return fail(ST_ENOMEM, "out of host memory");
    size_t cb, wb;
    carve(*cfg, (char *)cache, (char *)workspace, k, &cb, &wb);
    if (cache_bytes < cb || workspace_bytes < wb) {
        delete k;
        return cache_bytes < cb ? fail(ST_ENOMEM, "cache has %zu bytes, %zu needed", cache_bytes, cb)
                                : fail(ST_ENOMEM, "workspace has %zu bytes, %zu needed", workspace_bytes, wb);
    }
    k->rope = rope, k->table = table, k->stream = (hipStream_t)stream;
    *out = reinterpret_cast<st_paged *>(k);
    return ST_OK;
}

void st_paged_destroy(st_paged *h) { delete reinterpret_cast<Paged *>(h); }

int st_paged_append(st_paged *h, int32_t layer, const st_kv4_span *spans, int32_t n, const st_draft_tree *tree, const void *qkv, int64_t qkv_stride,
                    const void *q_norm, const void *k_norm, void *q_out, int64_t q_stride) {
    const Paged *k = reinterpret_cast<const Paged *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    const int64_t d = k->c.head_dim, width = (k->c.n_q_heads + 2 * (int64_t)k->c.n_kv_heads) * d;
    Kv4Table t;
    int rows;
    if (int rc = check_layer(*k, layer)) return rc;
    if (int rc = take_spans(*k, spans, n, true, tree != nullptr, &t, &rows)) return rc;
    if (tree && !tree->depth) return fail(ST_EINVAL, "tree: depth is NULL");
    if (tree && (uintptr_t)tree->depth & 3) return fail(ST_EINVAL, "tree: depth is not aligned to 4 bytes");
    if (int rc = check_matrix("qkv", qkv, qkv_stride, width)) return rc;
    if (int rc = check_matrix("q_out", q_out, q_stride, k->c.n_q_heads * d)) return rc;
    if (int rc = check_apart("qkv", qkv, qkv_stride, width, "q_out", q_out, q_stride, k->c.n_q_heads * d, rows)) return rc;
    if (!q_norm != !k_norm) return fail(ST_EINVAL, "q_norm and k_norm are given together or not at all");
    if (((uintptr_t)q_norm | (uintptr_t)k_norm) & 7) return fail(ST_EINVAL, "the norms are not aligned to 8 bytes");
    if (!rows) return ST_OK;
    launch_paged_append(*k, layer, t, rows, tree ? tree->depth : nullptr, (const uint16_t *)qkv, qkv_stride, (const uint16_t *)q_norm,
                        (const uint16_t *)k_norm, (uint16_t *)q_out, q_stride);
    return launched("st_paged_append", hipGetLastError());
}

static int check_sees(const st_draft_tree *tree, const st_kv4_span *spans, int n) {
    if (!tree->sees) return fail(ST_EINVAL, "tree: sees is NULL");
    if ((uintptr_t)tree->sees & 7) return fail(ST_EINVAL, "tree: sees is not aligned to 8 bytes");
    if (tree->words < 1 || tree->words > kTreeWords) return fail(ST_EINVAL, "tree: %d words, 1 to %d are supported", tree->words, kTreeWords);
    for (int j = 0; j < n; ++j)
        if (spans[j].rows > 64 * tree->words) return fail(ST_ERANGE, "span %d: %d rows, sees has bits for %d", j, spans[j].rows, 64 * tree->words);
    return ST_OK;
}

int st_paged_attend(st_paged *h, int32_t layer, const st_kv4_span *spans, int32_t n, const st_draft_tree *tree, const void *q, int64_t q_stride,
                    void *out, int64_t out_stride) {
    const Paged *k = reinterpret_cast<const Paged *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    const int64_t width = (int64_t)k->c.n_q_heads * k->c.head_dim;
    Kv4Table t;
    int rows;
    if (int rc = check_layer(*k, layer)) return rc;
    if (int rc = take_spans(*k, spans, n, false, false, &t, &rows)) return rc;
    if (tree)
        if (int rc = check_sees(tree, spans, n)) return rc;
    if (int rc = check_matrix("q", q, q_stride, width)) return rc;
    if (int rc = check_matrix("out", out, out_stride, width)) return rc;
    if (int rc = check_apart("q", q, q_stride, width, "out", out, out_stride, width, rows)) return rc;
    if (!rows) return ST_OK;
    return launch_paged_attend(*k, layer, t, tree ? tree->sees : nullptr, tree ? tree->words : 0, (const uint16_t *)q, q_stride, (uint16_t *)out, out_stride);
}

int st_paged_attend_plan(const st_paged_config *cfg, const st_kv4_span *spans, int32_t n, int32_t with_tree, int32_t *columns, int32_t *blocks,
                         int32_t *ranges) {
    if (int rc = check_config(cfg)) return rc;
    Paged k{};
    size_t cb, wb;
    Kv4Table t;
    int rows;
    carve(*cfg, nullptr, nullptr, &k, &cb, &wb);
    if (int rc = take_spans(k, spans, n, false, false, &t, &rows)) return rc;
    for (int j = 0; with_tree && j < n; ++j)
        if (spans[j].rows > 64 * kTreeWords) return fail(ST_ERANGE, "span %d: %d rows, trees have at most %d", j, spans[j].rows, 64 * kTreeWords);
    const PagedAttendPlan p = plan_paged_attend(k, t);
    if (columns) *columns = rows ? p.cols : 0;
    if (blocks) *blocks = rows ? (int32_t)std::min<int64_t>(p.blocks, INT32_MAX) : 0;
    for (int j = 0; ranges && j < n; ++j) ranges[j] = t.s[j].rows ? t.s[j].splits : 0;
    return ST_OK;
}

int st_paged_keep(st_paged *h, int32_t layer_lo, int32_t layer_hi, const st_kv4_span *spans, int32_t n, const int32_t *path, int32_t path_stride,
                  const int32_t *accepted) {
    const Paged *k = reinterpret_cast<const Paged *>(h);
    if (!k) return fail(ST_EINVAL, "cache is NULL");
    Kv4Table t;
    int rows;
    if (layer_lo < 0 || layer_hi > k->c.n_layers || layer_lo > layer_hi)
        return fail(ST_ERANGE, "layers [%d, %d) outside [0, %d)", layer_lo, layer_hi, k->c.n_layers);
    if (int rc = take_spans(*k, spans, n, false, false, &t, &rows)) return rc;
    if (!path || !accepted) return fail(ST_EINVAL, "path or accepted is NULL");
    if (((uintptr_t)path | (uintptr_t)accepted) & 3) return fail(ST_EINVAL, "path or accepted is not aligned to 4 bytes");
    if (path_stride < 0) return fail(ST_EINVAL, "path_stride is negative");
    if (!rows || !path_stride || layer_lo == layer_hi) return ST_OK;
    launch_paged_keep(*k, layer_lo, layer_hi, t, path, path_stride, accepted);
    return launched("st_paged_keep", hipGetLastError());
}

}  // extern "C"
