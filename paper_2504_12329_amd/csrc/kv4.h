// Host-side internals of the 4-bit key/value cache (kv4.hip, kv4_attend.hip, kv4_evict.hip): its record, the span table that
// the kernels take by value and the launchers the API layer calls.  Nothing here is part of the public ABI.
#pragma once

#include "st_internal.h"

namespace st {

// One sequence's part of a call, with what the launch gives it.
struct Kv4Span {
    int32_t seq, len, pos, rows;  // st_kv4_span
    int32_t row0;                 // its first row among the call's rows
    int32_t blk0;                 // its first block in the launch
    int32_t splits;               // key ranges its blocks are dealt to
    int32_t per;                  // tiles of slots in a range
    int32_t part0;                // its first row of partial results (rows x query heads of range 0, of range 1, ...)
};
// Passed to the kernels by value: no copy to the device precedes them, and a captured launch keeps it.  Three sizes: an append of
// 64 spans costs the host 4.3 us, one of up to four 3.5 (the C call through ctypes).
template <int CAP>
struct Kv4Spans {
    int32_t n;
    Kv4Span s[CAP];
};
constexpr int kKv4Few = 4, kKv4Some = 16;
typedef Kv4Spans<ST_KV4_MAX_SPANS> Kv4Table;
static_assert(sizeof(Kv4Table) <= 2400, "kernel arguments are at most 4 KB");
// f(the table in the smallest size that holds it)
template <int CAP, class F>
inline void with_table_of(const Kv4Table &t, F f) {
    Kv4Spans<CAP> small;
    small.n = t.n;
    for (int j = 0; j < CAP; ++j) small.s[j] = j < t.n ? t.s[j] : Kv4Span{};
    f(small);
}
template <class F>
inline void with_table(const Kv4Table &t, F f) {
    if (t.n <= kKv4Few) with_table_of<kKv4Few>(t, f);
    else if (t.n <= kKv4Some) with_table_of<kKv4Some>(t, f);
    else f(t);
}

// Attention: most columns (rows x query heads of a kv head) of a block, most key ranges, most blocks where key ranges are cut
constexpr int kKv4Columns = 128, kKv4Ranges = 64, kKv4Blocks = 512;

// The planes of one layer and its heads
struct Kv4View {
    uint8_t *k, *v, *ks, *vs;  // [sequence][kv head][slot][head_dim / 2 | head_dim / 32]
    int32_t nq, nkv, max_seq;
};

struct Kv4 {
    st_kv4_config c;
    uint8_t *plane[4];       // K codes, V codes, K scales, V scales, [layer][sequence][kv head][slot][...]
    size_t per_layer[4];     // bytes of a layer in each
    const float *rope;       // [max_pos][head_dim / 2][2]
    float *lse;              // [max_rows][n_q_heads] log2 of each row's softmax sum
    float *part_ml, *part_o; // partial results of the key ranges: (max, sum) and outputs (and behind those, scores)
    size_t part_rows;        // rows they hold
    size_t part_floats;      // in part_o
    uint64_t *kept;          // evict: a bit per slot, [layer][span][kv head][kept_words]
    size_t kept_words;
    hipStream_t stream;
    Kv4View view(int layer) const {
        return Kv4View{plane[0] + layer * per_layer[0], plane[1] + layer * per_layer[1], plane[2] + layer * per_layer[2],
                       plane[3] + layer * per_layer[3], c.n_q_heads, c.n_kv_heads, c.max_seq};
    }
};

// How attention deals out a call.  Fills in blk0, splits, per and part0 of the spans.
struct Kv4AttendPlan {
    int cols;      // columns of a block: 16 or 32 (k_kv4_few), 128 (k_kv4_chunk)
    int blocks;
    int join;      // rows of the longest span in several ranges, 0 without one
    int64_t most;  // columns of a kv head in the span with most rows
    bool fused;    // the ranges are joined by the kernel that sums up the weights
    int64_t score_at, score_stride;  // where in part_o the scores are kept, [row][query head][stride]; stride 0: they are not
};
Kv4AttendPlan plan_kv4_attend(const Kv4 &k, Kv4Table &t, bool weights);

// All enqueue only; the arguments have been checked.  `t` holds spans and row0; the launchers fill in the rest.
void launch_kv4_append(const Kv4 &k, int layer, const Kv4Table &t, int rows, const bf16_t *qkv, int64_t qkv_stride,
                       const bf16_t *q_norm, const bf16_t *k_norm, bf16_t *q_out, int64_t q_stride, float *weights,
                       int32_t *positions);
void launch_kv4_read(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int rows, bf16_t *k_out, bf16_t *v_out);
int launch_kv4_attend(const Kv4 &k, int layer, Kv4Table &t, const bf16_t *q, int64_t q_stride, bf16_t *out, int64_t out_stride,
                      float *weights);  // ST_ERANGE, and nothing launched, where no grid holds the weights' blocks
hipError_t launch_kv4_evict(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int keep, int recent, const float *w_in,
                            const int32_t *p_in, float *w_out, int32_t *p_out);  // with the error that its launches ended in

#ifdef __HIPCC__
// The span whose blocks block `b` belongs to: the last one that starts at or before it (spans without blocks share their start
// with the next one).  Wave-uniform; all lanes must be active.
template <int CAP>
__device__ __forceinline__ int kv4_span_of(const Kv4Spans<CAP> &t, int b) {
    if constexpr (CAP == kKv4Few) {
        int j = 0;
#pragma unroll
        for (int i = 1; i < CAP; ++i) j = i < t.n && t.s[i].blk0 <= b ? i : j;
        return j;
    }
    const int lane = threadIdx.x & 63;
    const bool at_or_before = lane < t.n && t.s[lane].blk0 <= b;
    return __builtin_amdgcn_readfirstlane(63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(at_or_before)));
}
constexpr int kKv4Nan = 255;  // scale byte of a group that held an infinity or a NaN
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// two codes (byte `B` of w: low nibble, high nibble) as two bf16
template <int B>
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
#endif

}  // namespace st
