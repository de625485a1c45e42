// Host-side internals of the key/value cache in pages (paged.hip, paged_attend.hip): its record, what the kernels take of it and the launchers.
// The span table is that of the 4-bit cache.  Nothing here is part of the public ABI.
#pragma once

#include "kv4.h"

namespace st {

// Attention: blocks that a call is cut into where it has the slots for them, and most key ranges of a span (a lane each in the join)
constexpr int kPagedBlocks = 512, kPagedRanges = 64, kPagedColumns = 128;
constexpr int kTreeWords = 16;  // most words of a row's bits

// One layer of the cache, and where its sequences' pages are
struct PagedView {
    uint16_t *k, *v;       // [page][kv head][slot of the page][head_dim]
    const int32_t *table;  // [sequence][max_pages]
    int32_t nq, nkv, n_pages, max_pages, shift;  // page_size = 1 << shift
};

struct Paged {
    st_paged_config c;
    uint16_t *plane[2];     // K, V
    size_t per_layer;       // numbers of a layer in each
    const int32_t *table;
    const float *rope;
    float *part_ml, *part_o;  // partial results of the key ranges: (max, sum) and outputs
    size_t part_rows;         // rows they hold
    int32_t shift;
    hipStream_t stream;
    PagedView view(int layer) const {
        return PagedView{plane[0] + layer * per_layer, plane[1] + layer * per_layer, table, c.n_q_heads, c.n_kv_heads, c.n_pages, c.max_pages, shift};
    }
};

struct PagedAttendPlan {
    int cols;        // columns of a block: 16 or 32 (k_paged_few), 128 (k_paged_chunk)
    int64_t blocks;
    int join;        // rows of the longest span in several ranges, 0 without one
};
// Fills in blk0, splits, per and part0 of the spans
PagedAttendPlan plan_paged_attend(const Paged &k, Kv4Table &t);

// All enqueue only; the arguments have been checked.
void launch_paged_append(const Paged &k, int layer, const Kv4Table &t, int rows, const int32_t *depth, const uint16_t *qkv, int64_t qkv_stride,
                         const uint16_t *q_norm, const uint16_t *k_norm, uint16_t *q_out, int64_t q_stride);
int launch_paged_attend(const Paged &k, int layer, Kv4Table &t, const uint64_t *sees, int words, const uint16_t *q, int64_t q_stride, uint16_t *out,
                        int64_t out_stride);  // ST_ERANGE, and nothing launched, where no grid holds the blocks
void launch_paged_keep(const Paged &k, int layer_lo, int layer_hi, const Kv4Table &t, const int32_t *path, int path_stride, const int32_t *accepted);

#ifdef __HIPCC__
// The two 16-bit types as the kernels see them: eight numbers as a matrix operand, two fp32 rounded to nearest, and the halves of a word
typedef __bf16 paged_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 paged_f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 paged_f16x2 __attribute__((ext_vector_type(2)));
typedef float paged_f32x2 __attribute__((ext_vector_type(2)));
typedef float paged_f32x4 __attribute__((ext_vector_type(4)));
typedef float paged_f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t paged_u32x4 __attribute__((ext_vector_type(4)));
struct Bf16 {
    typedef paged_bf16x8 vec8;
    static constexpr uint32_t kExponent = 0x7f807f80u, kLowBit = 0x00800080u;  // of both halves
    static constexpr float kRaise = 0.f;
    static __device__ __forceinline__ paged_f32x4 mfma16(vec8 a, vec8 b, paged_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ paged_f32x16 mfma32(vec8 a, vec8 b, paged_f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        typedef __bf16 pair __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(paged_f32x2{lo, hi}, pair));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
};
struct Fp16 {
    typedef paged_f16x8 vec8;
    static constexpr uint32_t kExponent = 0x7c007c00u, kLowBit = 0x04000400u;
    // A column's softmax weights, and their sum, are 2^15 times as large: with the largest at 1 those below 2^-14 would lose bits of the type and those below 2^-25 be 0, while the
    // sum in 32 bits has them.  Under one slot 17.5 above 450 equal ones the output was 0 instead of 1e-5 of their values.
    static constexpr float kRaise = 15.f;
    static __device__ __forceinline__ paged_f32x4 mfma16(vec8 a, vec8 b, paged_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ paged_f32x16 mfma32(vec8 a, vec8 b, paged_f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(paged_f32x2{lo, hi}, paged_f16x2));
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(paged_f16x2, w).x; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(paged_f16x2, w).y; }
};
// Sign bits of the halves of w that are infinite or NaN: an exponent of all ones is the one that a 1 carries into the sign's place
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    return ((w & T::kExponent) + T::kLowBit) & 0x80008000u;
}
__device__ __forceinline__ uint32_t halves_of(uint32_t signs) { return (signs >> 15) * 0xffffu; }  // all bits of the halves marked

// Page of a sequence's slot, -1 for a hole
__device__ __forceinline__ int page_of(const int32_t *pages, int n_pages, int index) {
    const int p = pages[index];
    return (uint32_t)p < (uint32_t)n_pages ? p : -1;
}
#endif

}  // namespace st
