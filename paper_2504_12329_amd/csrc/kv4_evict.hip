// Eviction from the 4-bit key/value cache by accumulated attention weight.
//
// Of a head's `len` slots `keep` stay: those of the last `recent` positions, then those of the largest weight, ties to the
// lowest position.  Attention does not depend on the order of slots, so nothing is compacted: the slots below `keep` that
// are freed take, in ascending order, the slots at or above it that stay, in ascending order.  A context brought back
// from keep + m to keep slots moves at most m of them, in place, and no slot is both read and written.
//
//   k_kv4_select  one block per head: the keep-th largest weight by three digits of 11 bits (histograms in LDS), among ties the positions
//                 likewise; writes a bit per slot.  Bound by latency: a few passes over 8 bytes per slot, which after the first come from L2.
//   k_kv4_move    several blocks per head: finds the i-th freed slot and the i-th late one in the bits and copies.
#include "kv4.h"
#include "st_device.h"

namespace st {

constexpr int kSelThreads = 1024, kBins = 2048, kCopies = 4;

// Order-preserving image of a weight: NaN below everything, -0 as 0
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t b = __float_as_uint(w + 0.0f);
    return w != w ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ int wave_sum_int(int v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// In the histogram's order (from the top bin down if TOP, else from bin 0 up) the bin that the `rank`-th entry (1-based) lies in, and the
// entries before that bin.  All kSelThreads threads; hist holds kCopies partial histograms; res is two ints of LDS.  Ends with a barrier.
template <bool TOP>
__device__ __forceinline__ void find_bin(const int *hist, int *wsum, int *res, int rank, int &bin, int &before) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int c[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int b = TOP ? kBins - 1 - (2 * tid + e) : 2 * tid + e;
        c[e] = 0;
#pragma unroll
        for (int v = 0; v < kCopies; ++v) c[e] += hist[v * kBins + b];
    }
    int run = c[0] + c[1];  // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(run, o, kWave);
        if (lane >= o) run += x;
    }
    if (lane == 63) wsum[wave] = run;
    __syncthreads();
    int base = run - c[0] - c[1];
    for (int v = 0; v < wave; ++v) base += wsum[v];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (base < rank && rank <= base + c[e]) res[0] = TOP ? kBins - 1 - (2 * tid + e) : 2 * tid + e, res[1] = base;
        base += c[e];
    }
    __syncthreads();
    bin = res[0], before = res[1];
    __syncthreads();
}

__global__ __launch_bounds__(kSelThreads) void k_kv4_select(const Kv4Table t, int nkv, int max_seq, size_t layer_slots, int keep,
                                                            int recent, const float *__restrict__ w_in,
                                                            const int32_t *__restrict__ p_in, float *__restrict__ w_out,
                                                            int32_t *__restrict__ p_out, uint64_t *__restrict__ kept,
                                                            size_t kept_words) {
    __shared__ int hist[kCopies * kBins], wsum[16], res[2];
    const Kv4Span sp = t.s[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = sp.len;
    const size_t at = blockIdx.z * layer_slots + ((size_t)sp.seq * nkv + blockIdx.x) * max_seq;
    const float *w = w_in + at;
    const int32_t *p = p_in + at;
    const bool copy = w_out != w_in;
    if (n <= keep) {
        if (copy)
            for (int i = tid; i < n; i += kSelThreads) w_out[at + i] = w[i], p_out[at + i] = p[i];
        return;
    }
    const int fixed_from = sp.pos - recent;  // positions from here on stay
    auto key_of = [&](int i) { return p[i] >= fixed_from ? 0xffffffffu : weight_key(w[i]); };
    auto clear = [&]() {
        for (int i = tid; i < kCopies * kBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
    };
    int *mine = hist + (wave % kCopies) * kBins;

    // how many stay without being asked
    int fixed = 0;
    for (int i = tid; i < n; i += kSelThreads) fixed += p[i] >= fixed_from;
    fixed = wave_sum_int(fixed);
    if (lane == 0) wsum[wave] = fixed;
    __syncthreads();
    fixed = 0;
    for (int v = 0; v < kSelThreads / 64; ++v) fixed += wsum[v];
    __syncthreads();

    // threshold: entries above it stay, `need` of those equal to it
    uint32_t threshold = 0xffffffffu;
    int need = keep;
    if (fixed < keep) {
        need = keep - fixed;
        uint32_t prefix = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
            const int shift = kShift[pass], mask = (1 << kWidth[pass]) - 1, above = shift + kWidth[pass];
            clear();
            for (int i = tid; i < n; i += kSelThreads) {
                const uint32_t k = key_of(i);
                if (k != 0xffffffffu && (pass == 0 || k >> (above & 31) == prefix)) atomicAdd(&mine[k >> shift & mask], 1);
            }
            __syncthreads();
            int bin, before;
            find_bin<true>(hist, wsum, res, need, bin, before);
            need -= before;
            prefix = prefix << kWidth[pass] | bin;
        }
        threshold = prefix;
    }
    // among the ties: the `need` lowest positions (and, should positions repeat, the lowest slots)
    uint32_t at_most = 0;
    int ties = need;
    {
        uint32_t prefix = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
            const int shift = kShift[pass], mask = (1 << kWidth[pass]) - 1, above = shift + kWidth[pass];
            clear();
            for (int i = tid; i < n; i += kSelThreads) {
                const uint32_t x = (uint32_t)p[i] ^ 0x80000000u;
                if (key_of(i) == threshold && (pass == 0 || x >> (above & 31) == prefix)) atomicAdd(&mine[x >> shift & mask], 1);
            }
            __syncthreads();
            int bin, before;
            find_bin<false>(hist, wsum, res, ties, bin, before);
            ties -= before;
            prefix = prefix << kWidth[pass] | bin;
        }
        at_most = prefix;
    }
    // `ties` of the slots with this weight and this position stay: the first ones
    uint64_t *bits = kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * nkv + blockIdx.x) * kept_words;
    int done = 0;  // of them, in the slots before
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {
        const int i = i0 + tid;
        bool stays = false, tie = false;
        float wi = 0.f;
        int pi = 0;
        if (i < n) {
            wi = w[i], pi = p[i];
            const uint32_t k = pi >= fixed_from ? 0xffffffffu : weight_key(wi), x = (uint32_t)pi ^ 0x80000000u;
            stays = k > threshold || (k == threshold && x < at_most);
            tie = k == threshold && x == at_most;
        }
        const uint64_t tied = __builtin_amdgcn_ballot_w64(tie);
        if (lane == 0) wsum[wave] = __popcll(tied);
        __syncthreads();
        int before = done;
        for (int v = 0; v < kSelThreads / 64; ++v) {
            if (v < wave) before += wsum[v];
            done += wsum[v];
        }
        if (tie) stays = before + __popcll(tied & ((1ull << lane) - 1)) < ties;
        const uint64_t word = __builtin_amdgcn_ballot_w64(stays);
        if (lane == 0 && i < n) bits[i >> 6] = word;
        if (copy && stays && i < keep) w_out[at + i] = wi, p_out[at + i] = pi;
        __syncthreads();
    }
}

// The r-th (0-based) set bit of x
__device__ __forceinline__ int nth_bit(uint64_t x, int r) {
    int at = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1) {
        const int c = __popcll(x & (((uint64_t)1 << step) - 1));
        if (r >= c) r -= c, x >>= step, at += step;
    }
    return at;
}

constexpr int kMoveThreads = 256;

template <int D>
__global__ __launch_bounds__(kMoveThreads) void k_kv4_move(const Kv4Table t, Kv4View view, size_t k_layer, size_t s_layer,
                                                           size_t layer_slots, int keep, const float *__restrict__ w_in,
                                                           const int32_t *__restrict__ p_in, float *__restrict__ w_out,
                                                           int32_t *__restrict__ p_out, const uint64_t *__restrict__ kept,
                                                           size_t kept_words, int parts) {
    constexpr int CB = D / 2, SB = D / 32, TPM = CB / 16 * 2;  // threads per slot: 16 bytes of keys or values each
    __shared__ int wave_n[kMoveThreads / 64], freed[kMoveThreads], late[kMoveThreads];
    const Kv4Span sp = t.s[blockIdx.y];
    const int n = sp.len, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (n <= keep) return;
    const int kvh = blockIdx.x / parts, part = blockIdx.x % parts;
    const uint64_t *bits = kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * view.nkv + kvh) * kept_words;
    const size_t head = ((size_t)sp.seq * view.nkv + kvh) * view.max_seq, lat = blockIdx.z * layer_slots + head;
    const int words = (n + 63) / 64;
    // bits of word i that count: freed slots below keep, or late ones from keep on
    auto word_of = [&](int i, bool want_late) -> uint64_t {
        if (i >= words) return 0;
        const int s0 = i * 64;
        uint64_t held = n - s0 >= 64 ? ~0ull : (1ull << (n - s0)) - 1, front = s0 >= keep ? 0 : keep - s0 >= 64 ? ~0ull : (1ull << (keep - s0)) - 1;
        return want_late ? bits[i] & held & ~front : ~bits[i] & held & front;
    };
    // Moves r = part * kMoveThreads + k * parts * kMoveThreads ..: the r-th freed slot takes the r-th late one.  A block
    // walks both lists' words once for each of its groups of kMoveThreads moves.
    for (int r0 = part * kMoveThreads;; r0 += parts * kMoveThreads) {
        int total = 0;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const bool want_late = which == 1;
            int *list = want_late ? late : freed;
            const int from = want_late ? keep / 64 : 0, to = want_late ? words : (keep + 63) / 64;
            int base = 0;  // entries in the words before
            for (int i0 = from; i0 < to; i0 += kMoveThreads) {
                const uint64_t x = i0 + tid < to ? word_of(i0 + tid, want_late) : 0;
                const int c = __popcll(x);
                int run = c;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int y = __shfl_up(run, o, kWave);
                    if (lane >= o) run += y;
                }
                __syncthreads();
                if (lane == 63) wave_n[wave] = run;
                __syncthreads();
                int first = base + run - c;
                for (int v = 0; v < kMoveThreads / 64; ++v) {
                    if (v < wave) first += wave_n[v];
                    base += wave_n[v];
                }
                for (int b = max(0, r0 - first); b < c && first + b < r0 + kMoveThreads; ++b) list[first + b - r0] = (i0 + tid) * 64 + nth_bit(x, b);
            }
            total = base;
        }
        __syncthreads();
        const int m = min(total - r0, kMoveThreads);
        for (int u = tid; u < m * TPM; u += kMoveThreads) {
            const int src = late[u / TPM], dst = freed[u / TPM], e = u % TPM;
            uint8_t *codes = (e < TPM / 2 ? view.k : view.v) + blockIdx.z * k_layer + head * CB + e % (TPM / 2) * 16;
            const u32x4 x = *reinterpret_cast<const u32x4 *>(codes + (size_t)src * CB);
            *reinterpret_cast<u32x4 *>(codes + (size_t)dst * CB) = x;
            if (e < 2) {  // the scales
                uint8_t *s = (e ? view.vs : view.ks) + blockIdx.z * s_layer + head * SB;
                if constexpr (SB == 4) reinterpret_cast<uint32_t *>(s)[dst] = reinterpret_cast<const uint32_t *>(s)[src];
                else reinterpret_cast<uint16_t *>(s)[dst] = reinterpret_cast<const uint16_t *>(s)[src];
            } else if (e == 2) {
                w_out[lat + dst] = w_in[lat + src];
            } else if (e == 3) {
                p_out[lat + dst] = p_in[lat + src];
            }
        }
        if (r0 + parts * kMoveThreads >= total) return;
        __syncthreads();
    }
}

void launch_kv4_evict(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int keep, int recent, const float *w_in,
                      const int32_t *p_in, float *w_out, int32_t *p_out) {
    const int nkv = k.c.n_kv_heads, layers = layer_hi - layer_lo;
    const size_t slots = (size_t)k.c.n_seq * nkv * k.c.max_seq, off = slots * layer_lo;
    hipLaunchKernelGGL(k_kv4_select, dim3(nkv, t.n, layers), dim3(kSelThreads), 0, k.stream, t, nkv, k.c.max_seq, slots, keep, recent,
                       w_in + off, p_in + off, w_out + off, p_out + off, k.kept, k.kept_words);
    int most = 0;  // moves of the longest span, at most
    for (int j = 0; j < t.n; ++j) {
        const int over = t.s[j].len - keep;
        most = over > most ? over : most;
    }
    if (most <= 0) return;
    if (most > keep) most = keep;
    const int parts = (most + kMoveThreads - 1) / kMoveThreads;
    auto *kern = k.c.head_dim == 128 ? k_kv4_move<128> : k_kv4_move<64>;
    hipLaunchKernelGGL(kern, dim3(nkv * parts, t.n, layers), dim3(kMoveThreads), 0, k.stream, t, k.view(layer_lo), k.per_layer[0],
                       k.per_layer[2], slots, keep, w_in + off, p_in + off, w_out + off, p_out + off, k.kept, k.kept_words, parts);
}

}  // namespace st
