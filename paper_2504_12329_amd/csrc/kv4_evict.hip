// Eviction from the 4-bit key/value cache by accumulated attention weight.
//
// Of a head's `len` slots `keep` stay: those of the last `recent` positions, then those of the largest weight, ties to the
// lowest position.  Attention does not depend on the order of slots, so nothing is compacted: the slots below `keep` that
// are freed take, in ascending order, the slots at or above it that stay, in ascending order.  A context brought back
// from keep + m to keep slots moves at most m of them, in place, and no slot is both read and written.
//
//   k_kv4_evict  one block per head: the keep-th largest weight by up to three digits of 11 bits (histograms in LDS), among ties the positions likewise;
//                a bit per slot, and the moves.  Bound by latency: weights and positions are read once, into registers up to 32768 slots
//                (beyond, once per digit).
//   k_kv4_move   where few heads move many slots: the moves, by several blocks per head.
#include "kv4.h"
#include "st_device.h"

namespace st {

constexpr int kSelThreads = 1024, kBins = 2048, kCopies = 4;
constexpr int kBitWords = 2048;  // bits of 131072 slots fit LDS; those of longer contexts go to the workspace

// Order-preserving image of a weight: NaN below everything, -0 as 0
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t b = __float_as_uint(w + 0.0f);
    return w != w ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr uint32_t kFixedKey = 0xffffffffu;  // of slots that stay without being asked (no weight has it)
constexpr uint32_t kNoKey = 0xfffffffeu;     // of no slot (nor has any weight this)

// Inclusive sum over the lanes of a wave
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp_add(int v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xf, false);
}
__device__ __forceinline__ int wave_running_sum(int v) {
    v = dpp_add<0x111, 0xf>(v);     // row_shr:1
    v = dpp_add<0x112, 0xf>(v);     // row_shr:2
    v = dpp_add<0x114, 0xf>(v);     // row_shr:4
    v = dpp_add<0x118, 0xf>(v);     // row_shr:8
    v = dpp_add<0x142, 0xa>(v);     // row_bcast15 into rows 1 and 3
    return dpp_add<0x143, 0xc>(v);  // row_bcast31 into rows 2 and 3
}

// In the histogram's order (from the top bin down if TOP, else from bin 0 up) the bin that the `rank`-th entry (1-based) lies in, the entries
// before that bin and those in it.  All kSelThreads threads; res is three ints of LDS.  Ends with a barrier, and leaves the histogram cleared.
struct Bin {
    int bin, before, count;
};
template <bool TOP>
__device__ __forceinline__ Bin find_bin(int *hist, int *wsum, int *res, int rank) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int c[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int b = TOP ? kBins - 1 - (2 * tid + e) : 2 * tid + e;
        c[e] = 0;
#pragma unroll
        for (int v = 0; v < kCopies; ++v) c[e] += hist[v * kBins + b], hist[v * kBins + b] = 0;
    }
    const int run = wave_running_sum(c[0] + c[1]);
    if (lane == 63) wsum[wave] = run;
    __syncthreads();
    int base = run - c[0] - c[1];
#pragma unroll
    for (int v = 0; v < kSelThreads / 64; ++v) base += v < wave ? wsum[v] : 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (base < rank && rank <= base + c[e]) res[0] = TOP ? kBins - 1 - (2 * tid + e) : 2 * tid + e, res[1] = base, res[2] = c[e];
        base += c[e];
    }
    __syncthreads();
    return Bin{res[0], res[1], res[2]};
}

// Entries r0 .. r0 + SIZE - 1 of the set bits of words [from, to) of word(i), in order, into list; returns how many set bits there are.  All THREADS
// threads; cnt: THREADS / 64 ints, pre: THREADS ints, xs: THREADS words of LDS.  Ends with a barrier.
template <int THREADS, int SIZE, class W>
__device__ __forceinline__ int list_bits(W word, int from, int to, int r0, int *list, int *cnt, int *pre, uint64_t *xs) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int total = 0;
    for (int i0 = from; i0 < to; i0 += THREADS) {
        const uint64_t x = i0 + tid < to ? word(i0 + tid) : 0;
        const int c = __popcll(x), run = wave_running_sum(c);
        if (lane == 63) cnt[wave] = run;
        __syncthreads();
        int first = total + run - c;
#pragma unroll
        for (int v = 0; v < THREADS / 64; ++v) {
            first += v < wave ? cnt[v] : 0;
            total += cnt[v];
        }
        pre[tid] = first - r0, xs[tid] = x;
        __syncthreads();
        const int n = min(THREADS, to - i0);
        // a wave a word, a lane a bit, four words at a time
        for (int j0 = wave; j0 < n; j0 += THREADS / 16) {
            uint64_t y[4];
            int at[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = min(j0 + e * (THREADS / 64), THREADS - 1);  // (words past n are zeros)
                y[e] = xs[j], at[e] = pre[j];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = at[e] + __popcll(y[e] & ((1ull << lane) - 1));
                if ((y[e] >> lane & 1) && j0 + e * (THREADS / 64) < n && r >= 0 && r < SIZE) list[r] = (i0 + j0 + e * (THREADS / 64)) * 64 + lane;
            }
        }
        __syncthreads();
    }
    return total;
}

// The bits of word i that count: freed slots below keep, or late ones from keep on (of n)
__device__ __forceinline__ uint64_t freed_word(uint64_t bits, int i, int keep) {
    return ~bits & (keep - i * 64 >= 64 ? ~0ull : (1ull << (keep - i * 64)) - 1);
}
__device__ __forceinline__ uint64_t late_word(uint64_t bits, int i, int n, int keep) {
    const int s0 = i * 64;
    const uint64_t held = n - s0 >= 64 ? ~0ull : (1ull << (n - s0)) - 1;
    return bits & held & (s0 >= keep ? ~0ull : ~((1ull << (keep - s0)) - 1));  // (word keep / 64 on)
}

struct Planes {  // of one layer, sequence and head
    uint8_t *k, *v, *ks, *vs;
    const float *w_in;
    const int32_t *p_in;
    float *w_out;
    int32_t *p_out;
};
// Slots late[i] to freed[i], i < m: D / 16 threads a slot, 16 bytes of codes each, a few slots' loads in flight
template <int D, int THREADS>
__device__ __forceinline__ void move_slots(const Planes &p, const int *late, const int *freed, int m) {
    constexpr int CB = D / 2, SB = D / 32, TPM = CB / 16 * 2, U = 4;
    for (int u0 = threadIdx.x; u0 < m * TPM; u0 += U * THREADS) {
        u32x4 x[U];
        uint32_t y[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = u0 + j * THREADS, e = u % TPM;
            if (u >= m * TPM) continue;
            const int src = late[u / TPM];
            x[j] = *reinterpret_cast<const u32x4 *>((e < TPM / 2 ? p.k : p.v) + (size_t)src * CB + e % (TPM / 2) * 16);
            const uint8_t *s = e ? p.vs : p.ks;
            if (e < 2) y[j] = SB == 4 ? reinterpret_cast<const uint32_t *>(s)[src] : reinterpret_cast<const uint16_t *>(s)[src];
            else if (e == 2) y[j] = __float_as_uint(p.w_in[src]);
            else if (e == 3) y[j] = (uint32_t)p.p_in[src];
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int u = u0 + j * THREADS, e = u % TPM;
            if (u >= m * TPM) continue;
            const int dst = freed[u / TPM];
            *reinterpret_cast<u32x4 *>((e < TPM / 2 ? p.k : p.v) + (size_t)dst * CB + e % (TPM / 2) * 16) = x[j];
            if (e < 2) {
                uint8_t *s = e ? p.vs : p.ks;
                if constexpr (SB == 4) reinterpret_cast<uint32_t *>(s)[dst] = y[j];
                else reinterpret_cast<uint16_t *>(s)[dst] = (uint16_t)y[j];
            } else if (e == 2) {
                p.w_out[dst] = __uint_as_float(y[j]);
            } else if (e == 3) {
                p.p_out[dst] = (int32_t)y[j];
            }
        }
    }
}

struct EvictArgs {
    Kv4View view;  // of the first layer
    size_t k_layer, s_layer, layer_slots;
    int keep, recent, parts;  // parts: blocks of k_kv4_move per head; 0: k_kv4_evict moves
    const float *w_in;
    const int32_t *p_in;
    float *w_out;
    int32_t *p_out;
    uint64_t *kept;
    size_t kept_words;
};
template <int D>
__device__ __forceinline__ Planes planes_of(const EvictArgs &a, const Kv4Span &sp, int kvh, int layer) {
    const size_t head = ((size_t)sp.seq * a.view.nkv + kvh) * a.view.max_seq, at = layer * a.layer_slots + head;
    const size_t k = layer * a.k_layer + head * (D / 2), s = layer * a.s_layer + head * (D / 32);
    return Planes{a.view.k + k, a.view.v + k, a.view.ks + s, a.view.vs + s, a.w_in + at, a.p_in + at, a.w_out + at, a.p_out + at};
}

// SINGLE: all slots are in registers (at most 1024 PER), else they are read anew for every digit
template <int D, int PER, bool SINGLE, int CAP>
__global__ __launch_bounds__(kSelThreads) void k_kv4_evict(const Kv4Spans<CAP> t, const EvictArgs a) {
    constexpr int kChunk = kSelThreads * PER, kList = 1024;
    __shared__ __align__(16) int hist[kCopies * kBins];
    __shared__ int wsum[kSelThreads / 64], res[3];
    __shared__ uint64_t bits_s[kBitWords];
    const Kv4Span sp = t.s[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = sp.len, keep = a.keep;
    const Planes pl = planes_of<D>(a, sp, blockIdx.x, blockIdx.z);
    const bool copy = a.w_out != a.w_in;
    if (n <= keep) {
        if (copy)
            for (int i = tid; i < n; i += kSelThreads) pl.w_out[i] = pl.w_in[i], pl.p_out[i] = pl.p_in[i];
        return;
    }
    const int fixed_from = sp.pos - a.recent;  // positions from here on stay
    uint32_t key[PER];  // (positions are read again where they decide between equal weights)
    auto load = [&](int i0) {
        constexpr int U = PER < 16 ? PER : 16;  // at a time
#pragma unroll
        for (int e0 = 0; e0 < PER; e0 += U) {
            if (i0 + e0 * kSelThreads >= n) break;
            int pos[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int i = i0 + (e0 + e) * kSelThreads + tid;
                pos[e] = i < n ? pl.p_in[i] : 0;
                key[e0 + e] = i < n ? __float_as_uint(pl.w_in[i]) : 0;
            }
#pragma unroll
            for (int e = 0; e < U; ++e) {
                key[e0 + e] = pos[e] >= fixed_from ? kFixedKey : weight_key(__uint_as_float(key[e0 + e]));
                if (i0 + (e0 + e) * kSelThreads + tid >= n) key[e0 + e] = kNoKey;
            }
        }
    };
    auto each = [&](auto f) {  // f(slot, key) over all slots (and some past the last, without a key)
        for (int i0 = 0; i0 < n; i0 += kChunk) {
            if (!SINGLE) load(i0);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                if (i0 + e * kSelThreads >= n) break;
                f(i0 + e * kSelThreads + tid, key[e]);
            }
        }
    };
    if (SINGLE) load(0);
    for (int i = tid; i < kCopies * kBins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    int *mine = hist + (wave % kCopies) * kBins;

    // Threshold: keys above it stay, and of those equal to it all, or `ties` by position.  The first digit also counts the slots that stay
    // without being asked.
    int fixed = 0;
    each([&](int, uint32_t k) {
        if (k < kNoKey) atomicAdd(&mine[k >> 21], 1);
        fixed += k == kFixedKey;
    });
    fixed = __builtin_amdgcn_readlane(wave_running_sum(fixed), 63);
    if (lane == 0) wsum[wave] = fixed;
    __syncthreads();
    fixed = 0;
#pragma unroll
    for (int v = 0; v < kSelThreads / 64; ++v) fixed += wsum[v];
    __syncthreads();
    uint32_t threshold = kFixedKey;
    bool all_equal = false;  // those equal to the threshold, or above it up to the digit's end, all stay
    int need = keep;
    if (fixed < keep) {
        need = keep - fixed;
        Bin b = find_bin<true>(hist, wsum, res, need);
        need -= b.before;
        uint32_t prefix = b.bin;
        int shift = 21;
        if (need != b.count) {
            each([&](int, uint32_t k) {
                if (k < kNoKey && k >> 21 == prefix) atomicAdd(&mine[k >> 10 & 2047], 1);
            });
            __syncthreads();
            b = find_bin<true>(hist, wsum, res, need);
            need -= b.before;
            prefix = prefix << 11 | b.bin, shift = 10;
            if (need != b.count) {
                each([&](int, uint32_t k) {
                    if (k < kNoKey && k >> 10 == prefix) atomicAdd(&mine[k & 1023], 1);
                });
                __syncthreads();
                b = find_bin<true>(hist, wsum, res, need);
                need -= b.before;
                prefix = prefix << 10 | b.bin, shift = 0;
            }
        }
        threshold = prefix << shift;
        all_equal = need == b.count;
    } else {
        __syncthreads();
        for (int i = tid; i < kCopies * kBins; i += kSelThreads) hist[i] = 0;  // (the first digit's)
        __syncthreads();
        all_equal = need == fixed;
    }
    // among the ties: the `need` lowest positions (and, should positions repeat, the lowest slots)
    uint32_t at_most = 0;
    int ties = need;
    if (!all_equal) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
            each([&](int i, uint32_t k) {
                if (k != threshold) return;
                const uint32_t x = (uint32_t)pl.p_in[i] ^ 0x80000000u;
                if ((pass == 0 || x >> (shift + width & 31) == at_most)) atomicAdd(&mine[x >> shift & ((1 << width) - 1)], 1);
            });
            __syncthreads();
            const Bin b = find_bin<false>(hist, wsum, res, ties);
            ties -= b.before;
            at_most = at_most << width | b.bin;
        }
    }
    // the bits
    uint64_t *bits = bits_s;
    if (n > kBitWords * 64 || a.parts) bits = a.kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * a.view.nkv + blockIdx.x) * a.kept_words;
    int done = 0;  // ties with the last position, in the slots before
    auto mark = [&](int i, uint32_t k) {  // (i may be past n)
        const uint32_t x = !all_equal && k == threshold ? (uint32_t)pl.p_in[i] ^ 0x80000000u : 0;
        bool stays = k != kNoKey && (all_equal ? k >= threshold : k > threshold || (k == threshold && x < at_most));
        if (!all_equal) {
            const bool tie = k == threshold && x == at_most;
            const uint64_t tied = __builtin_amdgcn_ballot_w64(tie);
            if (lane == 0) wsum[wave] = __popcll(tied);
            __syncthreads();
            int before = done;
#pragma unroll
            for (int v = 0; v < kSelThreads / 64; ++v) {
                before += v < wave ? wsum[v] : 0;
                done += wsum[v];
            }
            if (tie) stays = before + __popcll(tied & ((1ull << lane) - 1)) < ties;
            __syncthreads();
        }
        const uint64_t word = __builtin_amdgcn_ballot_w64(stays);
        if (lane == 0 && i < n) bits[i >> 6] = word;
        if (copy && stays && i < keep) pl.w_out[i] = pl.w_in[i], pl.p_out[i] = pl.p_in[i];
    };
    for (int i0 = 0; i0 < n; i0 += kChunk) {
        if (!SINGLE) load(i0);
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (i0 + e * kSelThreads < n) mark(i0 + e * kSelThreads + tid, key[e]);
    }
    if (a.parts) return;
    __syncthreads();
    // the moves; the histogram's memory holds the lists
    int *freed = hist, *late = hist + kList, *pre = hist + 2 * kList;
    uint64_t *xs = reinterpret_cast<uint64_t *>(hist + 3 * kList);
    static_assert(3 * kList + 2 * kSelThreads <= kCopies * kBins && kList == kSelThreads, "lists in the histogram");
    for (int r0 = 0;; r0 += kList) {
        list_bits<kSelThreads, kList>([&](int i) { return freed_word(bits[i], i, keep); }, 0, (keep + 63) / 64, r0, freed, wsum, pre, xs);
        const int total = list_bits<kSelThreads, kList>([&](int i) { return late_word(bits[i], i, n, keep); }, keep / 64, (n + 63) / 64, r0, late, wsum, pre, xs);
        move_slots<D, kSelThreads>(pl, late, freed, min(total - r0, kList));
        if (r0 + kList >= total) return;
        __syncthreads();
    }
}

// Moves part * 256 .. + 255, and every parts * 256 further, of a head
constexpr int kMoveThreads = 256;
template <int D, int CAP>
__global__ __launch_bounds__(kMoveThreads) void k_kv4_move(const Kv4Spans<CAP> t, const EvictArgs a) {
    __shared__ int freed[kMoveThreads], late[kMoveThreads], pre[kMoveThreads], cnt[kMoveThreads / 64];
    __shared__ uint64_t xs[kMoveThreads];
    const Kv4Span sp = t.s[blockIdx.y];
    const int n = sp.len, keep = a.keep, kvh = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    if (n <= keep) return;
    const Planes pl = planes_of<D>(a, sp, kvh, blockIdx.z);
    const uint64_t *bits = a.kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * a.view.nkv + kvh) * a.kept_words;
    for (int r0 = part * kMoveThreads;; r0 += a.parts * kMoveThreads) {
        list_bits<kMoveThreads, kMoveThreads>([&](int i) { return freed_word(bits[i], i, keep); }, 0, (keep + 63) / 64, r0, freed, cnt, pre, xs);
        const int total = list_bits<kMoveThreads, kMoveThreads>([&](int i) { return late_word(bits[i], i, n, keep); }, keep / 64, (n + 63) / 64, r0,
                                                                late, cnt, pre, xs);
        move_slots<D, kMoveThreads>(pl, late, freed, min(total - r0, kMoveThreads));
        if (r0 + a.parts * kMoveThreads >= total) return;
        __syncthreads();
    }
}

// Moves by blocks of their own from so many moves of one head, and below so many heads
constexpr int kMoveMany = 1024, kMoveHeads = 128;

void launch_kv4_evict(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int keep, int recent, const float *w_in,
                      const int32_t *p_in, float *w_out, int32_t *p_out) {
    const int nkv = k.c.n_kv_heads, layers = layer_hi - layer_lo;
    const size_t slots = (size_t)k.c.n_seq * nkv * k.c.max_seq, off = slots * layer_lo;
    int longest = 0;
    for (int j = 0; j < t.n; ++j) longest = t.s[j].len > longest ? t.s[j].len : longest;
    const int over = longest - keep > 0 ? longest - keep : 0, moves = over < keep ? over : keep;  // at most, of one head
    const int parts = moves > kMoveMany && nkv * t.n * layers < kMoveHeads ? (moves + kMoveThreads - 1) / kMoveThreads : 0;
    const EvictArgs a = {k.view(layer_lo), k.per_layer[0], k.per_layer[2], slots, keep, recent, parts, w_in + off, p_in + off, w_out + off,
                         p_out + off, k.kept, k.kept_words};
    with_table(t, [&](auto tab) {
        constexpr int CAP = sizeof(tab.s) / sizeof(Kv4Span);
#define ST_EVICT(DV)                                                                                         \
    (longest <= 4096    ? k_kv4_evict<DV, 4, true, CAP>                                                      \
     : longest <= 32768 ? k_kv4_evict<DV, 32, true, CAP>                                                     \
                        : k_kv4_evict<DV, 32, false, CAP>)
        auto *kern = k.c.head_dim == 128 ? ST_EVICT(128) : ST_EVICT(64);
#undef ST_EVICT
        hipLaunchKernelGGL(kern, dim3(nkv, t.n, layers), dim3(kSelThreads), 0, k.stream, tab, a);
        if (!parts) return;
        auto *move = k.c.head_dim == 128 ? k_kv4_move<128, CAP> : k_kv4_move<64, CAP>;
        hipLaunchKernelGGL(move, dim3(nkv * parts, t.n, layers), dim3(kMoveThreads), 0, k.stream, tab, a);
    });
}

}  // namespace st
