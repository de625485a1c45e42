// Eviction from the 4-bit key/value cache by accumulated attention weight.
//
// Of a head's `len` slots `keep` stay: those of the last `recent` positions, then those of the largest weight, ties to the
// lowest position.  Attention does not depend on the order of slots, so nothing is compacted: the slots below `keep` that are
// freed take, in ascending order, the slots at or above it that stay, in ascending order.  A context brought back from keep + m
// to keep slots moves at most m of them, in place, and no slot is both read and written.
//
// A slot's rank is that of 64 bits: its class and weight (32 bits, larger first), then its position (lower first).
// k_kv4_evict, one block per head, finds the keep-th by histograms of 11-bit digits in LDS until at most 128 slots share the
// digits so far, and ranks those against each other; it writes a bit per slot and moves.  Weights and positions are read once,
// the 32 bits kept in LDS (up to 24576 slots; beyond, they are read again for every digit).  Bound by latency, also of
// instructions, as every line runs but a few times: 128 heads of 500 to 6000 slots to 1024 19 us (measured at 18: 21 with loops
// unrolled 8 and 16 times); 56 heads of 577 slots to 512 8.2 us, 16 heads of 16385 slots 15.8 us.  Read again for every digit: 8
// heads of 32768 slots 46 us, two of 200000 260.  (Histograms over the range that the weights span, which need no second digit, cost
// a reduction first: 0.4 to 3 us more.)  k_kv4_move: where few heads move many slots, the moves by several blocks per head.
#include <atomic>

#include "kv4.h"
#include "st_device.h"

namespace st {

constexpr int kBins = 2048, kDirect = 128;
constexpr int kHeldSlots = 24576, kBitSlots = 131072;  // LDS: 4 bytes a slot, or a bit a slot (those of longer contexts go to the workspace)

// 32 bits that order slots: those that stay without being asked first (0), then by weight, larger first; -0 is 0, NaN is last
__device__ __forceinline__ uint32_t order_of(float w, bool fixed) {
    const uint32_t b = __float_as_uint(w + 0.0f);
    return fixed ? 0u : w != w ? 0xffffffffu : (b & 0x80000000u) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ uint32_t order_of(int pos) { return (uint32_t)pos ^ 0x80000000u; }

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

// The bin that the `rank`-th entry (1-based) of the histogram lies in, the entries before that bin and those in it.  All
// THREADS threads; hist is COPIES histograms, added up; res is three ints of LDS.  Ends with a barrier, and leaves the
// histograms cleared.
struct Bin {
    int bin, before, count;
};
template <int THREADS, int COPIES>
__device__ __forceinline__ Bin find_bin(int *hist, int *wsum, int *res, int rank) {
    constexpr int BPT = kBins / THREADS;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int c[BPT], sum = 0;
#pragma unroll
    for (int e = 0; e < BPT; ++e) c[e] = 0;
#pragma unroll
    for (int v = 0; v < COPIES; ++v)
#pragma unroll
        for (int e = 0; e < BPT; ++e) c[e] += hist[v * kBins + BPT * tid + e];
#pragma unroll
    for (int v = 0; v < COPIES; ++v)
#pragma unroll
        for (int e = 0; e < BPT; ++e) hist[v * kBins + BPT * tid + e] = 0;
#pragma unroll
    for (int e = 0; e < BPT; ++e) sum += c[e];
    const int run = wave_running_sum(sum);
    if (lane == 63) wsum[wave] = run;
    __syncthreads();
    int base = run - sum;
#pragma unroll
    for (int v = 0; v < THREADS / 64; ++v) base += v < wave ? wsum[v] : 0;
#pragma unroll
    for (int e = 0; e < BPT; ++e) {
        if (base < rank && rank <= base + c[e]) res[0] = BPT * tid + e, res[1] = base, res[2] = c[e];
        base += c[e];
    }
    __syncthreads();
    return Bin{res[0], res[1], res[2]};
}

// The bits of word i that count: freed slots below keep, or late ones from keep on (of n)
__device__ __forceinline__ uint64_t freed_word(uint64_t bits, int i, int keep) {
    return i * 64 >= keep ? 0 : ~bits & (keep - i * 64 >= 64 ? ~0ull : (1ull << (keep - i * 64)) - 1);
}
__device__ __forceinline__ uint64_t late_word(uint64_t bits, int i, int n, int keep) {
    const int s0 = i * 64;
    const uint64_t held = n - s0 >= 64 ? ~0ull : (1ull << (n - s0)) - 1;
    return s0 + 64 <= keep ? 0 : bits & held & (s0 >= keep ? ~0ull : ~((1ull << (keep - s0)) - 1));
}

// Entries r0 .. r0 + SIZE - 1 of the freed slots and of the late ones, in order, into list[0] and list[1]; returns how many there are
// of each.  Every wave counts all words' bits, 64 words at a time with a word to a lane, so that no wave waits for another; then it
// takes every WAVES-th word, with a bit to a lane.  All THREADS threads; ends with a barrier.
template <int THREADS, int SIZE>
__device__ __forceinline__ int list_moves(const uint64_t *bits, int n, int keep, int r0, int *freed, int *late) {
    constexpr int WAVES = THREADS / 64, U = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), words = (n + 63) / 64;
    int total[2] = {0, 0};
    for (int i0 = 0; i0 < words; i0 += 64 * U) {
        uint64_t b[U];
#pragma unroll
        for (int e = 0; e < U; ++e) b[e] = bits[min(i0 + 64 * e + lane, words - 1)];
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const int w0 = i0 + 64 * e, w = w0 + lane;
            if (w0 >= words) break;
            const uint64_t x[2] = {w < words ? freed_word(b[e], w, keep) : 0, w < words ? late_word(b[e], w, n, keep) : 0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int own = __popcll(x[h]), run = wave_running_sum(own), first = total[h] + run - own - r0;
                const int all = __builtin_amdgcn_readlane(run, 63);
                total[h] += all;
                if (!all || total[h] - all >= r0 + SIZE || total[h] <= r0) continue;  // none of the entries is in these words
                int *list = h ? late : freed;
                const bool inside = total[h] - all >= r0 && total[h] <= r0 + SIZE;
#pragma unroll
                for (int k = 0; k < 64; k += WAVES) {
                    const uint32_t y0 = __builtin_amdgcn_readlane((int)(uint32_t)x[h], k + wave), y1 = __builtin_amdgcn_readlane((int)(x[h] >> 32), k + wave);
                    if (!(y0 | y1)) continue;
                    const int r = __builtin_amdgcn_readlane(first, k + wave) + __builtin_amdgcn_mbcnt_hi(y1, __builtin_amdgcn_mbcnt_lo(y0, 0));
                    if (__builtin_amdgcn_inverse_ballot_w64((uint64_t)y1 << 32 | y0) && (inside || (uint32_t)r < (uint32_t)SIZE))
                        list[r] = (w0 + k + wave) * 64 + lane;
                }
            }
        }
    }
    __syncthreads();
    return total[1];
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

// The ledger's entries of the slots from `first` on that stay where they are, to another ledger
template <int THREADS>
__device__ __forceinline__ void copy_kept(const Planes &p, const uint64_t *bits, int first, int end) {
    for (int i = first + threadIdx.x; i < end; i += THREADS)
        if (bits[i >> 6] >> (i & 63) & 1) p.w_out[i] = p.w_in[i], p.p_out[i] = p.p_in[i];
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

// HELD: the slots' 32 bits are kept in LDS
template <int D, int THREADS, bool HELD, int CAP>
__global__ __launch_bounds__(THREADS) void k_kv4_evict(const Kv4Spans<CAP> t, const EvictArgs a) {
    constexpr int COPIES = THREADS / 256, WAVES = THREADS / 64;
    extern __shared__ __align__(16) uint64_t dyn[];  // the bits, then the slots' 32 bits
    __shared__ __align__(16) int hist[COPIES * kBins];  // (and later the lists of moves)
    __shared__ __align__(16) int wsum[WAVES], res[3], n_near;
    __shared__ __align__(16) uint32_t near_o[kDirect], near_p[kDirect];
    __shared__ __align__(16) int near_s[kDirect], near_rank[kDirect];
    const Kv4Span sp = t.s[blockIdx.y];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = sp.len, keep = a.keep;
    const Planes pl = planes_of<D>(a, sp, blockIdx.x, blockIdx.z);
    const bool copy = a.w_out != a.w_in;
    if (n <= keep) {
        if (copy)
            for (int i = tid; i < n; i += THREADS) pl.w_out[i] = pl.w_in[i], pl.p_out[i] = pl.p_in[i];
        return;
    }
    const int fixed_from = sp.pos - a.recent, words = (n + 63) / 64;  // positions from fixed_from on stay
    uint64_t *bits = dyn;
    if (n > kBitSlots || a.parts) bits = a.kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * a.view.nkv + blockIdx.x) * a.kept_words;
    uint32_t *held = reinterpret_cast<uint32_t *>(dyn + words);
    for (int i = tid; i < COPIES * kBins; i += THREADS) hist[i] = 0;
    if (tid == 0) n_near = 0;
    if (tid < kDirect) near_rank[tid] = 0;
    __syncthreads();
    int *mine = hist + (wave % COPIES) * kBins;
    // f(slot, its 32 bits) for all slots; whole waves, `in` says which lanes have one
    auto each = [&](auto f) {
        constexpr int U = HELD ? 1 : 4;
        for (int i0 = 0; i0 < n; i0 += U * THREADS) {
            uint32_t o[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int i = min(i0 + e * THREADS + tid, n - 1);
                o[e] = HELD ? held[i] : order_of(pl.w_in[i], pl.p_in[i] >= fixed_from);
            }
#pragma unroll
            for (int e = 0; e < U; ++e) f(i0 + e * THREADS + tid, o[e], i0 + e * THREADS + tid < n);
        }
    };
    // a histogram entry; those that stay anyway are many, share bin 0, and are counted aside
    int anyway = 0;
    auto count = [&](uint32_t o) {
        if (o >> 21) atomicAdd(&mine[o >> 21], 1);
        else ++anyway;
    };
    if constexpr (HELD) {
        constexpr int U = 4;
        for (int i0 = 0; i0 < n; i0 += U * THREADS) {
            int p[U];
            float w[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int i = min(i0 + e * THREADS + tid, n - 1);
                p[e] = pl.p_in[i], w[e] = pl.w_in[i];
            }
#pragma unroll
            for (int e = 0; e < U; ++e) {
                const int i = i0 + e * THREADS + tid;
                const uint32_t o = order_of(w[e], p[e] >= fixed_from);
                if (i < n) {
                    held[i] = o;
                    count(o);
                }
            }
        }
    } else {
        each([&](int, uint32_t o, bool in) {
            if (in) count(o);
        });
    }
    anyway = wave_running_sum(anyway);
    if (lane == 63 && anyway) atomicAdd(&mine[0], anyway);
    __syncthreads();
    // Digits of the 64 bits until few slots share them: `prefix` of the first `top` bits, of which `need` slots stay
    Bin b = find_bin<THREADS, COPIES>(hist, wsum, res, keep);
    int need = keep - b.before, top = 11;
    uint32_t prefix = b.bin, prefix_p = 0;  // of the 32 bits, and of the position's
    while (need != b.count && b.count > kDirect && top < 64) {
        const int width = top == 22 || top == 54 ? 10 : 11;
        const int from = top < 32 ? 32 - top : 64 - top;  // bits of the word below the prefix
        each([&](int i, uint32_t o, bool in) {
            if (top < 32) {
                if (in && o >> from == prefix) atomicAdd(&mine[o >> (from - width) & ((1 << width) - 1)], 1);
            } else if (in && o == prefix) {
                const uint32_t p = order_of(pl.p_in[i]);
                if (top == 32 || p >> from == prefix_p) atomicAdd(&mine[p >> (from - width) & ((1 << width) - 1)], 1);
            }
        });
        __syncthreads();
        b = find_bin<THREADS, COPIES>(hist, wsum, res, need);
        need -= b.before;
        if (top < 32) prefix = prefix << width | b.bin;
        else prefix_p = prefix_p << width | b.bin;
        top += width;
    }
    const bool all = need == b.count, ranked = !all && b.count <= kDirect;
    if (top <= 32) {
        // slots below `low` stay, of those from it to `high` all or the ones that rank below `need`
        const uint32_t low = prefix << (32 - top), high = low + ((1u << (32 - top)) - 1);
        each([&](int i, uint32_t o, bool in) {
            const uint64_t word = all ? __builtin_amdgcn_ballot_w64(in && o <= high) : __builtin_amdgcn_ballot_w64(in && o < low);
            if (lane == 0 && in) bits[i >> 6] = word;
            const bool like = in && o - low <= high - low;
            if (ranked && __builtin_amdgcn_ballot_w64(like)) {
                if (like) {
                    const int at = atomicAdd(&n_near, 1);
                    near_o[at] = o, near_p[at] = order_of(pl.p_in[i]), near_s[at] = i;
                }
            }
        });
    } else {
        const int from = 64 - top;
        int done = 0;  // of slots alike in all 64 bits (a ledger of repeated positions), the first stay
        each([&](int i, uint32_t o, bool in) {
            uint32_t p = 0;
            if (in && o == prefix) p = order_of(pl.p_in[i]);
            const bool less = in && (o < prefix || (o == prefix && p >> from < prefix_p)), like = in && o == prefix && p >> from == prefix_p;
            bool stays = less || (all && like);
            if (ranked && like) {
                const int at = atomicAdd(&n_near, 1);
                near_o[at] = o, near_p[at] = p, near_s[at] = i;
            }
            if (!all && !ranked) {
                const uint64_t alike = __builtin_amdgcn_ballot_w64(like);
                if (lane == 0) wsum[wave] = __popcll(alike);
                __syncthreads();
                int before = done;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    before += v < wave ? wsum[v] : 0;
                    done += wsum[v];
                }
                if (like) stays = before + __popcll(alike & ((1ull << lane) - 1)) < need;
                __syncthreads();
            }
            const uint64_t word = __builtin_amdgcn_ballot_w64(stays);
            if (lane == 0 && in) bits[i >> 6] = word;
        });
    }
    __syncthreads();
    if (ranked) {  // b.count slots, THREADS / kDirect threads each
        const int c = tid % kDirect;
        if (c < b.count) {
            const uint64_t x = (uint64_t)near_o[c] << 32 | near_p[c];
            const int slot = near_s[c];
            int rank = 0;
            for (int j = tid / kDirect; j < b.count; j += THREADS / kDirect) {
                const uint64_t y = (uint64_t)near_o[j] << 32 | near_p[j];
                rank += y < x || (y == x && near_s[j] < slot);
            }
            atomicAdd(&near_rank[c], rank);
        }
        __syncthreads();
        if (tid < b.count && near_rank[tid] < need)
            atomicOr(reinterpret_cast<unsigned long long *>(&bits[near_s[tid] >> 6]), 1ull << (near_s[tid] & 63));
        __syncthreads();
    }
    if (a.parts) return;
    if (copy) copy_kept<THREADS>(pl, bits, 0, keep);
    // the moves; the histogram's memory holds the lists
    constexpr int kList = THREADS;
    static_assert(2 * kList * sizeof(int) <= sizeof(hist), "lists in the histogram");
    int *freed = hist, *late = hist + kList;
    for (int r0 = 0;; r0 += kList) {
        const int total = list_moves<THREADS, kList>(bits, n, keep, r0, freed, late);
        move_slots<D, THREADS>(pl, late, freed, min(total - r0, kList));
        if (r0 + kList >= total) return;
        __syncthreads();
    }
}

// Ledger entries of a part of the slots that stay, and moves part * kMovesPer .. + kMovesPer - 1 of a head, which has blocks for all the
// moves that it can have.  Bound by latency: listing, then loads and stores.  16 heads with 2000 moves each 10.6 us; with the
// selection, measured at the time, 28.0 us at 256 moves a block, 29.5 at 512, 31.2 at 128.
constexpr int kMoveThreads = 1024, kMovesPer = 256;
template <int D, int CAP>
__global__ __launch_bounds__(kMoveThreads) void k_kv4_move(const Kv4Spans<CAP> t, const EvictArgs a) {
    __shared__ int freed[kMovesPer], late[kMovesPer];
    const Kv4Span sp = t.s[blockIdx.y];
    const int n = sp.len, keep = a.keep, kvh = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    if (n <= keep) return;
    const Planes pl = planes_of<D>(a, sp, kvh, blockIdx.z);
    const uint64_t *bits = a.kept + (((size_t)blockIdx.z * t.n + blockIdx.y) * a.view.nkv + kvh) * a.kept_words;
    if (a.w_out != a.w_in) {
        const int share = (keep + a.parts - 1) / a.parts;
        copy_kept<kMoveThreads>(pl, bits, part * share, min(keep, (part + 1) * share));
    }
    const int total = list_moves<kMoveThreads, kMovesPer>(bits, n, keep, part * kMovesPer, freed, late);
    move_slots<D, kMoveThreads>(pl, late, freed, min(total - part * kMovesPer, kMovesPer));
}

// Moves by blocks of their own from so many moves of one head, and below so many heads.  One launch : two, both of these kernels, us:
//   slots, kept      2048, 1024   2500, 1250   3000, 1500   4096, 2048   8192, 4096   16385, 4096
//     8 heads       10.8 : 12.1  11.9 : 12.5  12.9 : 13.0  15.8 : 13.4  26.3 : 15.6   44.1 : 20.6
//    32 heads       11.0 : 12.5  12.2 : 12.9  13.2 : 13.6  17.1 : 15.0  28.3 : 19.6   48.5 : 29.2
//    96 heads       11.8 : 16.5  13.3 : 16.2  14.6 : 17.9  19.0 : 23.5  31.3 : 33.1   52.0 : 47.5
//   128 heads       12.3 : 18.6  13.6 : 18.6  15.1 : 20.9  19.9 : 26.2  33.3 : 38.9   56.9 : 58.2
// (one is the better for 64 heads and more below some 3000 moves, and up to 1500 moves: the rule loses up to 4.5 us there)
constexpr int kMoveMany = 1024, kMoveHeads = 128;

// Up to 99 KB of LDS are asked for at the launch of a block of 1024 threads: allowed once per kernel and GPU
template <int D, int CAP>
static hipError_t allow_held_lds() {
    static std::atomic<uint64_t> allowed{0};  // a bit per GPU; those past 64 are asked every time
    int gpu = 0;
    hipError_t e = hipGetDevice(&gpu);
    if (e != hipSuccess) return e;
    const uint64_t bit = gpu >= 0 && gpu < 64 ? 1ull << gpu : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_kv4_evict<D, 1024, true, CAP>), hipFuncAttributeMaxDynamicSharedMemorySize,
                            kHeldSlots * 4 + kHeldSlots / 8);
    if (e == hipSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

template <int D, int CAP>
static hipError_t evict_in(const Kv4 &k, const Kv4Spans<CAP> &t, const EvictArgs &a, int longest, dim3 grid) {
    const size_t bit_bytes = (size_t)((longest + 63) / 64) * 8;
    // Blocks of 256 threads for short contexts (cheaper barriers and scans) and, where there is more than one block a compute unit, for longer ones, as two
    // of 1024 threads do not run side by side.  256 : 1024 threads, 56 heads of 300 slots 8.0 : 9.5 us, of 1100 16.6 : 11.9; 320 heads of 700 slots
    // 11.7 : 19.6, of 2500 25.5 : 27.4, of 4000 47.6 : 42.0.
    const int64_t heads = (int64_t)grid.x * grid.y * grid.z;
    if (longest <= (heads > 256 ? 2560 : 768)) {
        hipLaunchKernelGGL((k_kv4_evict<D, 256, true, CAP>), grid, dim3(256), bit_bytes + 4 * (size_t)longest, k.stream, t, a);
    } else if (longest <= kHeldSlots) {
        const hipError_t e = allow_held_lds<D, CAP>();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((k_kv4_evict<D, 1024, true, CAP>), grid, dim3(1024), bit_bytes + 4 * (size_t)longest, k.stream, t, a);
    } else {
        hipLaunchKernelGGL((k_kv4_evict<D, 1024, false, CAP>), grid, dim3(1024), longest <= kBitSlots ? bit_bytes : kBitSlots / 8, k.stream, t, a);
    }
    if (a.parts) hipLaunchKernelGGL((k_kv4_move<D, CAP>), dim3(grid.x * a.parts, grid.y, grid.z), dim3(kMoveThreads), 0, k.stream, t, a);
    return hipGetLastError();
}

hipError_t launch_kv4_evict(const Kv4 &k, int layer_lo, int layer_hi, const Kv4Table &t, int keep, int recent, const float *w_in,
                      const int32_t *p_in, float *w_out, int32_t *p_out) {
    const int nkv = k.c.n_kv_heads, layers = layer_hi - layer_lo;
    const size_t slots = (size_t)k.c.n_seq * nkv * k.c.max_seq, off = slots * layer_lo;
    int longest = 0;
    for (int j = 0; j < t.n; ++j) longest = t.s[j].len > longest ? t.s[j].len : longest;
    const int over = longest - keep > 0 ? longest - keep : 0, moves = over < keep ? over : keep;  // at most, of one head
    const int parts = moves > kMoveMany && nkv * t.n * layers < kMoveHeads ? (moves + kMovesPer - 1) / kMovesPer : 0;
    const EvictArgs a = {k.view(layer_lo), k.per_layer[0], k.per_layer[2], slots, keep, recent, parts, w_in + off, p_in + off, w_out + off,
                         p_out + off, k.kept, k.kept_words};
    hipError_t e = hipSuccess;
    with_table(t, [&](auto tab) {
        const dim3 grid(nkv, t.n, layers);
        e = k.c.head_dim == 128 ? evict_in<128>(k, tab, a, longest, grid) : evict_in<64>(k, tab, a, longest, grid);
    });
    return e;
}

}  // namespace st
