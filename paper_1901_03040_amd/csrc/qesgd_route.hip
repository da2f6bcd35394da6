// The router of a layer of experts: each token's k largest logits and their softmax, and the (token, choice) pairs sorted by expert.
//
//   p_e = exp(l_e - max l) / sum_i exp(l_i - max l);  gates: p at the chosen, or their share of the chosen ones' sum
//   place of a pair = pairs of lower experts + earlier pairs of its expert
//
// A token's logits lie in the registers of a part of a wave; the largest is found k times, ties by the lower number.  The sort counts: every block of
// tokens counts its pairs by expert, the counts of the blocks before a block and of the experts before an expert give each block its
// first places, and inside a block a pair finds the earlier ones of its expert by comparing the bits of the experts' numbers across the wave.  Only
// integers are counted, so the result is the same however the work falls.
//
// Measured, kernels by the trace: one token of 64 experts 3.8 us, 8192 tokens of 64 bf16 3.4 + 5.0 us (choice and places), which is launches and chains of trips to memory; 160001 of
// 257 f32, six each, softmax over all, 56 (choice: 165 MB, vector instructions, two thirds of them to find the largest six times) + 12.5 + 14 us, in a graph 76 together; gradient 66 us = 5.0 TB/s.
#include "qesgd_experts.h"
#include "qesgd_groups.h"
#include "qesgd_launch.h"

namespace qesgd {
namespace {

struct RParams {
    const void* logits;
    uint64_t ld;
    uint32_t T, E, k, all;
    int32_t* experts;
    float* gates;
    int32_t* offsets;
    int32_t* order;
    int32_t* slots;
    uint32_t* counts;                 // [blocks, E]
    uint32_t* totals;                 // [E], behind them
    uint32_t blocks;
    uint32_t block0;                  // of the launch, where the choice takes several
    uint32_t bits;                    // of E: those that an expert's number can have, and of -1 as E
};

template <uint32_t DT>
__device__ __forceinline__ float element(const void* x, uint64_t at) {
    if (DT == QESGD_F32) return ((const float*)x)[at];
    if (DT == QESGD_BF16) return __uint_as_float((uint32_t)((const unsigned short*)x)[at] << 16);
    return (float)((const _Float16*)x)[at];
}

// A logit as the choice compares it: a NaN as infinity.
__device__ __forceinline__ float compared(float v) { return __builtin_fminf(v, INFINITY); }

// Over L lanes (8 .. 64): each step combines halves that hold the same number, so mirrors do for the middle ones.
template <int L, class F>
__device__ __forceinline__ uint32_t over_lanes(uint32_t v, F f) {
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
    v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));       // row_half_mirror
    if (L >= 16) v = f(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));   // row_mirror
    if (L >= 32) { const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false); v = f(r[0], r[1]); }
    if (L >= 64) { const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false); v = f(r[0], r[1]); }
    return v;
}
__device__ __forceinline__ float larger(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }            // of numbers that are none of them NaN
template <int L>
__device__ __forceinline__ float most(float v) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(larger(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int L>
__device__ __forceinline__ uint32_t least(uint32_t v) { return over_lanes<L>(v, [](uint32_t a, uint32_t b) { return min(a, b); }); }
template <int L>
__device__ __forceinline__ float total(float v) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// exp(x) for x <= 0 (a NaN: NaN), 0 below 2^-126: by x log2(e) and that product's rest, right to two steps whatever x.
__device__ __forceinline__ float exp_below(float x) {
    const float high = x * 1.44269504f;
    const float rest = __builtin_fmaf(x, 1.925963033e-8f, __builtin_fmaf(x, 1.44269504f, -high));
    const float r = __builtin_amdgcn_exp2f(high);
    return x < -104.0f ? 0.0f : __builtin_fmaf(r, rest * 0.693147181f, r);       // also -infinity, which has no rest
}

// A token's logits, expert c * L + l, from element `from` on; behind the last one as closed ones.  All are loaded without asking, the last one more than once.
template <uint32_t DT, int L, int C>
__device__ __forceinline__ void load_logits(const void* x, uint64_t from, uint32_t E, uint32_t l, float (&v)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = element<DT>(x, from + min((uint32_t)c * L + l, E - 1u));
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = (uint32_t)c * L + l < E ? compared(v[c]) : -INFINITY;
}

// One token in L lanes, C logits each: expert c * L + l.  Lane j of them (j < k) ends with choice j in `expert` (-1: none) and `gate`.
template <uint32_t DT, int L, int C>
__device__ __forceinline__ void choose(const RParams& p, uint64_t t, uint32_t l, int32_t& expert, float& gate) {
    float v[C];
    load_logits<DT, L, C>(p.logits, t * p.ld, p.E, l, v);
    // In pairs, the larger first (of equals the lower expert): a choice looks for its expert among the larger ones only, and brings up the other one of the pair. From ten logits a
    // lane on: 160001 tokens of 257 experts, six each, 77.5 -> 74.6 us, 20001 of 1024, eight, 64 -> 56; 65536 of 128, four, 22.4 -> 22.8.
    constexpr bool PAIRS = C >= 10;
    constexpr int P = PAIRS ? (C + 1) / 2 : C;
    float first[P], second[P];
    uint32_t swapped = 0;                                      // bit q: the larger one of pair q is the latter
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if constexpr (PAIRS) {
            const float a = v[2 * q], b = 2 * q + 1 < C ? v[2 * q + 1] : -INFINITY;
            const bool swap = b > a;
            first[q] = swap ? b : a;
            second[q] = swap ? a : b;
            swapped |= swap ? 1u << q : 0u;
        } else {
            first[q] = v[q];
            second[q] = -INFINITY;
        }
    }
    const auto largest = [&] {
        float best = first[0];
#pragma unroll
        for (int q = 1; q < P; ++q) best = larger(first[q], best);
        return most<L>(best);
    };
    float high = largest();
    const float base = high;                                   // of infinity: every gate is NaN, as infinity - infinity is
    float sum = 0.0f;
    if (p.all) {
#pragma unroll
        for (int c = 0; c < C; ++c) sum += exp_below(v[c] - base);
    }
    float mine = -INFINITY;
    uint32_t mine_e = 0xFFFFFFFFu;
    for (uint32_t j = 0;;) {
        // the lowest expert among the largest
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int q = P - 1; q >= 0; --q) at = first[q] == high ? (PAIRS ? (uint32_t)q : (uint32_t)q * L + l) : at;
        if (PAIRS) at = at < 32 ? (2u * at + (swapped >> at & 1u)) * L + l : at;
        const uint32_t e = least<L>(at);
        if (l == j && high > -INFINITY) { mine = high; mine_e = e; }
        if (++j >= p.k) break;
        if constexpr (PAIRS) {
            const uint32_t gone = at == e ? e / L / 2u : 32u;  // only in the lane that has it
#pragma unroll
            for (int q = 0; q < P; ++q) {
                first[q] = gone == (uint32_t)q ? second[q] : first[q];
                second[q] = gone == (uint32_t)q ? -INFINITY : second[q];
            }
            swapped ^= gone < 32 ? 1u << gone : 0u;
        } else {
#pragma unroll
            for (int q = 0; q < P; ++q) first[q] = (uint32_t)q * L + l == e ? -INFINITY : first[q];
        }
        high = largest();
    }
    const bool open = mine > -INFINITY;
    const float part = open ? exp_below(mine - base) : 0.0f;
    sum = total<L>(p.all ? sum : part);
    expert = (int32_t)mine_e;
    gate = open ? part / sum : 0.0f;
}

// Blocks of 64 tokens, all at once where 16 lanes take one; a wave that takes many in turn waits for each one's logits.  With 4 / 8 / 16 waves a block, both launches: 8192
// tokens of 64 experts 9.0 / 8.0 / 7.7 us, 160001 of 257 75 / 73 / 75.  From 20 logits a lane on, of whose registers a CU has room for 16 waves of 64 lanes but not for two such
// blocks: 80001 tokens of 512 experts bf16 64 / 62 / 116 us, 20001 of 1024 f32 63 / 56 / 58.
constexpr uint32_t kBlockTokens = 64;
constexpr uint32_t choose_waves(int c) { return c < 20 ? 16 : 8; }

// The choices of a block of tokens and how many pairs each expert has there.
template <uint32_t DT, int L, int C>
__global__ void __launch_bounds__(choose_waves(C) * 64) k_route_choose(const RParams p) {
    constexpr uint32_t kChooseWaves = choose_waves(C);
    __shared__ uint32_t count[QESGD_MAX_EXPERTS];
    for (uint32_t e = threadIdx.x; e < p.E; e += kChooseWaves * 64u) count[e] = 0u;
    __syncthreads();
    const uint32_t l = threadIdx.x & (L - 1u), part = threadIdx.x / L;
    const uint32_t block = p.block0 + blockIdx.x, first = block * kBlockTokens, n = min(kBlockTokens, p.T - first);
    // every part of a wave makes as many turns: the exchanges between lanes are the whole wave's
    for (uint32_t i = part; i < ((n + 64u / L - 1u) & ~(64u / L - 1u)); i += kChooseWaves * 64u / L) {
        const uint64_t t = first + min(i, n - 1u);
        int32_t expert;
        float gate;
        choose<DT, L, C>(p, t, l, expert, gate);
        if (i < n && l < p.k) {
            p.experts[t * p.k + l] = expert;
            p.gates[t * p.k + l] = gate;
            if (expert >= 0) atomicAdd(&count[expert], 1u);
        }
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < p.E; e += kChooseWaves * 64u) p.counts[(uint64_t)block * p.E + e] = count[e];
}

// Many blocks: counts[block, e] becomes the pairs of e in the blocks before, totals[e] those of all.  A workgroup has four experts, a thread a stretch
// of blocks of one of them.
constexpr uint32_t kScanExperts = 4, kScanParts = 256;
__global__ void __launch_bounds__(kScanExperts * kScanParts) k_route_scan(const RParams p) {
    __shared__ uint32_t sums[kScanExperts * kScanParts / 64][kScanExperts];
    const uint32_t col = threadIdx.x % kScanExperts, part = threadIdx.x / kScanExperts;
    const uint32_t e = blockIdx.x * kScanExperts + col;
    const uint32_t length = (p.blocks + kScanParts - 1u) / kScanParts, from = part * length, to = min(from + length, p.blocks);
    uint32_t sum = 0;
    if (e < p.E)
#pragma unroll 8
        for (uint32_t b = from; b < to; ++b) sum += p.counts[(uint64_t)b * p.E + e];
    // over the parts: a wave has 16 of each expert, 4 lanes apart
    uint32_t behind = sum;
#pragma unroll
    for (uint32_t d = kScanExperts; d < 64u; d *= 2) {
        const uint32_t v = __shfl_up(behind, d);
        if ((threadIdx.x & 63u) >= d) behind += v;
    }
    const uint32_t wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63u) >= 64u - kScanExperts) sums[wave][col] = behind;
    __syncthreads();
    uint32_t before = behind - sum;
    for (uint32_t w = 0; w < wave; ++w) before += sums[w][col];
    if (e >= p.E) return;
    if (part == kScanParts - 1u) p.totals[e] = before + sum;
    for (uint32_t b0 = from; b0 < to; b0 += 8u) {
        uint32_t c[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) c[i] = b0 + i < to ? p.counts[(uint64_t)(b0 + i) * p.E + e] : 0u;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (b0 + i < to) p.counts[(uint64_t)(b0 + i) * p.E + e] = before;
            before += c[i];
        }
    }
}

// The lanes whose expert is this lane's.
__device__ __forceinline__ uint64_t alike(uint32_t e, uint32_t bits) {
    uint64_t same = ~0ull;
    for (uint32_t b = 0; b < bits; ++b) {
        const bool one = e >> b & 1u;
        const uint64_t ones = __ballot(one);
        same &= one ? ones : ~ones;
    }
    return same;
}

// The n pairs of a block, from `first` on, in WAVES waves' shares of up to TURNS * 64: order and slots.  expert[i]: that of pair share * wave + i * 64 + lane, -1 for
// none.  whole [E]: each expert's pairs in all blocks; at [WAVES, E]: at[0] those in the blocks before this one, the rest 0.  Only the
// first block writes the offsets.
template <uint32_t WAVES, uint32_t TURNS>
__device__ __forceinline__ void place(const RParams& p, uint64_t first, uint32_t n, uint32_t share, const int32_t (&expert)[TURNS], const uint32_t* whole, uint32_t* at,
                                      uint32_t* waves) {
    constexpr uint32_t threads = WAVES * 64u;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    // pairs of every wave but the last, counted one wave further on, where their number is wanted
    if (wave + 1u < WAVES) {
#pragma unroll
        for (uint32_t i = 0; i < TURNS; ++i)
            if (expert[i] >= 0) atomicAdd(&at[(wave + 1u) * p.E + expert[i]], 1u);
    }
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t base = 0; base < p.E; base += threads) {
        const uint32_t e = base + threadIdx.x, own = e < p.E ? whole[e] : 0u;
        const uint32_t behind = wave_prefix(own);
        if (lane == 63u) waves[wave] = behind;
        __syncthreads();
        uint32_t add = before;
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) add += w < wave ? waves[w] : 0u;
        if (e < p.E) {
            uint32_t to = add + behind - own;
            if (blockIdx.x == 0) p.offsets[e] = (int32_t)to;
            uint32_t mine[WAVES];
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) mine[w] = at[w * p.E + e];
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) {
                to += mine[w];
                at[w * p.E + e] = to;
            }
        }
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) before += waves[w];
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = (int32_t)before;
    volatile uint32_t* own = at + wave * p.E;
#pragma unroll
    for (uint32_t t = 0; t < TURNS; ++t) {
        const uint32_t i = wave * share + t * 64u + lane, e = expert[t] < 0 ? p.E : (uint32_t)expert[t];
        if (wave * share + t * 64u >= n || t * 64u >= share) break;      // uniform
        const uint64_t same = alike(e, p.bits);
        const uint32_t earlier = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
        uint32_t slot = 0;
        if (expert[t] >= 0) slot = own[e] + earlier;
        // the wave's reads are done before its first lane of each expert moves the place on: one wave's LDS operations stay in order
        __builtin_amdgcn_wave_barrier();
        if (expert[t] >= 0 && earlier == 0) own[e] = slot + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (i < n && t * 64u + lane < share) {
            p.slots[first + i] = expert[t] < 0 ? -1 : (int32_t)slot;
            if (expert[t] >= 0) p.order[slot] = (int32_t)(first + i);
        }
    }
}
// A wave's share of n pairs, in whole turns.
template <uint32_t WAVES>
__device__ __forceinline__ uint32_t share_of(uint32_t n) { return (((n + WAVES - 1u) / WAVES) + 63u) & ~63u; }

constexpr uint64_t kRouteScan = 64;
constexpr uint32_t kPlaceWaves = 4, kPlaceTurns = kBlockTokens * QESGD_MAX_CHOICES / (kPlaceWaves * 64);

// A block's pairs to their places.  SCANNED: counts holds what k_route_scan makes of it; otherwise every workgroup adds up the blocks for itself, its
// threads dealt to experts and blocks.
template <bool SCANNED>
__global__ void __launch_bounds__(kPlaceWaves * 64) k_route_place(const RParams p) {
    extern __shared__ uint32_t shared[];
    constexpr uint32_t threads = kPlaceWaves * 64u;
    uint32_t* at = shared;                                   // [waves, E]
    uint32_t* whole = shared + kPlaceWaves * p.E;            // [E]
    uint32_t* waves = whole + p.E;
    const uint32_t first_token = blockIdx.x * kBlockTokens, n = min(kBlockTokens, p.T - first_token) * p.k, share = share_of<kPlaceWaves>(n);
    const uint64_t first = (uint64_t)first_token * p.k;
    int32_t expert[kPlaceTurns];
#pragma unroll
    for (uint32_t t = 0; t < kPlaceTurns; ++t) {
        const uint32_t i = (threadIdx.x >> 6) * share + t * 64u + (threadIdx.x & 63u);
        expert[t] = t * 64u < share && i < n ? p.experts[first + i] : -1;
    }
    for (uint32_t i = threadIdx.x; i < kPlaceWaves * p.E; i += threads)
        at[i] = SCANNED && i < p.E ? p.counts[(uint64_t)blockIdx.x * p.E + i] : 0u;
    for (uint32_t e = threadIdx.x; e < p.E; e += threads) whole[e] = SCANNED ? p.totals[e] : 0u;
    __syncthreads();
    if (!SCANNED) {
        uint32_t across = 4;
        while (across < p.E && across < threads) across *= 2;
        const uint32_t part = threadIdx.x / across, parts = threads / across;
        for (uint32_t e = threadIdx.x % across; e < p.E; e += across) {
            uint32_t sum = 0, before = 0;
            for (uint32_t b0 = part; b0 < p.blocks; b0 += 32u * parts) {
                uint32_t c[32];
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i) c[i] = b0 + i * parts < p.blocks ? p.counts[(uint64_t)(b0 + i * parts) * p.E + e] : 0u;
#pragma unroll
                for (uint32_t i = 0; i < 32; ++i) {
                    before += b0 + i * parts < blockIdx.x ? c[i] : 0u;
                    sum += c[i];
                }
            }
            if (sum) atomicAdd(&whole[e], sum);
            if (before) atomicAdd(&at[e], before);
        }
        __syncthreads();
    }
    place<kPlaceWaves, kPlaceTurns>(p, first, n, share, expert, whole, at, waves);
}

// All of it in one workgroup, for the next tokens of some sequences.
constexpr uint32_t kSmallWaves = 16, kSmallPairs = 2048;
template <uint32_t DT, int L, int C>
__global__ void __launch_bounds__(kSmallWaves * 64) k_route_small(const RParams p) {
    extern __shared__ uint32_t shared[];
    constexpr uint32_t threads = kSmallWaves * 64u;
    __shared__ int32_t experts[kSmallPairs];
    uint32_t* at = shared;                                   // [waves, E]
    uint32_t* whole = shared + kSmallWaves * p.E;            // [E]
    uint32_t* waves = whole + p.E;
    for (uint32_t i = threadIdx.x; i < (kSmallWaves + 1u) * p.E; i += threads) shared[i] = 0u;
    __syncthreads();
    const uint32_t l = threadIdx.x & (L - 1u), part = threadIdx.x / L;
    for (uint32_t i = part; i < ((p.T + 64u / L - 1u) & ~(64u / L - 1u)); i += threads / L) {
        const uint64_t t = min(i, p.T - 1u);
        int32_t expert;
        float gate;
        choose<DT, L, C>(p, t, l, expert, gate);
        if (i < p.T && l < p.k) {
            p.experts[t * p.k + l] = expert;
            p.gates[t * p.k + l] = gate;
            experts[t * p.k + l] = expert;
            if (expert >= 0) atomicAdd(&whole[expert], 1u);
        }
    }
    __syncthreads();
    const uint32_t n = p.T * p.k, share = share_of<kSmallWaves>(n);
    int32_t expert[kSmallPairs / threads];
#pragma unroll
    for (uint32_t t = 0; t < kSmallPairs / threads; ++t) {
        const uint32_t i = (threadIdx.x >> 6) * share + t * 64u + (threadIdx.x & 63u);
        expert[t] = t * 64u < share && i < n ? experts[i] : -1;
    }
    place<kSmallWaves, kSmallPairs / threads>(p, 0, n, share, expert, whole, at, waves);
}

// Gradient of the gates.
struct BParams {
    const void* logits;
    uint64_t ld, ld_d;
    uint32_t T, E, k, all;
    const int32_t* experts;
    const float* gates;
    const float* dgates;
    void* dlogits;
    uint32_t block0;                  // of the launch, where there are several
};

template <uint32_t DT, int L, int C>
__global__ void __launch_bounds__(256) k_route_backward(const BParams p) {
    const uint32_t l = threadIdx.x & (L - 1u);
    const uint64_t i = (uint64_t)(p.block0 + blockIdx.x) * (256u / L) + threadIdx.x / L;
    const uint64_t t = min(i, (uint64_t)p.T - 1u);
    int32_t expert = -1;
    float g = 0.0f, d = 0.0f;
    if (l < p.k) {
        expert = p.experts[t * p.k + l];
        g = p.gates[t * p.k + l];
        d = p.dgates[t * p.k + l];
    }
    const bool there = expert >= 0 && (uint32_t)expert < p.E;
    const float gd = there ? g * d : 0.0f, s = total<L>(gd);
    float x[C], add[C];
#pragma unroll
    for (int c = 0; c < C; ++c) add[c] = 0.0f;
    for (uint32_t j = 0; j < p.k; ++j) {
        // choice j lies in lane j of the token's lanes
        const uint32_t from = (threadIdx.x & 63u & ~(L - 1u)) + j;
        const int32_t e = __shfl(there ? expert : -1, (int)from);
        const float v = __shfl(p.all ? gd : g * (d - s), (int)from);
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (e == c * L + (int32_t)l) add[c] += v;
    }
    if (p.all) {
        float high = -INFINITY;
        load_logits<DT, L, C>(p.logits, t * p.ld, p.E, l, x);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            high = larger(x[c], high);
        }
        high = most<L>(high);
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            // closed is 0, also where all are, and marked by its sign: an open one may be 0 too, and has a NaN where the token's gates are
            x[c] = x[c] == -INFINITY ? -0.0f : exp_below(x[c] - high);
            sum += x[c];
        }
        sum = total<L>(sum);
        const float part = s / sum;
#pragma unroll
        for (int c = 0; c < C; ++c) add[c] -= __float_as_uint(x[c]) == 0x80000000u ? 0.0f : x[c] * part;
    }
    if (i >= p.T) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const uint32_t e = (uint32_t)c * L + l;
        if (e < p.E) put<DT>(p.dlogits, t * p.ld_d + e, add[c]);
    }
}

// f(lanes of a token, logits of a lane): few lanes, because the exchanges between them cost the same for one token or four, and hardly more logits than
// there are.  wide: more lanes from 320 experts on, whose loads and stores of 32 bits take whole lines: gradient of 40001 x 512 f32 28.5 us, with 16 lanes 32.9; but 80001 x
// 512 bf16 73 and 51, and the choice 120 and 62.
template <class F>
void by_experts(uint32_t E, bool wide, F&& f) {
    using std::integral_constant;
#define QESGD_LANES(lanes, each) if (E <= lanes * each) return f(integral_constant<int, lanes>{}, integral_constant<int, each>{})
    QESGD_LANES(8, 1);
    QESGD_LANES(16, 1);
    QESGD_LANES(16, 2);
    QESGD_LANES(16, 3);
    QESGD_LANES(16, 4);
    QESGD_LANES(16, 5);
    QESGD_LANES(16, 6);
    QESGD_LANES(16, 8);
    QESGD_LANES(16, 10);
    QESGD_LANES(16, 12);
    QESGD_LANES(16, 14);
    QESGD_LANES(16, 17);
    QESGD_LANES(16, 20);
    if (wide) {
        QESGD_LANES(32, 12);
        QESGD_LANES(32, 16);
        QESGD_LANES(64, 10);
        QESGD_LANES(64, 12);
        QESGD_LANES(64, 16);
    }
    QESGD_LANES(16, 24);
    QESGD_LANES(16, 32);
    QESGD_LANES(32, 20);
    QESGD_LANES(32, 24);
    QESGD_LANES(32, 32);
#undef QESGD_LANES
}

// Where one workgroup does all of it: up to two tokens for every 16 lanes.  256 tokens of 64 experts, 8 each, took 14.3 us so and 9.0 us in two launches.
bool route_small(uint64_t T, uint32_t E, uint32_t k) { return T * k <= kSmallPairs && T <= 128; }
uint64_t route_blocks(uint64_t T) { return (T + kBlockTokens - 1) / kBlockTokens; }
// Where every block would have to add up the counts of so many that its threads make more than two turns of 32.
bool route_scanned(uint64_t blocks, uint32_t E) {
    uint64_t across = 4;
    while (across < E && across < kPlaceWaves * 64) across *= 2;
    return blocks * across * ((E + across - 1) / across) > kRouteScan * kPlaceWaves * 64;
}

}  // namespace

size_t route_workspace(uint64_t T, uint32_t E, uint32_t k) {
    if (route_small(T, E, k)) return 0;
    return (route_blocks(T) + 1) * E * sizeof(uint32_t);
}

int launch_route(const Route& a) {
    RParams p{};
    p.logits = a.logits;
    p.ld = a.ld;
    p.T = (uint32_t)a.T;
    p.E = a.E;
    p.k = a.k;
    p.all = a.all;
    p.experts = a.experts;
    p.gates = a.gates;
    p.offsets = a.offsets;
    p.order = a.order;
    p.slots = a.slots;
    while ((1u << p.bits) <= a.E) ++p.bits;
    if (route_small(a.T, a.E, a.k)) {
        by_type(a.dtype, [&](auto t) {
            by_experts(a.E, false, [&](auto l, auto c) {
                k_route_small<t.value, l.value, c.value><<<1, kSmallWaves * 64, ((kSmallWaves + 1) * a.E + kSmallWaves) * sizeof(uint32_t), a.stream>>>(p);
            });
        });
        return launched();
    }
    p.counts = a.workspace;
    p.blocks = (uint32_t)route_blocks(a.T);
    p.totals = p.counts + (uint64_t)p.blocks * a.E;
    int rc = QESGD_OK;
    by_type(a.dtype, [&](auto t) {
        by_experts(a.E, false, [&](auto l, auto c) {
            constexpr uint32_t threads = choose_waves(c.value) * 64;
            rc = by_launches(p.blocks, threads, [&](uint32_t first, uint32_t count) {
                p.block0 = first;
                k_route_choose<t.value, l.value, c.value><<<count, threads, 0, a.stream>>>(p);
            });
        });
    });
    if (rc != QESGD_OK) return rc;
    const uint32_t lds = ((kPlaceWaves + 1) * a.E + kPlaceWaves) * sizeof(uint32_t);
    if (route_scanned(p.blocks, a.E)) {
        k_route_scan<<<(a.E + kScanExperts - 1) / kScanExperts, kScanExperts * kScanParts, 0, a.stream>>>(p);
        if (rc = launched(); rc != QESGD_OK) return rc;
        k_route_place<true><<<p.blocks, kPlaceWaves * 64, lds, a.stream>>>(p);
    } else {
        k_route_place<false><<<p.blocks, kPlaceWaves * 64, lds, a.stream>>>(p);
    }
    return launched();
}

int launch_route_backward(const RouteBackward& a) {
    BParams p{};
    p.logits = a.logits;
    p.ld = a.ld;
    p.ld_d = a.ld_d;
    p.T = (uint32_t)a.T;
    p.E = a.E;
    p.k = a.k;
    p.all = a.all;
    p.experts = a.experts;
    p.gates = a.gates;
    p.dgates = a.dgates;
    p.dlogits = a.dlogits;
    int rc = QESGD_OK;
    by_type(a.dtype, [&](auto t) {
        by_experts(a.E, t.value == QESGD_F32, [&](auto l, auto c) {
            rc = by_launches((a.T + 256 / l.value - 1) / (256 / l.value), 256, [&](uint32_t first, uint32_t count) {
                p.block0 = first;
                k_route_backward<t.value, l.value, c.value><<<count, 256, 0, a.stream>>>(p);
            });
        });
    });
    return rc;
}

}  // namespace qesgd
