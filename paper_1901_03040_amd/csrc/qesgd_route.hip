// The router of a layer of experts: each token's k largest logits and their softmax, and the (token, choice) pairs sorted by expert.
//
//   p_e = exp(l_e - max l) / sum_i exp(l_i - max l);  gates: p at the chosen, or their share of the chosen ones' sum
//   place of a pair = pairs of lower experts + earlier pairs of its expert
//
// A token's logits lie in the registers of a part of a wave; the largest is found k times, ties by the lower number.  The sort counts: every block of
// tokens counts its pairs by expert, the counts of the blocks before a block and of the experts before an expert give each block its
// first places, and inside a block a pair finds the earlier ones of its expert by comparing the bits of the experts' numbers across the wave.  Only
// integers are counted, so the result is the same however the work falls.
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
    uint32_t block_tokens, blocks;
    uint32_t bits;                    // of E: those that an expert's number can have, and of -1 as E
};

template <uint32_t DT>
__device__ __forceinline__ float element(const void* x, uint64_t at) {
    if (DT == QESGD_F32) return ((const float*)x)[at];
    if (DT == QESGD_BF16) return __uint_as_float((uint32_t)((const unsigned short*)x)[at] << 16);
    return (float)((const _Float16*)x)[at];
}
template <uint32_t DT>
__device__ __forceinline__ void put_element(void* x, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)x)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)x)[at] = (_Float16)v;
    else ((__bf16*)x)[at] = (__bf16)v;
}

// Order of logits as integers: 0 for a closed expert, a NaN above all, the two zeros alike.
__device__ __forceinline__ uint32_t rank_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    if (v != v) return 0xFFFFFFFFu;
    if (b == 0xFF800000u) return 0u;
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t rank) { return __uint_as_float(rank & 0x80000000u ? rank ^ 0x80000000u : ~rank); }

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
template <int L>
__device__ __forceinline__ uint32_t most(uint32_t v) { return over_lanes<L>(v, [](uint32_t a, uint32_t b) { return max(a, b); }); }
template <int L>
__device__ __forceinline__ uint32_t least(uint32_t v) { return over_lanes<L>(v, [](uint32_t a, uint32_t b) { return min(a, b); }); }
template <int L>
__device__ __forceinline__ float total(float v) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// One token in L lanes, C logits each: expert c * L + l.  Lane j of them (j < k) ends with choice j in `expert` (-1: none) and `gate`.
template <uint32_t DT, int L, int C>
__device__ __forceinline__ void choose(const RParams& p, uint64_t t, uint32_t l, int32_t& expert, float& gate) {
    uint32_t rank[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const uint32_t e = (uint32_t)c * L + l;
        rank[c] = e < p.E ? rank_of(element<DT>(p.logits, t * p.ld + e)) : 0u;
    }
    uint32_t all_rank[C];
#pragma unroll
    for (int c = 0; c < C; ++c) all_rank[c] = rank[c];
    uint32_t top = 0, mine = 0, mine_e = 0xFFFFFFFFu;
    for (uint32_t j = 0; j < p.k; ++j) {
        uint32_t best = rank[0], at = l;
#pragma unroll
        for (int c = 1; c < C; ++c)
            if (rank[c] > best) { best = rank[c]; at = (uint32_t)c * L + l; }
        const uint32_t high = most<L>(best);
        const uint32_t e = least<L>(best == high ? at : 0xFFFFFFFFu);
        if (j == 0) top = high;
        if (l == j) { mine = high; mine_e = high ? e : 0xFFFFFFFFu; }
#pragma unroll
        for (int c = 0; c < C; ++c)
            if ((uint32_t)c * L + l == e) rank[c] = 0u;
    }
    const float base = logit_of(top);
    const float part = mine ? expf(logit_of(mine) - base) : 0.0f;
    float sum = part;
    if (p.all) {
        sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) sum += all_rank[c] ? expf(logit_of(all_rank[c]) - base) : 0.0f;
    }
    sum = total<L>(sum);
    expert = (int32_t)mine_e;
    gate = mine ? part / sum : 0.0f;
}

constexpr uint32_t kChooseWaves = 4;

// The choices of a block of tokens and how many pairs each expert has there.
template <uint32_t DT, int L, int C>
__global__ void __launch_bounds__(kChooseWaves * 64) k_route_choose(const RParams p) {
    __shared__ uint32_t count[QESGD_MAX_EXPERTS];
    for (uint32_t e = threadIdx.x; e < p.E; e += kChooseWaves * 64u) count[e] = 0u;
    __syncthreads();
    const uint32_t l = threadIdx.x & (L - 1u), part = threadIdx.x / L;
    const uint32_t first = blockIdx.x * p.block_tokens, n = min(p.block_tokens, p.T - first);
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
    for (uint32_t e = threadIdx.x; e < p.E; e += kChooseWaves * 64u) p.counts[(uint64_t)blockIdx.x * p.E + e] = count[e];
}

constexpr uint32_t kPlaceWaves = 4;

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

// Pairs first .. first + n of the block, wave w's share of them in order: order and slots.  at [waves, E]: the first places of each wave's.
__device__ __forceinline__ void place(const RParams& p, uint64_t first, uint32_t n, uint32_t share, uint32_t* at) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    volatile uint32_t* own = at + wave * p.E;
    const uint32_t from = wave * share, to = min(from + share, n);
    for (uint32_t i0 = from; i0 < to; i0 += 64u) {
        const uint32_t i = i0 + lane;
        const int32_t expert = i < to ? p.experts[first + i] : -1;
        const uint32_t e = expert < 0 ? p.E : (uint32_t)expert;
        const uint64_t same = alike(e, p.bits);
        const uint32_t earlier = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
        uint32_t to_place = 0;
        if (expert >= 0) to_place = own[e] + earlier;
        // the wave's reads are done before its first lane of each expert moves the place on: one wave's LDS operations stay in order
        __builtin_amdgcn_wave_barrier();
        if (expert >= 0 && earlier == 0) own[e] = to_place + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (i < to) {
            p.slots[first + i] = expert < 0 ? -1 : (int32_t)to_place;
            if (expert >= 0) p.order[to_place] = (int32_t)(first + i);
        }
    }
}

// counts [blocks, E] holds each block's pairs; every workgroup adds up the blocks before it, and all of them for the experts' first places.
__global__ void __launch_bounds__(kPlaceWaves * 64) k_route_place(const RParams p) {
    extern __shared__ uint32_t shared[];
    constexpr uint32_t threads = kPlaceWaves * 64u;
    uint32_t* at = shared;                                   // [waves, E]
    uint32_t* whole = shared + kPlaceWaves * p.E;            // [E]: of all blocks
    uint32_t* waves = whole + p.E;
    for (uint32_t e = threadIdx.x; e < p.E; e += threads) {
        uint32_t sum = 0, before = 0;
#pragma unroll 8
        for (uint32_t b = 0; b < p.blocks; ++b) {
            const uint32_t c = p.counts[(uint64_t)b * p.E + e];
            before += b < blockIdx.x ? c : 0u;
            sum += c;
        }
        whole[e] = sum;
        at[e] = before;
        for (uint32_t w = 1; w < kPlaceWaves; ++w) at[w * p.E + e] = 0u;
    }
    __syncthreads();
    const uint32_t first_token = blockIdx.x * p.block_tokens, n = min(p.block_tokens, p.T - first_token) * p.k;
    const uint64_t first = (uint64_t)first_token * p.k;
    const uint32_t share = (((n + kPlaceWaves - 1u) / kPlaceWaves) + 63u) & ~63u;
    // pairs of every wave but the last, counted one wave further on, where their number is wanted
    for (uint32_t i = threadIdx.x; i < n; i += threads) {
        const uint32_t w = i / share + 1u;
        const int32_t expert = p.experts[first + i];
        if (w < kPlaceWaves && expert >= 0) atomicAdd(&at[w * p.E + expert], 1u);
    }
    __syncthreads();
    // experts' first places; only the first workgroup writes them out
    uint32_t pairs = 0;
    {
        uint32_t before = 0;
        for (uint32_t base = 0; base < p.E; base += threads) {
            const uint32_t e = base + threadIdx.x, own = e < p.E ? whole[e] : 0u;
            const uint32_t behind = wave_prefix(own);
            if ((threadIdx.x & 63u) == 63u) waves[threadIdx.x >> 6] = behind;
            __syncthreads();
            uint32_t add = before;
            for (uint32_t w = 0; w < threadIdx.x >> 6; ++w) add += waves[w];
            if (e < p.E) {
                uint32_t place = add + behind - own;
                if (blockIdx.x == 0) p.offsets[e] = (int32_t)place;
                for (uint32_t w = 0; w < kPlaceWaves; ++w) {
                    place += at[w * p.E + e];
                    at[w * p.E + e] = place;
                }
            }
            for (uint32_t w = 0; w < kPlaceWaves; ++w) before += waves[w];
            __syncthreads();
        }
        pairs = before;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = (int32_t)pairs;
    place(p, first, n, share, at);
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
};

template <uint32_t DT, int L, int C>
__global__ void __launch_bounds__(256) k_route_backward(const BParams p) {
    const uint32_t l = threadIdx.x & (L - 1u);
    const uint64_t i = (uint64_t)blockIdx.x * (256u / L) + threadIdx.x / L;
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
        float top = -INFINITY;
        uint32_t high = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint32_t e = (uint32_t)c * L + l;
            x[c] = e < p.E ? element<DT>(p.logits, t * p.ld + e) : -INFINITY;
            high = max(high, rank_of(x[c]));
        }
        high = most<L>(high);
        top = logit_of(high);
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[c] = x[c] == -INFINITY ? 0.0f : expf(x[c] - top);
            sum += x[c];
        }
        sum = total<L>(sum);
#pragma unroll
        for (int c = 0; c < C; ++c) add[c] -= x[c] == 0.0f ? 0.0f : x[c] / sum * s;
    }
    if (i >= p.T) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const uint32_t e = (uint32_t)c * L + l;
        if (e < p.E) put_element<DT>(p.dlogits, t * p.ld_d + e, add[c]);
    }
}

// f(lanes of a token, logits of a lane): the least room for E logits.
template <class F>
void by_experts(uint32_t E, F&& f) {
    using std::integral_constant;
    if (E <= 8) f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (E <= 16) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (E <= 32) f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    else if (E <= 64) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (E <= 128) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    else if (E <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (E <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

uint32_t route_block_tokens(uint64_t T, uint32_t E) {
    uint64_t blocks = (T + 63) / 64;
    if (blocks > 256) blocks = 256;
    return (uint32_t)((T + blocks - 1) / blocks);
}

}  // namespace

size_t route_workspace(uint64_t T, uint32_t E, uint32_t k) {
    const uint64_t tokens = route_block_tokens(T, E);
    return ((T + tokens - 1) / tokens) * E * sizeof(uint32_t);
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
    p.counts = a.workspace;
    p.block_tokens = route_block_tokens(a.T, a.E);
    p.blocks = (p.T + p.block_tokens - 1) / p.block_tokens;
    while ((1u << p.bits) <= a.E) ++p.bits;
    by_type(a.dtype, [&](auto t) {
        by_experts(a.E, [&](auto l, auto c) { k_route_choose<t.value, l.value, c.value><<<p.blocks, kChooseWaves * 64, 0, a.stream>>>(p); });
    });
    if (const int rc = launched(); rc != QESGD_OK) return rc;
    k_route_place<<<p.blocks, kPlaceWaves * 64, ((kPlaceWaves + 1) * a.E + kPlaceWaves) * sizeof(uint32_t), a.stream>>>(p);
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
        by_experts(a.E, [&](auto l, auto c) {
            const uint64_t groups = (a.T + 256 / l.value - 1) / (256 / l.value);
            if (!grid_ok(groups, 256)) { rc = QESGD_ERR_DIM; return; }
            k_route_backward<t.value, l.value, c.value><<<(uint32_t)groups, 256, 0, a.stream>>>(p);
        });
    });
    return rc != QESGD_OK ? rc : launched();
}

}  // namespace qesgd
