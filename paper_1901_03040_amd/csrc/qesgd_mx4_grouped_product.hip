// Products of packed 4-bit rows grouped by expert, on the tiles of the product of two matrices.
//
//   C[r, n] = sum_k A[r, k] B_e[n, k] for the rows r of group e        a tile's rows end with its group
//   D_e[n, k] = sum over the rows r of group e of A[r, n] B[r, k]      a tile's contraction is its group's rows
//
// Element products are exact, sums are fp32.
//
// Bound by the matrix units at the power the card allows them: 16 experts of 4096 x 4096, 32768 rows bf16 286 us = 3.8 PFLOP/s; small groups by
// the reading of the experts' matrices and by launches, short contractions by a tile's beginning and by the writing of the result.
#include "qesgd_experts.h"
#include "qesgd_groups.h"
#include "qesgd_mx4_codes.h"
#include "qesgd_mx4_tiles.h"

namespace qesgd {
namespace {

struct PParams {
    const unsigned char* a;
    const unsigned char* b;
    uint64_t a_scales, b_scales, b_stride;
    const int32_t* offsets;
    uint32_t E, R;
    void* c;
    uint64_t ldc;
    uint32_t N, K;                        // rows of B_e; columns of D_e
    uint32_t row_codes, row_scales;       // of either operand
    uint32_t tiles_m, tiles_n;            // of one expert's D; of C, at most: offsets that fall could make more of them than a number holds
    bool stream;                          // C or D in whole lines that nothing finds in a cache again
    uint32_t pieces;                      // of the contraction; with more than one the sums go to partial [pieces, all of C or D]
    float* partial;
    uint64_t sums;                        // of a piece
};

// Non-temporal stores of results made of whole lines (parts of lines cost such a store a read: rows of 2049 numbers 38 -> 50 us): of products where the result is larger than what the
// memory-side cache keeps for its reader, of gradients where their writing out at the kernel's end counts.  Us without / with, and in brackets with the call that reads the result:
// products 16 experts, 32768 rows, N = K = 4096 bf16 312 / 280, 8, 16384, 4096, 4096 134 MB 151 / 151 (181 / 190), 50, 25990, 1024, 576 53 MB 24.8 / 23.2 (39.5 / 41.7), 16,
// 8192, 1024, 1024 17 MB 14.2 / 12.2 (23.2 / 23.0), 49, 3621, 832, 3142 6 MB 20.9 / 20.7 (25.1 / 25.9); gradients 8, 16384, 4096, 4096 251 / 207, 50, 25990, 576, 1024 118 MB
// 47.6 / 46.2 (68.6 / 68.8), 16, 4096, 1024, 1024 67 MB 18.2 / 17.4 (32.8 / 31.9), 4, 996, 320, 3136 16 MB 8.4 / 7.6 (17.9 / 16.5), 8, 2048, 512, 512 8 MB 6.3 / 6.3 (12.4 / 12.5).
constexpr uint64_t kStreamProduct = 192ull << 20, kStreamGradient = 12ull << 20;
inline bool whole_lines(const void* c, uint64_t row_bytes) { return ((uintptr_t)c | row_bytes) % 128 == 0; }

// Four numbers of a row, whose rows begin at any element.
template <uint32_t DT, bool STREAM>
__device__ __forceinline__ void put_four(void* c, uint64_t at, const float (&v)[4]) {
    if constexpr (DT == QESGD_F32) {
        vec4_any* to = (vec4_any*)((float*)c + at);
        const vec4 x = {v[0], v[1], v[2], v[3]};
        if (STREAM) __builtin_nontemporal_store(x, to);
        else *to = x;
    } else {
        typedef uvec2 __attribute__((aligned(2))) uvec2_any;
        uvec2 x;
        if constexpr (DT == QESGD_BF16) x = uvec2{__builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2], (__bf16)v[3]})};
        else x = uvec2{__builtin_bit_cast(uint32_t, f16x2{(_Float16)v[0], (_Float16)v[1]}), __builtin_bit_cast(uint32_t, f16x2{(_Float16)v[2], (_Float16)v[3]})};
        uvec2_any* to = (uvec2_any*)((unsigned short*)c + at);
        if (STREAM) __builtin_nontemporal_store(x, to);
        else *to = x;
    }
}

// B's rows in fours where a wave has two fragments side by side.
template <class S>
using OrderB = std::conditional_t<S::FN == 2, InFours, Straight>;

// The wave's fragments to rows and columns from row0 and col0 on, of rows up to M and columns up to N.  In fours 16 lanes write a row's 64 columns at once: an element a lane took
// four times as many stores, and a wave has 63 on their way.
template <class S, uint32_t DT>
__device__ __forceinline__ void store_tile(const Mx4Ops<S>& ops, void* c, uint64_t ldc, uint32_t M, uint32_t N, uint32_t row0, uint32_t col0, bool stream) {
    const uint32_t lane = threadIdx.x & 63u;
    row0 = __builtin_amdgcn_readfirstlane(row0);
    col0 = __builtin_amdgcn_readfirstlane(col0);
    if (row0 >= M || col0 >= N) return;
    const bool whole = row0 + S::FM * 32u <= M && col0 + S::FN * 32u <= N;
    if constexpr (S::FN == 2) {
        const uint32_t row = row0 + 4u * (lane >> 5) + (lane >> 4 & 1u), col = col0 + 4u * (lane & 15u);
        const uint64_t base = (uint64_t)row * ldc + col;
        const auto four = [&](int i, int e, float (&v)[4]) {
            // rows of 16 lanes exchanged: two columns of one matrix row, from either fragment
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(ops.acc[i][j][e]), __float_as_uint(ops.acc[i][j][e + 1]), false, false);
                v[2 * j] = __uint_as_float(two[0]);
                v[2 * j + 1] = __uint_as_float(two[1]);
            }
        };
        const auto all = [&](auto put) {
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    float v[4];
                    four(i, e, v);
                    put((uint32_t)(i * 32 + 8 * (e >> 2) + (e & 3)), v);
                }
        };
        if (whole && stream) {
            asm volatile("; streamed");              // keeps the two arms apart, which the compiler would merge into ordinary stores
            all([&](uint32_t r, const float (&v)[4]) { put_four<DT, true>(c, base + r * ldc, v); });
        } else if (whole) {
            all([&](uint32_t r, const float (&v)[4]) { put_four<DT, false>(c, base + r * ldc, v); });
        } else if (col0 + 64u <= N || (N - col0) % 4u == 0) {
            all([&](uint32_t r, const float (&v)[4]) {
                if (col < N && row + r < M) put_four<DT, false>(c, base + r * ldc, v);
            });
        } else {
            // a row's last ones are fewer than four: a number a lane, in the columns that its rows of B are
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store_fragment<DT>(c, ldc, M, N, row0 + i * 32u + 4u * (lane >> 5), col + 2u * j + (lane >> 4 & 1u), false, ops.acc[i][j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j)
                // a lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r
                store_fragment<DT>(c, ldc, M, N, row0 + i * 32u + 4u * (lane >> 5), col0 + j * 32u + (lane & 31u), whole, ops.acc[i][j]);
    }
}

// Steps first .. first + count of `steps`, piece number `piece` of them: an even first one, because scales come in pairs.  A short contraction leaves some pieces
// without any.
__device__ __forceinline__ void piece_of(const PParams& p, uint32_t piece, uint32_t steps, uint32_t& first, uint32_t& count) {
    first = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)piece * steps / p.pieces)) & ~1u;
    count = (piece + 1u == p.pieces ? steps : __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)(piece + 1u) * steps / p.pieces)) & ~1u) - first;
}

template <class S>
__device__ __forceinline__ void multiply_tile(Mx4Ops<S>& ops, uint32_t steps, unsigned char* lds0, unsigned char* lds1, unsigned char* lds2, unsigned char* lds3) {
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) ops.acc[i][j] = acc16{};
    if constexpr (S::BUFFERS == 2) {
        unsigned char* const buffers[2] = {lds0, lds1};
        run_steps(ops, steps, buffers);
    } else {
        unsigned char* const buffers[4] = {lds0, lds1, lds2, lds3};
        run_steps(ops, steps, buffers);
    }
}

template <class S, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_mx4_grouped_product(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds2[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char lds3[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char scales[Mx4Ops<S>::scale_buffers * Mx4Ops<S>::scale_bytes];
    constexpr uint32_t lg = S::BM == 64 ? 6 : S::BM == 128 ? 7 : 8;
    static_assert((1 << lg) == S::BM, "tiles of a power of two");
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    // the workgroups that have a tile are dealt to the XCDs among themselves: those behind the last tile come last of all
    const uint32_t all = min(all_tiles(p.offsets, p.E, p.R, Power{lg}), p.tiles_m) * p.tiles_n;
    if (blockIdx.x >= all * p.pieces) return;
    uint32_t t = tile_of_workgroup(blockIdx.x, all * p.pieces), piece = 0, first = 0, steps = (p.row_codes + kStepBytes - 1u) / kStepBytes;
    const uint32_t all_steps = steps;
    if (p.pieces > 1) {
        piece = __builtin_amdgcn_readfirstlane(t / all);
        t -= piece * all;
        piece_of(p, piece, all_steps, first, steps);
    }
    Group g;
    if (!group_of_tile(p.offsets, p.E, p.R, Power{lg}, p.tiles_n, t, g)) return;
    uint32_t tm, tn;
    banded_tile(t - g.first, (g.hi - g.lo + S::BM - 1u) >> lg, p.tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const uint32_t m0 = g.lo + tm * S::BM, n0 = tn * S::BN;
    const unsigned char* b = p.b + g.e * p.b_stride;
    Mx4Ops<S> ops;
    ops.a = p.a + (uint64_t)m0 * p.row_codes + (uint64_t)first * kStepBytes;
    ops.b = b + (uint64_t)n0 * p.row_codes + (uint64_t)first * kStepBytes;
    ops.la.init(p.row_codes, g.hi - m0);
    ops.lb.init(p.row_codes, p.N - n0, OrderB<S>{});
    ops.scales = scales;
    ops.init_scales(p.a + p.a_scales + (uint64_t)m0 * p.row_scales + first * 8u, b + p.b_scales + (uint64_t)n0 * p.row_scales + first * 8u, g.hi - m0, p.N - n0,
                    p.row_scales, p.row_scales - first * 8u, wm, wn, OrderB<S>{});
    ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
    ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
    ops.steps = steps;
    ops.half = p.row_codes % kStepBytes != 0 && first + steps == all_steps;
    ops.h = h;
    multiply_tile(ops, steps, lds0, lds1, lds2, lds3);

    // pieces are of fp32, as DT is for them
    void* c = p.pieces > 1 ? (void*)(p.partial + piece * p.sums) : p.c;
    store_tile<S, DT>(ops, c, p.pieces > 1 ? p.N : p.ldc, g.hi, p.N, m0 + wm * S::FM * 32u, n0 + wn * S::FN * 32u, p.stream);
}

template <class S, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_mx4_grouped_gradient(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds2[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char lds3[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char scales[Mx4Ops<S>::scale_buffers * Mx4Ops<S>::scale_bytes];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    // experts differ in rows, so every XCD gets its share of each one's tiles, a run of them: 8 experts of 4096 x 4096, 16384 rows 357 -> 266 us
    const uint32_t tiles = p.tiles_m * p.tiles_n, e = __builtin_amdgcn_readfirstlane(blockIdx.x / tiles), piece = blockIdx.y;
    uint32_t tm, tn;
    banded_tile(tile_of_workgroup(blockIdx.x - e * tiles, tiles), p.tiles_m, p.tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const Group g = group_number(p.offsets, p.E, p.R, Power{7}, e);
    // bytes of a row's codes before the group and of the group, as far as the rows go
    const uint32_t begin = __builtin_amdgcn_readfirstlane(min(g.first * 64u, p.row_codes));
    const uint32_t bytes = __builtin_amdgcn_readfirstlane(min(((g.hi - g.lo + 127u) >> 7) * 64u, p.row_codes - begin));
    const uint32_t all_steps = (bytes + kStepBytes - 1u) / kStepBytes;
    uint32_t first = 0, steps = all_steps;
    if (p.pieces > 1) piece_of(p, piece, all_steps, first, steps);
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN, from = begin + first * kStepBytes;
    Mx4Ops<S> ops;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) ops.acc[i][j] = acc16{};
    if (steps) {
        ops.a = p.a + (uint64_t)m0 * p.row_codes + from;
        ops.b = p.b + (uint64_t)n0 * p.row_codes + from;
        ops.la.init(p.row_codes, p.N - m0);
        ops.lb.init(p.row_codes, p.K - n0, OrderB<S>{});
        ops.scales = scales;
        ops.init_scales(p.a + p.a_scales + (uint64_t)m0 * p.row_scales + from / 16u, p.b + p.b_scales + (uint64_t)n0 * p.row_scales + from / 16u,
                        p.N - m0, p.K - n0, p.row_scales, (bytes - first * kStepBytes) / 16u, wm, wn, OrderB<S>{});
        ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
        ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
        ops.steps = steps;
        ops.half = bytes % kStepBytes != 0 && first + steps == all_steps;
        ops.h = h;
        multiply_tile(ops, steps, lds0, lds1, lds2, lds3);
    }
    const uint64_t of_expert = (uint64_t)e * p.N * p.K;
    void* d = p.pieces > 1 ? (void*)(p.partial + piece * p.sums + of_expert) : (void*)((unsigned char*)p.c + of_expert * (DT == QESGD_F32 ? 4u : 2u));
    store_tile<S, DT>(ops, d, p.K, p.N, p.K, m0 + wm * S::FM * 32u, n0 + wn * S::FN * 32u, p.stream);
}

// A result from the sums of the pieces, added in order (see PieceSum).  Four numbers a lane where rows allow it, eight pieces on their way: the sums
// come from the memory-side cache and are few, so it is a launch and a latency.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_mx4_piece_sum(const PieceSum p) {
    const uint64_t i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 4u;
    if (i >= p.sums) return;
    uint64_t lo = 0, hi = ~0ull;
    if (p.offsets) {
        lo = held(p.offsets[0], p.R);
        hi = held(p.offsets[p.E], p.R);
    }
    uint64_t row = i / p.cols;
    uint32_t col = (uint32_t)(i - row * p.cols);
    if (row >= hi || row + 3u < lo) return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if ((p.sums & 3u) == 0) {
        for (uint32_t k0 = 0; k0 < p.pieces; k0 += 8) {
            float x[8][4];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) *(float4*)x[k] = *(const float4*)(p.partial + min(k0 + k, p.pieces - 1u) * p.sums + i);
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += k0 + k < p.pieces ? x[k][e] : 0.0f;
        }
    } else {
        for (uint32_t k = 0; k < p.pieces; ++k)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (i + e < p.sums) v[e] += p.partial[k * p.sums + i + e];
    }
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        if (i + e < p.sums && row >= lo && row < hi) put<DT>(p.c, row * p.ldc + col, v[e]);
        if (++col == p.cols) { col = 0; ++row; }
    }
}

// ---- large tiles, one after the other ------------------------------------------
//
// A workgroup takes every gridDim-th tile.  The loads of a tile's first two steps are on their way while the last two of the tile before are multiplied,
// and while that one is stored: a tile of its own workgroup begins with a launch, a search and a trip to memory, 6 us where 16 steps take 33.
// Steps come in pairs, because buffers and scales do: where a tile has an odd number, its last one comes once more with scales of zero.

// Tiles before each group and offsets, in LDS.
struct GroupTable {
    uint32_t first[QESGD_MAX_EXPERTS + 1];
    uint32_t row[QESGD_MAX_EXPERTS + 1];
};
// By the first wave.
__device__ __forceinline__ void fill_table(GroupTable& table, const int32_t* offsets, uint32_t E, uint32_t R, uint32_t lg) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;
    for (uint32_t base = 0; base < E; base += 64u) {
        uint32_t lo, hi;
        const uint32_t behind = before + wave_prefix(group_tiles(offsets, E, R, Power{lg}, base + lane, lo, hi));
        if (base + lane < E) {
            table.first[base + lane + 1u] = behind;
            table.row[base + lane] = lo;
            if (base + lane + 1u == E) table.row[E] = hi;
        }
        before = lane_value(behind, 63u);
    }
    if (lane == 0) table.first[0] = 0;
}
// The group with tile number `tile` of the groups' tiles.  Uniform.
__device__ __forceinline__ uint32_t table_group(const GroupTable& table, uint32_t E, uint32_t tile) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t base = 0;
    for (; base + 64u < E; base += 64u)
        if (tile < (uint32_t)__builtin_amdgcn_readfirstlane((int)table.first[base + 64u])) break;
    const uint64_t found = __ballot(tile < table.first[min(base + lane + 1u, E)]);
    return base + (found ? (uint32_t)__builtin_ctzll(found) : 0u);
}

// What the loads of a tile need beside the operands, and where its result goes.
struct ChainTile {
    uint32_t steps;                       // of 256 columns, the last one maybe half
    bool half;
    uint32_t m0, n0, rows_a, rows_b;
    uint32_t e;
};

template <class S>
struct Mx4Chain : Mx4Ops<S> {
    using B = Mx4Ops<S>;
    uint32_t first;                       // mask of the scales of a step's first half

    __device__ __forceinline__ void aim(const unsigned char* a, const unsigned char* b, const unsigned char* sa, const unsigned char* sb, uint32_t pitch,
                                        uint32_t row_scales, uint32_t bytes, const ChainTile& t, uint32_t wm, uint32_t wn) {
        B::a = a;
        B::b = b;
        B::la.init(pitch, t.rows_a);
        B::lb.init(pitch, t.rows_b, OrderB<S>{});
        B::init_scales(sa, sb, t.rows_a, t.rows_b, row_scales, bytes / 16u, wm, wn, OrderB<S>{});
        B::steps = t.steps;
        B::half = t.half;
    }
    __device__ __forceinline__ void fetch(uint32_t step, unsigned char* to) { B::fetch(min(step, B::steps - 1u), to); }
    __device__ __forceinline__ void fetch_pair(uint32_t step, uint32_t buffer) {
        const uint32_t word = min(step * 8u + (threadIdx.x & 3u) * 4u, B::last_word);
        const uint32_t to = lds_number(B::scales) + buffer * B::scale_bytes + B::scale_at;
#pragma unroll
        for (int i = 0; i < B::NA; ++i) load_to_lds_4(B::sa, B::off_a[i] + word, to + i * S::threads * 4);
#pragma unroll
        for (int i = 0; i < B::NB; ++i) load_to_lds_4(B::sb, B::off_b[i] + word, to + S::BM * 16 + i * S::threads * 4);
    }
    // Step `step` of a tile of `steps`.
    __device__ __forceinline__ void arrive(uint32_t step, uint32_t steps, bool half, uint32_t buffer) {
        const unsigned char* from = B::scales + buffer * B::scale_bytes + (step & 1u) * 8u;
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { const uint2 v = *(const uint2*)(from + B::scale_at_a + f * 512); B::ya[f][0] = v.x; B::ya[f][1] = v.y; }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { const uint2 v = *(const uint2*)(from + B::scale_at_b + f * 512); B::yb[f][0] = v.x; B::yb[f][1] = v.y; }
        first = step < steps ? 0xFFFFFFFFu : 0u;
        B::second = step < steps && !(half && step + 1u == steps) ? 0xFFFFFFFFu : 0u;
    }
    __device__ __forceinline__ void next() {
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { B::xa[f][0] = (B::ya[f][0] & first) >> (8u * B::h); B::xa[f][1] = (B::ya[f][1] & B::second) >> (8u * B::h); }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { B::xb[f][0] = (B::yb[f][0] & first) >> (8u * B::h); B::xb[f][1] = (B::yb[f][1] & B::second) >> (8u * B::h); }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) B::acc[i][j] = acc16{};
    }
};

// advance(tile): aims ops at the workgroup's next tile, false where there is none; finish(tile): stores the sums.
template <class S, class Advance, class Finish>
__device__ __forceinline__ void run_chain(Mx4Chain<S>& ops, unsigned char* const (&lds)[2], Advance&& advance, Finish&& finish) {
    static_assert(S::BUFFERS == 2 && Mx4Chain<S>::scale_buffers == 2, "a tile's buffers take turns");
    constexpr int PARTS = Mx4Ops<S>::PARTS;
    typename Mx4Ops<S>::Frag f[2];
    ChainTile here, there;
    if (!advance(here)) return;
    uint32_t pair = 0;
    ops.fetch(0, lds[0]);
    ops.fetch_pair(0, 0);
    ops.fetch(1, lds[1]);
    ops.clear();
    wait_and_meet<Mx4Ops<S>::LOADS>();
    ops.arrive(0, here.steps, here.half, 0);
    ops.next();
    ops.read(f[0], lds[0], 0);
    // one step of `here`: the step behind it is number `then` of a tile of `steps`, and the loads are those of step `load` of the tile that ops aims at
    const auto step = [&](auto even, uint32_t then, uint32_t steps, bool half, uint32_t load) {
        constexpr bool EVEN = decltype(even)::value;
        asm volatile("" : "+v"(ops.at_a), "+v"(ops.at_b));
#pragma unroll
        for (int p = 0; p + 1 < PARTS; ++p) {
            ops.read(f[(p + 1) & 1], lds[EVEN ? 0 : 1], p + 1);
            ops.multiply(f[p & 1], p);
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_and_meet<0>();
        ops.arrive(then, steps, half, EVEN ? pair : pair ^ 1u);
        ops.fetch(load, lds[EVEN ? 0 : 1]);
        if (EVEN) ops.fetch_pair(load, pair ^ 1u);
        ops.read(f[0], lds[EVEN ? 1 : 0], 0);
        __builtin_amdgcn_sched_barrier(0);
        ops.multiply(f[1], PARTS - 1);
        ops.next();
    };
    for (;;) {
        bool more = false;
        for (uint32_t t = 0; t < here.steps; t += 2) {
            const bool last = t + 2u >= here.steps;
            if (last) more = advance(there);
            const bool on = last && more;              // otherwise the loads behind the end are of this tile's last step again, and nothing uses them
            step(std::true_type{}, t + 1u, here.steps, here.half, on ? 0u : t + 2u);
            step(std::false_type{}, on ? 0u : t + 2u, on ? there.steps : here.steps, on ? there.half : here.half, on ? 1u : t + 3u);
            pair ^= 1u;
        }
        finish(here);
        if (!more) break;
        ops.clear();
        here = there;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): nothing is on its way to LDS when the workgroup ends
}

// GRADIENT: D_e = A_e B_e^T over the columns of group e, tiles of each expert dealt to the XCDs; else C, tiles of the groups' rows.
template <class S, uint32_t DT, bool GRADIENT>
__global__ void __launch_bounds__(S::threads) k_mx4_grouped_chain(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char scales[Mx4Ops<S>::scale_buffers * Mx4Ops<S>::scale_bytes];
    __shared__ GroupTable table;
    constexpr uint32_t lg = GRADIENT ? 7 : S::BM == 64 ? 6 : S::BM == 128 ? 7 : 8;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    if (wave == 0) fill_table(table, p.offsets, p.E, p.R, lg);
    __syncthreads();
    const uint32_t tiles = p.tiles_m * p.tiles_n;
    const uint32_t all = GRADIENT ? tiles * p.E : min((uint32_t)__builtin_amdgcn_readfirstlane((int)table.first[p.E]), p.tiles_m) * p.tiles_n;
    Mx4Chain<S> ops;
    ops.scales = scales;
    ops.h = lane >> 5;
    ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
    ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
    uint32_t v = blockIdx.x;
    const auto place = [&](ChainTile& t, uint32_t& begin, uint32_t& bytes) {
        uint32_t tm, tn;
        if constexpr (GRADIENT) {
            t.e = v / tiles;
            banded_tile(tile_of_workgroup(v - t.e * tiles, tiles), p.tiles_m, p.tiles_n, tm, tn);
            const uint32_t from = (uint32_t)__builtin_amdgcn_readfirstlane((int)table.first[t.e]);
            const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane((int)table.first[t.e + 1u]);
            begin = min(from * 64u, p.row_codes);
            bytes = min((to - from) * 64u, p.row_codes - begin);
            t.m0 = tm * S::BM;
            t.n0 = tn * S::BN;
            t.rows_a = p.N - t.m0;
            t.rows_b = p.K - t.n0;
        } else {
            const uint32_t tile = tile_of_workgroup(v, all);
            t.e = table_group(table, p.E, tile / p.tiles_n);
            const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)table.row[t.e]), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)table.row[t.e + 1u]);
            const uint32_t from = (uint32_t)__builtin_amdgcn_readfirstlane((int)table.first[t.e]);
            banded_tile(tile - from * p.tiles_n, (hi - lo + S::BM - 1u) >> lg, p.tiles_n, tm, tn);
            begin = 0;
            bytes = p.row_codes;
            t.m0 = lo + tm * S::BM;
            t.n0 = tn * S::BN;
            t.rows_a = hi - t.m0;
            t.rows_b = p.N - t.n0;
        }
        t.m0 = __builtin_amdgcn_readfirstlane(t.m0);
        t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
        t.rows_a = __builtin_amdgcn_readfirstlane(t.rows_a);
        t.rows_b = __builtin_amdgcn_readfirstlane(t.rows_b);
        t.steps = (bytes + kStepBytes - 1u) / kStepBytes;
        t.half = bytes % kStepBytes != 0;
    };
    const auto finish = [&](const ChainTile& t) {
        if constexpr (GRADIENT) {
            void* d = (unsigned char*)p.c + (uint64_t)t.e * p.N * p.K * (DT == QESGD_F32 ? 4u : 2u);
            store_tile<S, DT>(ops, d, p.K, p.N, p.K, t.m0 + wm * S::FM * 32u, t.n0 + wn * S::FN * 32u, p.stream);
        } else {
            store_tile<S, DT>(ops, p.c, p.ldc, t.m0 + t.rows_a, p.N, t.m0 + wm * S::FM * 32u, t.n0 + wn * S::FN * 32u, p.stream);
        }
    };
    if constexpr (GRADIENT) {
        // experts without rows have no steps: their zeros come first
        ops.clear();
        for (; v < all; v += gridDim.x) {
            ChainTile t;
            uint32_t begin, bytes;
            place(t, begin, bytes);
            if (!bytes) finish(t);
        }
        v = blockIdx.x;
    }
    const auto advance = [&](ChainTile& t) {
        for (; v < all; v += gridDim.x) {
            uint32_t begin, bytes;
            place(t, begin, bytes);
            if (!bytes) continue;
            const uint32_t b_row = GRADIENT ? 0u : t.e;
            const unsigned char* b = p.b + b_row * p.b_stride;
            ops.aim(p.a + (uint64_t)t.m0 * p.row_codes + begin, b + (uint64_t)t.n0 * p.row_codes + begin,
                    p.a + p.a_scales + (uint64_t)t.m0 * p.row_scales + begin / 16u, b + p.b_scales + (uint64_t)t.n0 * p.row_scales + begin / 16u,
                    p.row_codes, p.row_scales, bytes, t, wm, wn);
            v += gridDim.x;
            return true;
        }
        return false;
    };
    unsigned char* const buffers[2] = {lds0, lds1};
    run_chain(ops, buffers, advance, finish);
}

// Tiles of `edge` rows that the groups make, from their mean size: half a tile more than their rows, and one at least.
uint64_t group_tiles(const GroupProduct& a, uint64_t edge) {
    const uint64_t groups = a.E < a.R ? a.E : a.R, tiles = a.R / edge + groups / 2;
    return tiles > groups ? tiles : groups;
}

// The edge of the tiles, and the pieces of the contraction, from how long they take on 256 CUs (tile_us), the larger edge where it hardly matters.  A piece has at least
// four steps; the sums of the pieces cost a launch, and are written and read at about 4 TB/s.  Measured, us, with 64 / 128 / 256:
//   products   16 experts, 32768 rows, N = K = 4096 660 / 348 / 280;  13, 9003, 1000, 2049 32.9 / 23.9 / 21.6;  8, 2048, 2048, 2048 15.6 / 11.9 / 16.8;
//              64, 1024, 1024, 1024 12.1 / 8.5 / 12.1;  8, 256, 4096, 4096 17.9 / 15.6 / 26.2;  64, 16384, 2048, 1024 70 / 40 / 35;  50, 25990, 576, 1024 32.5 / 20.0 / 22.3
//   gradients  8, 16384, 4096, 4096 544 / 256 / 207;  64, 4096, 1024, 1024 96 / 47 / 54;  16, 1024, 512, 512 8.9 / 7.5 / 8.9;  13, 9003, 1000, 2049 59 / 34.0 / 34.7
// and, one piece / as many as chosen, graph of 8 calls:
//   products   1 expert, 64 rows, N 1000, K 16384 20.3 / 9.9 (12 pieces);  8, 64, 512, 8192 12.0 / 8.8 (4);  1, 512, 1000, 25088 29.7 / 21.7 (2);
//              1, 1, 4096, 4096 7.8 / 7.5 (4);  23, 74, 152, 3597 7.6 / 8.0 (3)
//   gradients  1, 65536, 256, 256 69 / 14.9 (16);  1, 16384, 64, 64 19.6 / 7.5 (16);  4, 65536, 256, 512 39.7 / 27.7 (2)
struct Cut { uint32_t edge, pieces; };
constexpr uint32_t kMostPieces = 16;
template <class F>
Cut choose_cut(F&& tiles, double steps, double around, uint64_t sums) {
    Cut best{64, 1};
    double least = 1e300;
    for (uint32_t edge : {64u, 128u, 256u}) {
        const uint64_t n = tiles(edge);
        for (uint32_t pieces = 1; pieces <= kMostPieces && (pieces == 1 || (pieces * 4.0 <= steps && n * pieces <= 1024)); ++pieces) {
            const double us = tile_us(n * pieces, edge, steps / pieces + around) + (pieces == 1 ? 0.0 : 2.0 + (double)pieces * (double)sums * 2e-6);
            if (us <= least * (pieces == 1 ? 1.02 : 1.0)) {
                least = us;
                best = Cut{edge, pieces};
            }
        }
    }
    return best;
}
Cut product_cut(const GroupProduct& a) {
    return choose_cut([&](uint64_t edge) { return group_tiles(a, edge) * ((a.N + edge - 1) / edge); }, (double)((a.K + 255) / 256), 0.0, a.R * a.N);
}
// The contraction of a group of the mean size, and as much as two steps for the beginning and the end of a tile.
Cut gradient_cut(const GroupProduct& a) {
    return choose_cut([&](uint64_t edge) { return a.E * ((a.N + edge - 1) / edge) * ((a.K + edge - 1) / edge); }, 0.5 + (double)a.R / (double)a.E / 256.0, 2.0,
                      a.E * a.N * a.K);
}

int launch_sum(const GroupProduct& a, const PParams& p, const int32_t* offsets, uint32_t cols) {
    return launch_piece_sum(PieceSum{p.partial, p.pieces, p.sums, offsets, p.E, p.R, cols, p.c, p.ldc}, a.dtype, a.stream);
}

template <class S>
int launch_product_tiles(const GroupProduct& a, PParams& p) {
    p.tiles_n = (p.N + S::BN - 1) / S::BN;
    // the most tiles that R rows in E groups make
    const uint64_t groups = a.E < a.R ? a.E : a.R;
    p.tiles_m = (uint32_t)((a.R + (S::BM - 1) * groups) / S::BM);
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n * p.pieces;
    if (!grid_ok(tiles, S::threads)) return QESGD_ERR_DIM;
    by_type(p.pieces > 1 ? QESGD_F32 : a.dtype, [&](auto t) { k_mx4_grouped_product<S, t.value><<<(uint32_t)tiles, S::threads, 0, a.stream>>>(p); });
    const int rc = launched();
    return rc != QESGD_OK || p.pieces == 1 ? rc : launch_sum(a, p, p.offsets, p.N);
}

// One workgroup a CU, as its LDS has room for.  Where it gets three tiles or more; with fewer their search costs more than it saves.  A workgroup a tile / the chain,
// us: products of 16 experts, 32768 rows, N = K = 4096 297 / 280 (3.9 PFLOP/s), 8, 16384 158 / 150, 64, 16384, 2048, 1024 39.6 / 35.3, but 13, 9003, 1000,
// 2049 (164 tiles) 21.6 / 23.4; gradients 8, 16384, 4096, 4096 217 / 207, but 13, 9003, 1000, 2049 (468 tiles) 34.7 / 39.7.
constexpr uint64_t kChainTiles = 512;
template <class S, bool GRADIENT>
int launch_chain(const GroupProduct& a, PParams& p) {
    const uint64_t groups = a.E < a.R ? a.E : a.R;
    p.tiles_m = GRADIENT ? (p.N + S::BM - 1) / S::BM : (uint32_t)((a.R + (S::BM - 1) * groups) / S::BM);
    p.tiles_n = ((GRADIENT ? p.K : p.N) + S::BN - 1) / S::BN;
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n * (GRADIENT ? a.E : 1);
    if (!grid_ok(tiles, S::threads)) return QESGD_ERR_DIM;
    const uint32_t places = tiles < 256 ? (uint32_t)tiles : 256u;
    by_type(a.dtype, [&](auto t) { k_mx4_grouped_chain<S, t.value, GRADIENT><<<places, S::threads, 0, a.stream>>>(p); });
    return launched();
}

template <class S>
int launch_gradient_tiles(const GroupProduct& a, PParams& p) {
    p.tiles_m = (p.N + S::BM - 1) / S::BM;
    p.tiles_n = (p.K + S::BN - 1) / S::BN;
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n * a.E;
    if (!grid_ok(tiles * p.pieces, S::threads)) return QESGD_ERR_DIM;
    by_type(p.pieces > 1 ? QESGD_F32 : a.dtype, [&](auto t) {
        k_mx4_grouped_gradient<S, t.value><<<dim3((uint32_t)tiles, p.pieces), S::threads, 0, a.stream>>>(p);
    });
    const int rc = launched();
    return rc != QESGD_OK || p.pieces == 1 ? rc : launch_sum(a, p, nullptr, p.K);
}

}  // namespace

int launch_piece_sum(const PieceSum& p, uint32_t dtype, hipStream_t stream) {
    const uint64_t groups = (p.sums + 1023) / 1024;
    if (!grid_ok(groups, 256)) return QESGD_ERR_DIM;
    by_type(dtype, [&](auto t) { k_mx4_piece_sum<t.value><<<(uint32_t)groups, 256, 0, stream>>>(p); });
    return launched();
}

size_t grouped_product_workspace(const GroupProduct& a) {
    const uint32_t pieces = product_cut(a).pieces;
    return pieces > 1 ? pieces * a.R * a.N * sizeof(float) : 0;
}
size_t grouped_gradient_workspace(const GroupProduct& a) {
    const uint32_t pieces = gradient_cut(a).pieces;
    return pieces > 1 ? pieces * a.E * a.N * a.K * sizeof(float) : 0;
}

int launch_grouped_product(const GroupProduct& a) {
    qesgd_mx4_layout A, B;
    int rc = make_mx4_layout(a.R, a.K, &A);
    if (rc == QESGD_OK) rc = make_mx4_layout(a.N, a.K, &B);
    if (rc != QESGD_OK) return rc;
    PParams p{};
    p.a = a.a;
    p.b = a.b;
    p.a_scales = A.scales_off;
    p.b_scales = B.scales_off;
    p.b_stride = a.b_stride;
    p.offsets = a.offsets;
    p.E = a.E;
    p.R = (uint32_t)a.R;
    p.c = a.c;
    p.ldc = a.ldc;
    p.N = (uint32_t)a.N;
    p.row_codes = (uint32_t)A.row_codes;
    p.row_scales = (uint32_t)A.row_scales;
    const Cut cut = product_cut(a);
    p.pieces = cut.pieces;
    p.partial = a.workspace;
    p.sums = a.R * a.N;
    p.stream = cut.pieces == 1 && a.R * a.ldc * dtype_bytes(a.dtype) >= kStreamProduct && whole_lines(a.c, a.ldc * dtype_bytes(a.dtype));
    if (cut.edge == 64) return launch_product_tiles<TileShape<2, 2, 1, 1, 4>>(a, p);
    if (cut.edge == 128) return launch_product_tiles<TileShape<2, 2, 2, 2, 2>>(a, p);
    if (cut.pieces == 1 && group_tiles(a, 256) * ((a.N + 255) / 256) > kChainTiles) return launch_chain<TileShape<2, 4, 4, 2, 2>, false>(a, p);
    return launch_product_tiles<TileShape<2, 4, 4, 2, 2>>(a, p);
}

int launch_grouped_gradient(const GroupProduct& a) {
    qesgd_mx4_layout A, B;
    const uint64_t columns = grouped_columns(a.R, a.E);
    int rc = columns ? make_mx4_layout(a.N, columns, &A) : QESGD_ERR_DIM;
    if (rc == QESGD_OK) rc = make_mx4_layout(a.K, columns, &B);
    if (rc != QESGD_OK) return rc;
    PParams p{};
    p.a = a.a;
    p.b = a.b;
    p.a_scales = A.scales_off;
    p.b_scales = B.scales_off;
    p.offsets = a.offsets;
    p.E = a.E;
    p.R = (uint32_t)a.R;
    p.c = a.c;
    p.N = (uint32_t)a.N;
    p.K = (uint32_t)a.K;
    p.row_codes = (uint32_t)A.row_codes;
    p.row_scales = (uint32_t)A.row_scales;
    p.ldc = a.K;
    const Cut cut = gradient_cut(a);
    p.pieces = cut.pieces;
    p.partial = a.workspace;
    p.sums = a.E * a.N * a.K;
    p.stream = cut.pieces == 1 && p.sums * dtype_bytes(a.dtype) >= kStreamGradient && whole_lines(a.c, a.K * dtype_bytes(a.dtype));
    if (cut.edge == 64) return launch_gradient_tiles<TileShape<2, 2, 1, 1, 4>>(a, p);
    if (cut.edge == 128) return launch_gradient_tiles<TileShape<2, 2, 2, 2, 2>>(a, p);
    if (cut.pieces == 1 && a.E * ((a.N + 255) / 256) * ((a.K + 255) / 256) > kChainTiles) return launch_chain<TileShape<2, 4, 4, 2, 2>, true>(a, p);
    return launch_gradient_tiles<TileShape<2, 4, 4, 2, 2>>(a, p);
}

}  // namespace qesgd
