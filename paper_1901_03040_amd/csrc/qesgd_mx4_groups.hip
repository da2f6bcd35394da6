// Rows of tokens, in the order of their experts, to 4-bit microscaled codes: along the rows, along the rows of each group, or both from one read.
//
// The form along a group's rows is what a contraction over the group needs: group e's columns begin at a multiple of 128 (of 64 bytes of
// codes, of four scales), so the product walks whole blocks and no block holds rows of two experts.
//
// A row goes to k experts and is read k times, from the memory-side cache where x fits it.  16384 tokens x 2 x 4096 bf16 along the rows 48 us = 340 MB at 7.1 TB/s, 54 where x is another
// one each time; 8192 x 2, both forms, 37 (47) us nearest and 70 (72) stochastic, which is its arithmetic (two Philox calls for 8 elements).
#include "qesgd_experts.h"
#include "qesgd_groups.h"
#include "qesgd_launch.h"
#include "qesgd_mx4_codes.h"

namespace qesgd {
namespace {

struct GParams {
    const void* x;
    uint64_t ld;
    uint32_t T;
    const int32_t* order;
    uint32_t per, per_factor, per_shift;          // n / per = the upper half of n * per_factor, shifted
    const int32_t* offsets;
    uint32_t E, R, cols;
    uint32_t groups;                  // of 128 columns in a row
    uint32_t groups_t;                // of 128 rows in the form along the groups
    uint64_t slots;                   // R * groups * 128
    unsigned char* packed;
    uint64_t scales_off;
    unsigned char* packed_t;
    uint64_t scales_t_off;
    uint32_t key0, key1, round, worker;
};

// The rows of x that rows row[i] take, p.T for a row that is none of them (in[i] false) or has none.  All of order's numbers are on their way before the first is
// used: the loads of x wait for them once.
template <int N>
__device__ __forceinline__ void sources(const GParams& p, const uint32_t (&row)[N], const bool (&in)[N], uint32_t (&out)[N]) {
    int32_t pair[N];
#pragma unroll
    for (int i = 0; i < N; ++i) pair[i] = p.order ? p.order[min(row[i], p.R - 1u)] : (int32_t)row[i];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t n = (uint32_t)pair[i], q = p.per == 1u ? n : __umulhi(n, p.per_factor) >> p.per_shift;
        out[i] = in[i] && pair[i] >= 0 ? min(q, p.T) : p.T;
    }
}

// Along the rows: a lane owns 8 consecutive slots of the padded matrix, a quad a block, a wave kGChunks chunks of 512.
// One, two and four chunks a wave: 52 / 47 / 49 us there; stochastic 74 with two.
constexpr uint32_t kGWaves = 4, kGChunks = 2;

template <uint32_t DT, bool STOCHASTIC>
__global__ void __launch_bounds__(kGWaves * 64) k_mx4_group_rows(const GParams p) {
    if (STOCHASTIC) round_down();
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t begin = held(p.offsets[0], p.R), end = held(p.offsets[p.E], p.R);
    const uint64_t wave0 = ((uint64_t)blockIdx.x * kGWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (kGChunks * kChunk);
    const uint32_t group0 = (uint32_t)(wave0 >> 7), row0 = group0 / p.groups;                // uniform
    if (row0 >= end) return;
    uint32_t row[kGChunks], col[kGChunks], from[kGChunks];
    bool in[kGChunks];
#pragma unroll
    for (uint32_t c = 0; c < kGChunks; ++c) {
        // the wave's 4 kGChunks groups of 128 end at most so many rows
        uint32_t r = row0, g = group0 - row0 * p.groups + c * 4u + (lane >> 4);
        if (p.groups >= 4u * kGChunks) {
            const uint32_t over = g >= p.groups ? 1u : 0u;
            r += over;
            g -= over ? p.groups : 0u;
        } else {
            const uint32_t more = g / p.groups;
            r += more;
            g -= more * p.groups;
        }
        row[c] = r;
        col[c] = g * 128u + (lane & 15u) * 8u;
        in[c] = r >= begin && r < end;
    }
    sources(p, row, in, from);
    Eight<DT> v[kGChunks];
#pragma unroll
    for (uint32_t c = 0; c < kGChunks; ++c) {
        const uint32_t n = from[c] >= p.T || col[c] >= p.cols ? 0u : min(p.cols - col[c], 8u);
        v[c].load(p.x, n ? from[c] * p.ld + col[c] : 0u, n);
    }
#pragma unroll
    for (uint32_t c = 0; c < kGChunks; ++c) {
        const uint64_t slot = wave0 + c * kChunk + lane * kLaneElems;
        const uint32_t sb = scale_byte<STOCHASTIC>(quad_max(v[c].top()));
        const uint32_t word = encode8<DT, STOCHASTIC>(v[c], sb, slot >> 3, p.worker, p.round, p.key0, p.key1);
        const uint32_t scales = row_bytes(sb, lane);
        if (in[c]) {                                           // slots come in 128s: a row of lanes is in or out
            *(uint32_t*)(p.packed + (slot >> 1)) = word;
            if ((lane & 15u) == 0) *(uint32_t*)(p.packed + p.scales_off + (slot >> 5)) = scales;
        }
    }
}

// Both forms, or that along the groups alone, of 128 rows of one group x 128 columns.  The rows' form is made while the tile is read; the raw
// elements go to LDS, and then a lane takes 32 rows of one column.
// The tiles in order: all of some columns on one XCD, whose L2 would join their 64 bytes of a column into lines, took 34 us for 36 where x lay in a cache and 51 for 49 where it did not.
constexpr uint32_t kTile = 128, kBothThreads = 512;

template <uint32_t DT, bool STOCHASTIC>
__global__ void __launch_bounds__(kBothThreads) k_mx4_group_both(const GParams p) {
    if (STOCHASTIC) round_down();
    typedef typename std::conditional<DT == QESGD_F32, float, unsigned short>::type elem;
    // 32 rows, then 64 bytes of room: the four blocks of a column that a quad reads at once lie in different banks
    constexpr uint32_t kRoom = 64 / sizeof(elem);
    __shared__ __attribute__((aligned(16))) elem tile[kTile * kTile + 4 * kRoom];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t tr = blockIdx.x / p.groups, tc = blockIdx.x - tr * p.groups;
    Group g;
    if (!group_of_tile(p.offsets, p.E, p.R, Power{7}, 1, tr, g)) return;
    const uint32_t r0 = g.lo + (tr - g.first) * kTile, c0 = tc * kTile;
    const uint32_t col = (lane & 15u) * 8u;
    const uint32_t n = c0 + col >= p.cols ? 0u : min(p.cols - c0 - col, 8u);
    uint32_t rows[4], from_row[4];
    bool in[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        rows[i] = r0 + i * 32u + wave * 4u + (lane >> 4);
        in[i] = rows[i] < g.hi;
    }
    sources(p, rows, in, from_row);
    Eight<DT> v[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const bool there = from_row[i] < p.T && n;
        v[i].load(p.x, there ? from_row[i] * p.ld + c0 + col : 0u, there ? n : 0u);
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t r = i * 32u + wave * 4u + (lane >> 4), row = r0 + r;
        elem* to = tile + r * kTile + (r >> 5) * kRoom + col;
        if constexpr (DT == QESGD_F32) {
            *(vec4*)to = vec4{v[i].v[0], v[i].v[1], v[i].v[2], v[i].v[3]};
            *(vec4*)(to + 4) = vec4{v[i].v[4], v[i].v[5], v[i].v[6], v[i].v[7]};
        } else {
            *(uvec4*)to = v[i].v;
        }
        if (p.packed) {
            const uint64_t slot = (uint64_t)row * (p.groups * 128u) + c0 + col;
            const uint32_t sb = scale_byte<STOCHASTIC>(quad_max(v[i].top()));
            const uint32_t word = encode8<DT, STOCHASTIC>(v[i], sb, slot >> 3, p.worker, p.round, p.key0, p.key1);
            const uint32_t scales = row_bytes(sb, lane);
            if (row < g.hi) {
                *(uint32_t*)(p.packed + (slot >> 1)) = word;
                if ((lane & 15u) == 0) *(uint32_t*)(p.packed + p.scales_off + (slot >> 5)) = scales;
            }
        }
    }
    __syncthreads();
    // A lane takes 32 rows of a column: one of 32-bit elements, or of 16-bit ones either of the pair that a word of LDS holds.
    const uint32_t block = lane & 3u, word_col = DT == QESGD_F32 ? threadIdx.x >> 2 : (threadIdx.x >> 2) & 63u;
    const uint32_t side = DT == QESGD_F32 ? 0u : threadIdx.x >> 8;
    const uint32_t* from = (const uint32_t*)tile + block * (32u * kTile + kRoom) * sizeof(elem) / 4u + word_col;
    uint32_t raw[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) raw[j] = from[j * (kTile * sizeof(elem) / 4u)];
    Eight<DT> y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == QESGD_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[j].v[e] = __uint_as_float(raw[j * 8 + e]);
        } else {
            // the lower (upper) halves of two rows' words, as a pair along the column
            const uint32_t pick = side ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[j].v[e] = __builtin_amdgcn_perm(raw[j * 8 + 2 * e + 1], raw[j * 8 + 2 * e], pick);
        }
    }
    const uint32_t c = DT == QESGD_F32 ? word_col : word_col * 2u + side;
    const uint32_t sb = scale_byte<STOCHASTIC>(max(max(y[0].top(), y[1].top()), max(y[2].top(), y[3].top())));
    const uint64_t slot = (uint64_t)(c0 + c) * (p.groups_t * 128ull) + tr * kTile + block * 32u;
    uvec4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = encode8<DT, STOCHASTIC>(y[j], sb, (slot >> 3) + j, p.worker, p.round, p.key0, p.key1);
    uint32_t scales = sb << (8u * block);
    scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0xB1, 0xF, 0xF, false);
    scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x4E, 0xF, 0xF, false);
    if (c0 + c < p.cols) {
        *(uvec4*)(p.packed_t + (slot >> 1)) = w;
        if (block == 0) *(uint32_t*)(p.packed_t + p.scales_t_off + (slot >> 5)) = scales;
    }
}

}  // namespace

int launch_quantize_groups(const GroupQuantize& a) {
    qesgd_mx4_layout L{}, T{};
    int rc = make_mx4_layout(a.R, a.cols, &L);
    if (rc == QESGD_OK) rc = make_mx4_layout(a.cols, grouped_columns(a.R, a.E), &T);
    if (rc != QESGD_OK) return rc;
    GParams p{};
    p.x = a.x;
    p.ld = a.ld;
    p.T = (uint32_t)a.T;
    p.order = a.order;
    p.per = a.per;
    divide_by(a.per, p.per_factor, p.per_shift);
    p.offsets = a.offsets;
    p.E = a.E;
    p.R = (uint32_t)a.R;
    p.cols = (uint32_t)a.cols;
    p.groups = (uint32_t)(L.row_codes / 64);
    p.groups_t = (uint32_t)(T.row_codes / 64);
    p.slots = a.R * L.row_codes * 2;
    p.packed = a.packed;
    p.scales_off = L.scales_off;
    p.packed_t = a.packed_t;
    p.scales_t_off = T.scales_off;
    p.key0 = (uint32_t)a.seed;
    p.key1 = (uint32_t)(a.seed >> 32);
    p.round = a.round;
    p.worker = a.worker;
    const bool both = a.packed_t != nullptr;
    constexpr uint64_t tile = kGWaves * kGChunks * kChunk;
    const uint64_t blocks = both ? (uint64_t)p.groups_t * p.groups : (p.slots + tile - 1) / tile;
    const uint32_t threads = both ? kBothThreads : kGWaves * 64;
    if (!grid_ok(blocks, threads)) return QESGD_ERR_DIM;
    by_type(a.dtype, [&](auto t) {
        constexpr uint32_t DT = t.value;
        if (both && a.stochastic) k_mx4_group_both<DT, true><<<(uint32_t)blocks, threads, 0, a.stream>>>(p);
        else if (both) k_mx4_group_both<DT, false><<<(uint32_t)blocks, threads, 0, a.stream>>>(p);
        else if (a.stochastic) k_mx4_group_rows<DT, true><<<(uint32_t)blocks, threads, 0, a.stream>>>(p);
        else k_mx4_group_rows<DT, false><<<(uint32_t)blocks, threads, 0, a.stream>>>(p);
    });
    return launched();
}

}  // namespace qesgd
