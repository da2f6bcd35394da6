// Groups of rows on the device: which group a tile belongs to, found by every wave for itself from the offsets (not installed).
//
// The sizes are known on the device only, so a launch has room for the most tiles that R rows in E groups can make and a workgroup finds out
// what it has to do: a prefix sum over the groups' tiles, 64 groups at a time.  Up to 64 groups that is one load and some ten
// instructions, about as long as a trip to memory; a launch of its own that lists the tiles would take more than that.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qesgd {

// Inclusive prefix sum over the 64 lanes.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);   // row_shr:1
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);   // row_shr:2
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);   // row_shr:4
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);   // row_shr:8
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);   // row_bcast:15 to rows 1 and 3
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);   // row_bcast:31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, uint32_t lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)lane); }

// An offset held to 0 .. R: whatever the caller's memory holds, rows stay inside the buffers.
__device__ __forceinline__ uint32_t held(int32_t offset, uint32_t R) { return offset < 0 ? 0u : min((uint32_t)offset, R); }

struct Group {
    uint32_t e, lo, hi;              // rows lo .. hi - 1
    uint32_t first;                  // tiles of the groups before it
};

// How many tiles a number of rows makes: tiles of 2^lg rows, and of N.
struct Power {
    uint32_t lg;
    __device__ __forceinline__ uint32_t tiles(uint32_t rows) const { return (rows + (1u << lg) - 1u) >> lg; }
};
template <uint32_t N>
struct Times {
    __device__ __forceinline__ uint32_t tiles(uint32_t rows) const { return (rows + N - 1u) / N; }
};

// Tiles of group i; lo and hi of that group.
template <class Edge>
__device__ __forceinline__ uint32_t group_tiles(const int32_t* offsets, uint32_t E, uint32_t R, Edge edge, uint32_t i, uint32_t& lo, uint32_t& hi) {
    const uint32_t at = min(i, E - 1u);
    lo = held(offsets[at], R);
    hi = held(offsets[at + 1u], R);
    return i < E && hi > lo ? edge.tiles(hi - lo) : 0u;
}

// All groups' tiles.
template <class Edge>
__device__ __forceinline__ uint32_t all_tiles(const int32_t* offsets, uint32_t E, uint32_t R, Edge edge) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t total = 0, lo, hi;
    for (uint32_t base = 0; base < E; base += 64u) total += group_tiles(offsets, E, R, edge, base + lane, lo, hi);
    return lane_value(wave_prefix(total), 63u);
}

// The group of tile `tile` (times `each`: a group's tiles count so many times); false where there are not so many.  Uniform.
template <class Edge>
__device__ __forceinline__ bool group_of_tile(const int32_t* offsets, uint32_t E, uint32_t R, Edge edge, uint32_t each, uint32_t tile, Group& g) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t before = 0;
    for (uint32_t base = 0; base < E; base += 64u) {
        uint32_t lo, hi;
        const uint32_t tiles = group_tiles(offsets, E, R, edge, base + lane, lo, hi) * each;
        const uint32_t behind = before + wave_prefix(tiles);
        const uint64_t found = __ballot(tile < behind);
        if (found) {
            const uint32_t at = (uint32_t)__builtin_ctzll(found);
            g.e = base + at;
            g.lo = lane_value(lo, at);
            g.hi = lane_value(hi, at);
            g.first = lane_value(behind - tiles, at);
            return true;
        }
        before = lane_value(behind, 63u);
    }
    return false;
}

// Group e.
template <class Edge>
__device__ __forceinline__ Group group_number(const int32_t* offsets, uint32_t E, uint32_t R, Edge edge, uint32_t e) {
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t total = 0, lo, hi;
    for (uint32_t base = 0; base < e; base += 64u) {
        const uint32_t tiles = group_tiles(offsets, E, R, edge, base + lane, lo, hi);
        total += base + lane < e ? tiles : 0u;
    }
    Group g;
    g.e = e;
    g.first = lane_value(wave_prefix(total), 63u);
    g.lo = held(offsets[e], R);
    g.hi = max(held(offsets[e + 1u], R), g.lo);
    return g;
}

}  // namespace qesgd
