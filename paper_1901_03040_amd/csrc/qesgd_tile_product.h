// C = A B^T of two matrices whose rows lie along the contraction: the pipeline that the 4-bit product and the
// orthogonalisation share (not installed).
//
// A workgroup owns a BM x BN tile of C.  The contraction runs in steps of 128 bytes of every row of A and B.  A step's
// rows go from memory to LDS without passing through registers (16 bytes a lane) into one of two buffers, while the
// matrix instructions read the other; one barrier a step.  A row of a step is 8 chunks of 16 bytes; chunk c of row r lies at
// place c ^ (r & 7), so that the eight lanes that one cycle serves (8 rows, the same chunk) touch all banks once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qesgd {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kStepBytes = 128;

// WM x WN waves, each of FM x FN fragments of 32 x 32.
template <int WM_, int WN_, int FM_, int FN_>
struct TileShape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    static constexpr int threads = WM * WN * 64;
    static constexpr int lds = 2 * (BM + BN) * (int)kStepBytes;
};

// One step of ROWS rows to LDS.  `off` (set by tile_offsets) holds the lane's byte offsets from the tile's first row.
template <int ROWS, int THREADS>
struct TileLoader {
    static constexpr int N = ROWS * 8 / THREADS;
    static_assert(N >= 1 && ROWS * 8 % THREADS == 0, "every thread moves the same number of chunks");
    uint32_t off[N];
    uint32_t wave_at;

    // Row r of the tile is row min(r, rows - 1) of what is there: no row beyond the end is read.
    __device__ __forceinline__ void init(uint32_t pitch, uint32_t rows) {
        wave_at = (threadIdx.x >> 6) * 1024u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t at = i * THREADS + threadIdx.x, r = at >> 3, c = (at & 7u) ^ (r & 7u);
            off[i] = min(r, rows - 1u) * pitch + c * 16u;
        }
    }
    // `limit`: bytes of the row that are left in this step (128, or 64: the chunks of the second half then repeat the first).
    __device__ __forceinline__ void load(const unsigned char* base, unsigned char* lds, bool half) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t o = half ? off[i] - (((threadIdx.x & 7u) ^ ((threadIdx.x >> 3) & 7u)) & 4u) * 16u : off[i];
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)(base + o),
                                             (__attribute__((address_space(3))) uint32_t*)(lds + i * (THREADS * 16) + wave_at),
                                             16, 0, 0);
        }
    }
};

// Number of the tile that workgroup b of n takes: ids go round-robin over the 8 XCDs, so each XCD gets one run of tiles, whose rows
// of A and B its own L2 then holds.
__device__ __forceinline__ uint32_t tile_of_workgroup(uint32_t b, uint32_t n) {
    const uint32_t per = n >> 3, left = n & 7u, x = b & 7u;
    return (b >> 3) + x * per + (x < left ? x : left);
}

}  // namespace qesgd
