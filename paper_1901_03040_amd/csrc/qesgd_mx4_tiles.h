// Tiles of products of packed 4-bit matrices on the scaled matrix instruction: a lane's operand is 32 elements of one row, which is one
// block of the format, next to its scale byte, so nothing is unpacked.  What the product of two matrices and those by groups of rows share (not installed).
#pragma once

#include "qesgd_launch.h"
#include "qesgd_matrix.h"
#include "qesgd_tile_product.h"

namespace qesgd {

// A fragment whose lane holds column `col` and rows row + 8 q + r, r = 0..3.
template <uint32_t DT>
__device__ __forceinline__ void store_fragment(void* c, uint64_t ldc, uint32_t M, uint32_t N, uint32_t row, uint32_t col, bool whole, const acc16& acc) {
    const uint64_t base = (uint64_t)row * ldc + col;
    if (whole) {
#pragma unroll
        for (int e = 0; e < 16; ++e) put<DT>(c, base + (8u * (e >> 2) + (e & 3)) * ldc, acc[e]);
    } else if (col < N) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (row + 8u * (e >> 2) + (e & 3) < M) put<DT>(c, base + (8u * (e >> 2) + (e & 3)) * ldc, acc[e]);
    }
}

template <class S>
struct Mx4Ops {
    static constexpr int PARTS = 4;                            // 64 columns each: one matrix instruction deep
    struct Frag { int4v a[S::FM], b[S::FN]; };
    // Scales of two steps: 16 bytes of every row of the tile, four words a row.  A load from memory for each fragment instead touches 32
    // lines for 128 bytes, 96 times a step, and held the kernel at a quarter of the matrix rate.
    static constexpr int NA = S::BM * 4 / S::threads, NB = S::BN * 4 / S::threads;
    static constexpr int LOADS = (S::BM + S::BN) * 8 / S::threads, PAIR_LOADS = NA + NB;
    static constexpr int scale_bytes = (S::BM + S::BN) * 16;
    // with N buffers a pair comes N steps ahead, while up to N / 2 others are still wanted: one more, and a power of two
    static constexpr uint32_t scale_buffers = S::BUFFERS == 2 ? 2 : 4;
    TileLoader<S::BM, S::threads> la;
    TileLoader<S::BN, S::threads> lb;
    const unsigned char *a, *b;
    const unsigned char *sa, *sb;                              // scales of the tile's first rows
    unsigned char* scales;                                     // in LDS
    uint32_t off_a[NA], off_b[NB];                             // rows of the words that the lane moves
    uint32_t last_word, scale_at, scale_at_a, scale_at_b;
    uint32_t ya[S::FM][2], yb[S::FN][2], xa[S::FM][2], xb[S::FN][2];            // of the next step, and of this one
    uint32_t at_a, at_b, steps, h, second;
    bool half;
    acc16 acc[S::FM][S::FN];

    // a, b: the first scales of the tile's first rows, of which there are rows_a and rows_b; row_scales: bytes from one row to the next; bytes: of a row's
    // scales from there to the end of the contraction.
    template <class Order = Straight>
    __device__ __forceinline__ void init_scales(const unsigned char* a, const unsigned char* b, uint32_t rows_a, uint32_t rows_b, uint32_t row_scales,
                                                uint32_t bytes, uint32_t wm, uint32_t wn, Order of_b = {}) {
        last_word = bytes - 4u;
        sa = a;
        sb = b;
#pragma unroll
        for (int i = 0; i < NA; ++i) off_a[i] = min((i * S::threads + threadIdx.x) >> 2, rows_a - 1u) * row_scales;
#pragma unroll
        for (int i = 0; i < NB; ++i) off_b[i] = min(of_b((i * S::threads + threadIdx.x) >> 2), rows_b - 1u) * row_scales;
        scale_at = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * 256u);
        scale_at_a = (wm * S::FM * 32u + (threadIdx.x & 31u)) * 16u;
        scale_at_b = (S::BM + wn * S::FN * 32u + (threadIdx.x & 31u)) * 16u;
    }
    __device__ __forceinline__ void fetch_pair(uint32_t step) {
        // a row ends with a whole word; what would lie behind it takes that one again
        const uint32_t word = min(step * 8u + (threadIdx.x & 3u) * 4u, last_word);
        const uint32_t to = lds_number(scales) + ((step >> 1) & (scale_buffers - 1u)) * scale_bytes + scale_at;
#pragma unroll
        for (int i = 0; i < NA; ++i) load_to_lds_4(sa, off_a[i] + word, to + i * S::threads * 4);
#pragma unroll
        for (int i = 0; i < NB; ++i) load_to_lds_4(sb, off_b[i] + word, to + S::BM * 16 + i * S::threads * 4);
    }
    __device__ __forceinline__ void fetch(uint32_t step, unsigned char* to) {
        const bool short_step = half && step + 1 == steps;
        la.load(a + (uint64_t)step * kStepBytes, to, short_step);
        lb.load(b + (uint64_t)step * kStepBytes, to + S::BM * kStepBytes, short_step);
    }
    __device__ __forceinline__ void arrive(uint32_t step) {
        const unsigned char* from = scales + ((step >> 1) & (scale_buffers - 1u)) * scale_bytes + (step & 1u) * 8u;
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { const uint2 v = *(const uint2*)(from + scale_at_a + f * 512); ya[f][0] = v.x; ya[f][1] = v.y; }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { const uint2 v = *(const uint2*)(from + scale_at_b + f * 512); yb[f][0] = v.x; yb[f][1] = v.y; }
        // The second half of a half step repeats the first half's codes and takes 2^-127 on either side: those products, at most
        // 36 * 2^-254, are zero in fp32.
        second = half && step + 1 >= steps ? 0u : 0xFFFFFFFFu;
    }
    // A lane's blocks of a step are scale bytes 2 s + h of its row: a shift by 8 h brings them to bytes 0 and 2 of the two words.
    __device__ __forceinline__ void next() {
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { xa[f][0] = ya[f][0] >> (8u * h); xa[f][1] = (ya[f][1] & second) >> (8u * h); }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { xb[f][0] = yb[f][0] >> (8u * h); xb[f][1] = (yb[f][1] & second) >> (8u * h); }
    }
    __device__ __forceinline__ void read(Frag& f, const unsigned char* from, int part) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i) f.a[i] = *(const int4v*)(from + (at_a ^ (part * 32u)) + i * 4096);
#pragma unroll
        for (int j = 0; j < S::FN; ++j) f.b[j] = *(const int4v*)(from + (at_b ^ (part * 32u)) + j * 4096);
    }
    __device__ __forceinline__ static int8v wide(const int4v& v) { return int8v{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; }
    template <int PART>
    __device__ __forceinline__ void multiply_part(const Frag& f) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(f.a[i]), wide(f.b[j]), acc[i][j], 4, 4, (PART & 1) * 2,
                                                                           (int)xa[i][PART >> 1], (PART & 1) * 2, (int)xb[j][PART >> 1]);
    }
    __device__ __forceinline__ void multiply(const Frag& f, int part) {
        switch (part) {
            case 0: multiply_part<0>(f); break;
            case 1: multiply_part<1>(f); break;
            case 2: multiply_part<2>(f); break;
            default: multiply_part<3>(f); break;
        }
    }
};

// How long so many tiles take on 256 CUs, us.  A step of 256 columns takes, us: 64 x 64 tiles 0.30 while a CU has one, 0.62 with two; 128 x 128 0.85 and
// 1.5; 256 x 256 1.2 on an empty chip, 2.3 on a full one.
inline double tile_us(uint64_t groups, uint32_t edge, double steps) {
    const uint64_t slots = edge == 256 ? 256 : 512, left = groups % slots;
    const double full = edge == 256 ? 2.3 : edge == 128 ? 1.5 : 0.62;
    const double last = left == 0 ? 0.0 : edge == 256 ? 1.2 + 1.1 * (double)left / 256.0 : left <= 256 ? (edge == 128 ? 0.85 : 0.30) : full;
    return ((double)(groups / slots) * full + last) * steps + (double)((groups + slots - 1) / slots);
}

}  // namespace qesgd
