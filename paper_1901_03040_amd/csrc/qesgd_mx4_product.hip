// C = A B^T of two packed 4-bit matrices on the scaled matrix instruction: a lane's operand is 32 elements of one row, which is one
// block of the format, next to its scale byte, so nothing is unpacked.  Element products are exact, sums are fp32.
#include <stdlib.h>
#include <type_traits>

#include "qesgd_internal.h"
#include "qesgd_matrix.h"
#include "qesgd_tile_product.h"

namespace qesgd {
namespace {

struct PParams {
    const unsigned char* a;
    const unsigned char* b;
    const unsigned char* a_scales;
    const unsigned char* b_scales;
    void* c;
    uint64_t ldc;
    uint32_t M, N;
    uint32_t row_codes, row_scales;       // of either operand: both have K columns
    uint32_t tiles_m, tiles_n;
};

template <uint32_t DT>
__device__ __forceinline__ void put(void* c, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)c)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)c)[at] = (_Float16)v;
    else ((__bf16*)c)[at] = (__bf16)v;
}

template <class S>
struct Mx4Ops {
    static constexpr int PARTS = 4;                            // 64 columns each: one matrix instruction deep
    static constexpr int LOADS = (S::BM + S::BN) * 8 / S::threads;
    struct Frag { int4v a[S::FM], b[S::FN]; };
    // Scales of two steps: 16 bytes of every row of the tile, four words a row.  A load from memory for each fragment instead touches 32
    // lines for 128 bytes, 96 times a step, and held the kernel at a quarter of the matrix rate.
    static constexpr int NA = S::BM * 4 / S::threads, NB = S::BN * 4 / S::threads;
    static constexpr int scale_bytes = (S::BM + S::BN) * 16;
    TileLoader<S::BM, S::threads> la;
    TileLoader<S::BN, S::threads> lb;
    const unsigned char *a, *b;
    const unsigned char *sa, *sb;                              // scales of the tile's first rows
    unsigned char* scales;                                     // in LDS, two buffers
    uint32_t off_a[NA], off_b[NB];                             // rows of the words that the lane moves
    uint32_t row_scales, scale_at, scale_at_a, scale_at_b;
    uint32_t ya[S::FM][2], yb[S::FN][2], xa[S::FM][2], xb[S::FN][2];            // of the next step, and of this one
    uint32_t at_a, at_b, steps, h, second;
    bool half;
    acc16 acc[S::FM][S::FN];

    __device__ __forceinline__ void init_scales(const PParams& p, uint32_t m0, uint32_t n0, uint32_t wm, uint32_t wn) {
        row_scales = p.row_scales;
        sa = p.a_scales + (uint64_t)m0 * row_scales;
        sb = p.b_scales + (uint64_t)n0 * row_scales;
#pragma unroll
        for (int i = 0; i < NA; ++i) off_a[i] = min((i * S::threads + threadIdx.x) >> 2, p.M - m0 - 1u) * row_scales;
#pragma unroll
        for (int i = 0; i < NB; ++i) off_b[i] = min((i * S::threads + threadIdx.x) >> 2, p.N - n0 - 1u) * row_scales;
        scale_at = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * 256u);
        scale_at_a = (wm * S::FM * 32u + (threadIdx.x & 31u)) * 16u;
        scale_at_b = (S::BM + wn * S::FN * 32u + (threadIdx.x & 31u)) * 16u;
    }
    __device__ __forceinline__ void fetch_pair(uint32_t step) {
        // a row ends with a whole word; what would lie behind it takes that one again
        const uint32_t word = min(step * 8u + (threadIdx.x & 3u) * 4u, row_scales - 4u);
        const uint32_t to = lds_number(scales) + ((step >> 1) & 1u) * scale_bytes + scale_at;
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
        const unsigned char* from = scales + ((step >> 1) & 1u) * scale_bytes + (step & 1u) * 8u;
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

template <class S, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_mx4_product(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char scales[2 * Mx4Ops<S>::scale_bytes];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    uint32_t tm, tn;
    banded_tile(tile_of_workgroup(blockIdx.x, gridDim.x), p.tiles_m, p.tiles_n, tm, tn);
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN;
    Mx4Ops<S> ops;
    ops.a = p.a + (uint64_t)m0 * p.row_codes;
    ops.b = p.b + (uint64_t)n0 * p.row_codes;
    ops.la.init(p.row_codes, p.M - m0);
    ops.lb.init(p.row_codes, p.N - n0);
    ops.scales = scales;
    ops.init_scales(p, m0, n0, wm, wn);
    ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
    ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
    ops.steps = (p.row_codes + kStepBytes - 1u) / kStepBytes;
    ops.half = p.row_codes % kStepBytes != 0;
    ops.h = h;
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) ops.acc[i][j] = acc16{};
    unsigned char* const buffers[2] = {lds0, lds1};
    run_steps(ops, ops.steps, buffers);

    // a lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const uint32_t col = n0 + (wn * S::FN + j) * 32u + (lane & 31u);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t row = m0 + (wm * S::FM + i) * 32u + 8u * (e >> 2) + 4u * h + (e & 3);
                if (row < p.M && col < p.N) put<DT>(p.c, (uint64_t)row * p.ldc + col, ops.acc[i][j][e]);
            }
        }
}

template <class S>
int launch_product_as(const Mx4Product& a, PParams& p) {
    p.tiles_m = (p.M + S::BM - 1) / S::BM;
    p.tiles_n = (p.N + S::BN - 1) / S::BN;
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n;
    if (tiles >= (1ull << 31)) return QESGD_ERR_DIM;
    switch (a.dtype) {
        case QESGD_F32: k_mx4_product<S, QESGD_F32><<<(uint32_t)tiles, S::threads, 0, a.stream>>>(p); break;
        case QESGD_BF16: k_mx4_product<S, QESGD_BF16><<<(uint32_t)tiles, S::threads, 0, a.stream>>>(p); break;
        default: k_mx4_product<S, QESGD_F16><<<(uint32_t)tiles, S::threads, 0, a.stream>>>(p); break;
    }
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

}  // namespace

size_t mx4_product_workspace(uint64_t M, uint64_t N, uint64_t K) { return 0; }

int launch_mx4_product(const Mx4Product& a) {
    qesgd_mx4_layout A, B;
    int rc = make_mx4_layout(a.M, a.K, &A);
    if (rc == QESGD_OK) rc = make_mx4_layout(a.N, a.K, &B);
    if (rc != QESGD_OK) return rc;
    PParams p{};
    p.a = a.a;
    p.b = a.b;
    p.a_scales = a.a + A.scales_off;
    p.b_scales = a.b + B.scales_off;
    p.c = a.c;
    p.ldc = a.ldc;
    p.M = (uint32_t)a.M;
    p.N = (uint32_t)a.N;
    p.row_codes = (uint32_t)A.row_codes;
    p.row_scales = (uint32_t)A.row_scales;
        const char* e = getenv("MXE");
    switch (e ? atoi(e) : 128) {
        case 256: return launch_product_as<TileShape<2, 4, 4, 2, 2>>(a, p);
        case 64: return launch_product_as<TileShape<2, 2, 1, 1, 2>>(a, p);
        default: return launch_product_as<TileShape<2, 2, 2, 2, 2>>(a, p);
    }
}

}  // namespace qesgd
