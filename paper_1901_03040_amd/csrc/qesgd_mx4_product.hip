// C = A B^T of two packed 4-bit matrices on the scaled matrix instruction: a lane's operand is 32 elements of one row, which is one
// block of the format, next to its scale byte, so nothing is unpacked.  Element products are exact, sums are fp32.
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
    uint32_t tiles_m, tiles_n, tiles;
    uint32_t pieces;                      // of the contraction; with more than one the sums go to partial [pieces, M, N]
    float* partial;
};

template <uint32_t DT>
__device__ __forceinline__ void put(void* c, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)c)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)c)[at] = (_Float16)v;
    else ((__bf16*)c)[at] = (__bf16)v;
}

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

    __device__ __forceinline__ void init_scales(const PParams& p, uint32_t m0, uint32_t n0, uint32_t wm, uint32_t wn, uint32_t first) {
        const uint32_t row_scales = p.row_scales;
        last_word = row_scales - first * 8u - 4u;
        sa = p.a_scales + (uint64_t)m0 * row_scales + first * 8u;
        sb = p.b_scales + (uint64_t)n0 * row_scales + first * 8u;
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

// 4096 x 4096 x 25088 (256 x 256 tiles) 190 us = 4.4 PFLOP/s, where the card lowers its clock to about 1.7 GHz; 8192 x 4096 x 4096 77 us = 3.6, its
// prologue and epilogue being a fifth of a tile's 16 steps.  Small tiles are bound by the CU's path from L2 to LDS: a step of 64 x 64, 18 KB, takes
// 0.30 us of a CU, with one workgroup on it or with two.
template <class S, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_mx4_product(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds2[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char lds3[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char scales[Mx4Ops<S>::scale_buffers * Mx4Ops<S>::scale_bytes];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    uint32_t t = tile_of_workgroup(blockIdx.x, gridDim.x), tm, tn;
    const uint32_t all_steps = (p.row_codes + kStepBytes - 1u) / kStepBytes;
    uint32_t piece = 0, first = 0, steps = all_steps;
    if (p.pieces > 1) {
        piece = __builtin_amdgcn_readfirstlane(t / p.tiles);
        t -= piece * p.tiles;
        // pieces begin with an even step, because scales come in pairs
        first = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)piece * all_steps / p.pieces)) & ~1u;
        steps = (piece + 1 == p.pieces ? all_steps : __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)(piece + 1) * all_steps / p.pieces)) & ~1u) - first;
    }
    banded_tile(t, p.tiles_m, p.tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN;
    Mx4Ops<S> ops;
    ops.a = p.a + (uint64_t)m0 * p.row_codes + (uint64_t)first * kStepBytes;
    ops.b = p.b + (uint64_t)n0 * p.row_codes + (uint64_t)first * kStepBytes;
    ops.la.init(p.row_codes, p.M - m0);
    ops.lb.init(p.row_codes, p.N - n0);
    ops.scales = scales;
    ops.init_scales(p, m0, n0, wm, wn, first);
    ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
    ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
    ops.steps = steps;
    ops.half = p.row_codes % kStepBytes != 0 && first + steps == all_steps;
    ops.h = h;
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

    // a lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r
    const bool whole = m0 + S::BM <= p.M && n0 + S::BN <= p.N;                 // uniform: most tiles store without asking
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const uint32_t col = n0 + (wn * S::FN + j) * 32u + (lane & 31u), row = m0 + (wm * S::FM + i) * 32u + 4u * h;
            if (p.pieces > 1) store_fragment<QESGD_F32>(p.partial + (uint64_t)piece * p.M * p.N, p.N, p.M, p.N, row, col, whole, ops.acc[i][j]);
            else store_fragment<DT>(p.c, p.ldc, p.M, p.N, row, col, whole, ops.acc[i][j]);
        }
}

// C from the sums of the pieces, added in order.  Four numbers a lane where rows allow it, eight pieces on their way: the sums come from the
// memory-side cache and are few, so it is a launch and a latency.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_mx4_product_sum(const PParams p) {
    const uint64_t count = (uint64_t)p.M * p.N, i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 4u;
    if (i >= count) return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if ((count & 3u) == 0) {
        for (uint32_t k0 = 0; k0 < p.pieces; k0 += 8) {
            float x[8][4];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) *(float4*)x[k] = *(const float4*)(p.partial + min(k0 + k, p.pieces - 1u) * count + i);
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += k0 + k < p.pieces ? x[k][e] : 0.0f;
        }
    } else {
        for (uint32_t k = 0; k < p.pieces; ++k)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (i + e < count) v[e] += p.partial[k * count + i + e];
    }
    uint32_t row = (uint32_t)(i / p.N), col = (uint32_t)(i - (uint64_t)row * p.N);
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        if (i + e < count) put<DT>(p.c, (uint64_t)row * p.ldc + col, v[e]);
        if (++col == p.N) { col = 0; ++row; }
    }
}

// A few rows of A (up to 32 are right): what counts is to have all of B on its way at once.  A workgroup owns 32 columns of C; its waves take the steps of the
// contraction in turn, each straight from memory to registers, and their sums meet in LDS, added in the order of the waves.
constexpr int kFewWaves = 16;
constexpr uint64_t kFewRows = 16, kFewColumns = 8192;
template <uint32_t DT>
__global__ void __launch_bounds__(kFewWaves * 64) k_mx4_product_few(const PParams p) {
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][16][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5, l = lane & 31u;
    const uint32_t n0 = blockIdx.x * 32u;
    const uint32_t ra = min(l, p.M - 1u), rb = min(n0 + l, p.N - 1u);
    const unsigned char *a = p.a + (uint64_t)ra * p.row_codes, *b = p.b + (uint64_t)rb * p.row_codes;
    const unsigned char *sa = p.a_scales + (uint64_t)ra * p.row_scales, *sb = p.b_scales + (uint64_t)rb * p.row_scales;
    const uint32_t steps = (p.row_codes + kStepBytes - 1u) / kStepBytes;
    const bool half = p.row_codes % kStepBytes != 0;
    acc16 acc = {};
    for (uint32_t s = wave; s < steps; s += kFewWaves) {
        // the second half of a half step: codes once more and 2^-127 on either side, which gives zeros (see arrive)
        const bool short_step = half && s + 1 == steps;
        const uint32_t second = short_step ? 0u : 64u, words = short_step ? 0u : 4u, keep = short_step ? 0u : 0xFFFFFFFFu;
        int4v va[4], vb[4];
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
            const uint32_t at = s * kStepBytes + (q >> 1) * second + (2u * (q & 1u) + h) * 16u;
            vb[q] = *(const int4v*)(b + at);
            va[q] = *(const int4v*)(a + at);
        }
        const uint32_t xb[2] = {*(const uint32_t*)(sb + s * 8u) >> (8u * h), (*(const uint32_t*)(sb + s * 8u + words) & keep) >> (8u * h)};
        const uint32_t xa[2] = {*(const uint32_t*)(sa + s * 8u) >> (8u * h), (*(const uint32_t*)(sa + s * 8u + words) & keep) >> (8u * h)};
        const auto wide = [](const int4v& v) { return int8v{v[0], v[1], v[2], v[3], 0, 0, 0, 0}; };
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(va[0]), wide(vb[0]), acc, 4, 4, 0, (int)xa[0], 0, (int)xb[0]);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(va[1]), wide(vb[1]), acc, 4, 4, 2, (int)xa[0], 2, (int)xb[0]);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(va[2]), wide(vb[2]), acc, 4, 4, 0, (int)xa[1], 0, (int)xb[1]);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(va[3]), wide(vb[3]), acc, 4, 4, 2, (int)xa[1], 2, (int)xb[1]);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[wave][e][lane] = acc[e];
    __syncthreads();
    const uint32_t used = min((uint32_t)kFewWaves, steps);
    for (uint32_t i = threadIdx.x; i < 1024u; i += kFewWaves * 64u) {
        const uint32_t e = i >> 6, ln = i & 63u, row = 8u * (e >> 2) + 4u * (ln >> 5) + (e & 3u), col = n0 + (ln & 31u);
        float v = 0.0f;
        for (uint32_t w = 0; w < used; ++w) v += sums[w][e][ln];
        if (row < p.M && col < p.N) put<DT>(p.c, (uint64_t)row * p.ldc + col, v);
    }
}

int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

// f(the number of dtype as a constant)
template <class F>
void by_type(uint32_t dtype, F&& f) {
    switch (dtype) {
        case QESGD_F32: f(std::integral_constant<uint32_t, QESGD_F32>{}); break;
        case QESGD_BF16: f(std::integral_constant<uint32_t, QESGD_BF16>{}); break;
        default: f(std::integral_constant<uint32_t, QESGD_F16>{}); break;
    }
}

template <class S>
int launch_tiles(const Mx4Product& a, PParams& p, uint32_t pieces) {
    p.tiles_m = (p.M + S::BM - 1) / S::BM;
    p.tiles_n = (p.N + S::BN - 1) / S::BN;
    const uint64_t tiles = (uint64_t)p.tiles_m * p.tiles_n;
    if (!grid_ok(tiles * pieces, S::threads)) return QESGD_ERR_DIM;
    p.tiles = (uint32_t)tiles;
    p.pieces = pieces;
    p.partial = a.workspace;
    by_type(pieces > 1 ? QESGD_F32 : a.dtype, [&](auto t) { k_mx4_product<S, t.value><<<p.tiles * pieces, S::threads, 0, a.stream>>>(p); });
    const int rc = launched();
    if (rc != QESGD_OK || pieces == 1) return rc;
    const uint64_t groups = ((uint64_t)p.M * p.N + 1023) / 1024;
    by_type(a.dtype, [&](auto t) { k_mx4_product_sum<t.value><<<(uint32_t)groups, 256, 0, a.stream>>>(p); });
    return launched();
}

// Which kernel, and how many pieces of the contraction, from how long the workgroups take on 256 CUs.  A step of 256 columns takes, us:
// 64 x 64 tiles 0.30 while a CU has one, 0.62 with two; 128 x 128 0.85 and 1.5; 256 x 256 1.2 on an empty chip, 2.3 on a full one.
// Measured over 26 shapes, us with 64 / 128 / 256:
//   64 x 4096 x 4096 6.9 / 13.4 / 26.2;  512 x 4096 x 4096 12.5 / 14.9 / 27.7;  1024 x 4096 x 4096 22.6 / 17.6 / 28.3;  4096 x 4096 x 4096
//   82.7 / 50.2 / 40.8;  3000 x 5000 x 700 26.8 / 19.9 / 16.0
// and the pieces, 64 x 64 in 1 / 4 / 8 / 16: 1 x 1000 x 25088 27.8 / 11.8 / 8.9 / 8.5;  512 x 1000 x 25088 28.4 / 21.8 / 25.0 / 31.5;
// 64 x 4096 x 4096 in 1 / 2 / 4 6.9 / 8.5 / 10.3.
// edge 0: k_mx4_product_few, up to 16 rows where every wave has one step at most.  Few / 64 x 64: 1 x 4096 x 4096 5.5 / 6.8, 16 x 4096 x 4096 6.5 / 6.8,
// 32 x 4096 x 4096 8.1 / 7.0, 1 x 16384 x 4096 10.6 / 7.5 (calls from Python: 4.9 is what the call itself takes).
struct Cut { uint32_t edge, pieces; };

double cut_us(uint64_t groups, uint32_t edge, uint64_t steps) {
    const uint64_t slots = edge == 256 ? 256 : 512, left = groups % slots;
    const double full = edge == 256 ? 2.3 : edge == 128 ? 1.5 : 0.62;
    const double last = left == 0 ? 0.0 : edge == 256 ? 1.2 + 1.1 * (double)left / 256.0 : left <= 256 ? (edge == 128 ? 0.85 : 0.30) : full;
    return ((double)(groups / slots) * full + last) * (double)steps + (double)((groups + slots - 1) / slots);
}

Cut choose_cut(uint64_t M, uint64_t N, uint64_t K) {
    const uint64_t steps = (K + 255) / 256;
    if (M <= kFewRows && steps <= kFewWaves && N <= kFewColumns) return Cut{0, 1};
    Cut best{64, 1};
    double least = 1e300;
    for (uint32_t edge : {64u, 128u, 256u}) {
        const uint64_t tiles = ((M + edge - 1) / edge) * ((N + edge - 1) / edge);
        // a piece has at least four steps; the sums of the pieces cost a launch, and are written and read at about 4 TB/s
        for (uint32_t pieces = 1; pieces <= 16 && (pieces == 1 || (pieces * 4 <= steps && tiles * pieces <= 1024)); ++pieces) {
            const double us = cut_us(tiles * pieces, edge, (steps + pieces - 1) / pieces) + (pieces == 1 ? 0.0 : 2.0 + (double)pieces * (double)(M * N) * 2e-6);
            if (us < least) {
                least = us;
                best = Cut{edge, pieces};
            }
        }
    }
    return best;
}

}  // namespace

size_t mx4_product_plan(Mx4Product& a) {
    const Cut cut = choose_cut(a.M, a.N, a.K);
    a.edge = cut.edge;
    a.pieces = cut.pieces;
    return cut.pieces > 1 ? cut.pieces * a.M * a.N * sizeof(float) : 0;
}

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
    const Cut cut{a.edge, a.pieces};
    switch (cut.edge) {
        case 0:
            by_type(a.dtype, [&](auto t) { k_mx4_product_few<t.value><<<(p.N + 31) / 32, kFewWaves * 64, 0, a.stream>>>(p); });
            return launched();
        case 64: return launch_tiles<TileShape<2, 2, 1, 1, 4>>(a, p, cut.pieces);
        case 128: return launch_tiles<TileShape<2, 2, 2, 2, 2>>(a, p, cut.pieces);
        default: return launch_tiles<TileShape<2, 4, 4, 2, 2>>(a, p, cut.pieces);
    }
}

}  // namespace qesgd
