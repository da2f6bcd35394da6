// C = A B^T of two packed 4-bit matrices on the scaled matrix instruction: a lane's operand is 32 elements of one row, which is one
// block of the format, next to its scale byte, so nothing is unpacked.  Element products are exact, sums are fp32.
#include "qesgd_mx4_tiles.h"

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
    ops.init_scales(p.a_scales + (uint64_t)m0 * p.row_scales + first * 8u, p.b_scales + (uint64_t)n0 * p.row_scales + first * 8u, p.M - m0, p.N - n0,
                    p.row_scales, p.row_scales - first * 8u, wm, wn);
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

// Which kernel, and how many pieces of the contraction, from how long the workgroups take (tile_us).
// Measured over 26 shapes, us with 64 / 128 / 256:
//   64 x 4096 x 4096 6.9 / 13.4 / 26.2;  512 x 4096 x 4096 12.5 / 14.9 / 27.7;  1024 x 4096 x 4096 22.6 / 17.6 / 28.3;  4096 x 4096 x 4096
//   82.7 / 50.2 / 40.8;  3000 x 5000 x 700 26.8 / 19.9 / 16.0
// and the pieces, 64 x 64 in 1 / 4 / 8 / 16: 1 x 1000 x 25088 27.8 / 11.8 / 8.9 / 8.5;  512 x 1000 x 25088 28.4 / 21.8 / 25.0 / 31.5;
// 64 x 4096 x 4096 in 1 / 2 / 4 6.9 / 8.5 / 10.3.
// edge 0: k_mx4_product_few, up to 16 rows where every wave has one step at most.  Few / 64 x 64: 1 x 4096 x 4096 5.5 / 6.8, 16 x 4096 x 4096 6.5 / 6.8,
// 32 x 4096 x 4096 8.1 / 7.0, 1 x 16384 x 4096 10.6 / 7.5 (calls from Python: 4.9 is what the call itself takes).
struct Cut { uint32_t edge, pieces; };

Cut choose_cut(uint64_t M, uint64_t N, uint64_t K) {
    const uint64_t steps = (K + 255) / 256;
    if (M <= kFewRows && steps <= kFewWaves && N <= kFewColumns) return Cut{0, 1};
    Cut best{64, 1};
    double least = 1e300;
    for (uint32_t edge : {64u, 128u, 256u}) {
        const uint64_t tiles = ((M + edge - 1) / edge) * ((N + edge - 1) / edge);
        // a piece has at least four steps; the sums of the pieces cost a launch, and are written and read at about 4 TB/s
        for (uint32_t pieces = 1; pieces <= 16 && (pieces == 1 || (pieces * 4 <= steps && tiles * pieces <= 1024)); ++pieces) {
            const double us = tile_us(tiles * pieces, edge, (double)((steps + pieces - 1) / pieces)) + (pieces == 1 ? 0.0 : 2.0 + (double)pieces * (double)(M * N) * 2e-6);
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
