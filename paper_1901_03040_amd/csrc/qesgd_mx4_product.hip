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
    uint32_t tiles_m, tiles_n;
};

template <uint32_t DT>
__device__ __forceinline__ void put(void* c, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)c)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)c)[at] = (_Float16)v;
    else ((__bf16*)c)[at] = (__bf16)v;
}

template <class S, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_mx4_product(const PParams p) {
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t t = tile_of_workgroup(blockIdx.x, gridDim.x);
    const uint32_t tm = t % p.tiles_m, tn = t / p.tiles_m;
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN;
    const unsigned char* a = p.a + (uint64_t)m0 * p.row_codes;
    const unsigned char* b = p.b + (uint64_t)n0 * p.row_codes;
    TileLoader<S::BM, S::threads> la;
    TileLoader<S::BN, S::threads> lb;
    la.init(p.row_codes, p.M - m0);
    lb.init(p.row_codes, p.N - n0);
    const uint32_t steps = (p.row_codes + 127u) / 128u;
    const bool ragged = (p.row_codes & 127u) != 0;

    const unsigned char* sa[S::FM];
    const unsigned char* sb[S::FN];
#pragma unroll
    for (int f = 0; f < S::FM; ++f) sa[f] = p.a_scales + (uint64_t)min(m0 + (wm * S::FM + f) * 32u + (lane & 31u), p.M - 1u) * p.row_scales;
#pragma unroll
    for (int f = 0; f < S::FN; ++f) sb[f] = p.b_scales + (uint64_t)min(n0 + (wn * S::FN + f) * 32u + (lane & 31u), p.N - 1u) * p.row_scales;

    acc16 acc[S::FM][S::FN] = {};
    uint32_t at[4];                               // a lane's four chunks of a row
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) at[s] = (lane & 31u) * 128u + (((2u * s + h) ^ (lane & 7u)) * 16u);

    uint32_t ra[S::FM][2], rb[S::FN][2], xa[S::FM][2], xb[S::FN][2];      // scales: on their way, and of this step
    auto fetch = [&](uint32_t step, unsigned char* to) {
        const bool half = ragged && step + 1 == steps;
        // 256 columns have 8 scale bytes a row; the half step at the end has 4 and takes them twice
        const uint32_t o0 = step * 8u, o1 = o0 + (half ? 0u : 4u);
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { ra[f][0] = *(const uint32_t*)(sa[f] + o0); ra[f][1] = *(const uint32_t*)(sa[f] + o1); }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { rb[f][0] = *(const uint32_t*)(sb[f] + o0); rb[f][1] = *(const uint32_t*)(sb[f] + o1); }
        la.load(a + (uint64_t)step * 128u, to, half);
        lb.load(b + (uint64_t)step * 128u, to + S::BM * kStepBytes, half);
    };
    // A lane's blocks of a step are scale bytes 2 s + h of its row: a shift by 8 h brings them to bytes 0 and 2 of the two words.
    auto scales = [&]() {
#pragma unroll
        for (int f = 0; f < S::FM; ++f) { xa[f][0] = ra[f][0] >> (8u * h); xa[f][1] = ra[f][1] >> (8u * h); }
#pragma unroll
        for (int f = 0; f < S::FN; ++f) { xb[f][0] = rb[f][0] >> (8u * h); xb[f][1] = rb[f][1] >> (8u * h); }
    };
    auto compute = [&](uint32_t step, const unsigned char* from) {
        const bool half = ragged && step + 1 == steps;
        const unsigned char* fa = from + wm * S::FM * 32 * kStepBytes;
        const unsigned char* fb = from + (S::BM + wn * S::FN * 32) * kStepBytes;
        auto part = [&](auto s_) {
            constexpr int s = decltype(s_)::value;
            int8v va[S::FM], vb[S::FN];
#pragma unroll
            for (int f = 0; f < S::FM; ++f) {
                const int4v v = *(const int4v*)(fa + f * 4096 + at[s]);
                va[f] = int8v{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int f = 0; f < S::FN; ++f) {
                const int4v v = *(const int4v*)(fb + f * 4096 + at[s]);
                vb[f] = int8v{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va[i], vb[j], acc[i][j], 4, 4, (s & 1) * 2,
                                                                               (int)xa[i][s >> 1], (s & 1) * 2, (int)xb[j][s >> 1]);
        };
        part(std::integral_constant<int, 0>{});
        part(std::integral_constant<int, 1>{});
        if (!half) {
            part(std::integral_constant<int, 2>{});
            part(std::integral_constant<int, 3>{});
        }
    };

    fetch(0, lds0);
    uint32_t step = 0;
    for (;;) {
        __syncthreads();
        scales();
        if (step + 1 < steps) fetch(step + 1, lds1);
        compute(step, lds0);
        if (++step == steps) break;
        __syncthreads();
        scales();
        if (step + 1 < steps) fetch(step + 1, lds0);
        compute(step, lds1);
        if (++step == steps) break;
    }

    // a lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const uint32_t col = n0 + (wn * S::FN + j) * 32u + (lane & 31u);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t row = m0 + (wm * S::FM + i) * 32u + 8u * (e >> 2) + 4u * h + (e & 3);
                if (row < p.M && col < p.N) put<DT>(p.c, (uint64_t)row * p.ldc + col, acc[i][j][e]);
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
    return launch_product_as<TileShape<2, 2, 2, 2>>(a, p);
}

}  // namespace qesgd
