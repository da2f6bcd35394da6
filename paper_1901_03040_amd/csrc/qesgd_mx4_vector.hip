// Rows of a few tokens times packed 4-bit matrices, the rows as they are.
//
//   y[r, n] = sum_k x[row, k] W_e[n, k]
//
// What bounds it is the reading of W: 17/32 of a byte an element.  A lane takes one block of a row of W, 16 bytes and a scale, and the conversion makes
// 32 bf16 numbers of it, which have room for the sign, the two bits and the scale: no rounding.  x is written as a sum of bf16 numbers
// (one for bf16, two for f16's 11 bits, three for f32's 24), each a row of its own for the matrix instruction, whose 16 rows
// would stand empty otherwise; so all products are exact and a single row of f32 costs no more instructions than one of bf16.
//
// A wave owns 16 rows of W and takes steps of 128 columns; the waves of a workgroup share the columns among them, and their sums are added
// in order.  The rows of x go to LDS once, split.
#include "qesgd_experts.h"
#include "qesgd_groups.h"
#include "qesgd_launch.h"
#include "qesgd_mx4_codes.h"

namespace qesgd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float acc4 __attribute__((ext_vector_type(4)));

struct VParams {
    const void* x;
    uint64_t ld;
    uint32_t T;
    const int32_t* order;
    uint32_t per;
    const unsigned char* w;
    uint64_t w_stride, scales_off;
    const int32_t* offsets;
    uint32_t E, R, N, K;
    uint32_t row_codes, row_scales;
    void* y;
    uint64_t ldy;
    uint32_t splits;                  // waves that share a row's columns: 1 .. kVWaves
    uint32_t part_columns;            // columns of x that lie in LDS at a time, a multiple of 128 * splits
    uint32_t lds_rows;
};

constexpr uint32_t kVWaves = 16;

template <uint32_t DT>
__device__ __forceinline__ void put_row(void* y, uint64_t at, float v) {
    if (DT == QESGD_F32) ((float*)y)[at] = v;
    else if (DT == QESGD_F16) ((_Float16*)y)[at] = (_Float16)v;
    else ((__bf16*)y)[at] = (__bf16)v;
}

// The upper 16 bits of v: a bf16 number no larger than v, so that nothing overflows.
__device__ __forceinline__ uint32_t upper(float v) { return __float_as_uint(v) & 0xFFFF0000u; }

// Eight elements as PARTS times eight bf16 numbers, the largest parts first.  Infinities and NaN are whole in the first one.
template <uint32_t DT, uint32_t PARTS>
__device__ __forceinline__ void split(const Eight<DT>& x, uvec4 (&out)[PARTS]) {
    if constexpr (DT == QESGD_BF16) {
        out[0] = x.v;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            uint32_t part[2][PARTS];
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                float v = x.at(2 * i + h);
                const bool fine = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
                for (uint32_t q = 0; q < PARTS; ++q) {
                    part[h][q] = upper(v);
                    v = v - __uint_as_float(part[h][q]);
                }
                if (!fine) {
                    part[h][0] = x.at(2 * i + h) != x.at(2 * i + h) ? 0x7FC00000u : part[h][0];
#pragma unroll
                    for (uint32_t q = 1; q < PARTS; ++q) part[h][q] = 0u;
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < PARTS; ++q) out[q][i] = part[0][q] >> 16 | part[1][q];
        }
    }
}

// The 32 bf16 numbers of a block as four operands of eight.
__device__ __forceinline__ void block_values(const uvec4& codes, uint32_t byte, bf16x8 (&out)[4]) {
    const float scale = __uint_as_float(byte << 23);              // the conversion reads the exponent field; 255 gives NaN
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = codes[i];
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
        out[i] = bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    }
}

template <uint32_t DT>
__global__ void __launch_bounds__(kVWaves * 64) k_mx4_vector_product(const VParams p) {
    constexpr uint32_t PARTS = DT == QESGD_F32 ? 3 : DT == QESGD_F16 ? 2 : 1, ROWS = 16 / PARTS;
    extern __shared__ __attribute__((aligned(16))) unsigned char rows_lds[];            // [lds_rows][part_columns bf16 and 16 bytes]
    __shared__ __attribute__((aligned(16))) float sums[kVWaves][4][64];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t l = lane & 15u, block = lane >> 4;
    const uint32_t e = blockIdx.y;
    uint32_t lo = 0, hi = p.R;
    if (p.offsets) {
        lo = held(p.offsets[e], p.R);
        hi = held(p.offsets[e + 1u], p.R);
        if (lo >= hi) return;
    }
    const uint32_t share = wave % p.splits, n0 = (blockIdx.x * (kVWaves / p.splits) + wave / p.splits) * 16u;
    const unsigned char* w = p.w + e * p.w_stride;
    const uint32_t row = min(n0 + l, p.N - 1u);
    const unsigned char* codes = w + (uint64_t)row * p.row_codes + block * 16u;
    const unsigned char* scales = w + p.scales_off + (uint64_t)row * p.row_scales + block;
    const uint32_t steps = p.row_codes / 64u, pitch = p.part_columns * 2u + 16u;
    for (uint32_t r0 = lo; r0 < hi; r0 += ROWS) {
        const uint32_t rows = min(ROWS, hi - r0);
        acc4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t c0 = 0; c0 < steps * 128u; c0 += p.part_columns) {
            const uint32_t here = min(p.part_columns, steps * 128u - c0), eights = here / 8u;
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < rows * eights; i += kVWaves * 64u) {
                const uint32_t r = i / eights, col = (i - r * eights) * 8u;
                const int32_t pair = p.order ? p.order[r0 + r] : (int32_t)(r0 + r);
                const uint32_t s = pair < 0 ? p.T : p.per == 1 ? (uint32_t)pair : (uint32_t)pair / p.per;
                const uint32_t n = s >= p.T || c0 + col >= p.K ? 0u : min(p.K - c0 - col, 8u);
                Eight<DT> v;
                v.load(p.x, n ? s * p.ld + c0 + col : 0u, n);
                uvec4 parts[PARTS];
                split<DT, PARTS>(v, parts);
#pragma unroll
                for (uint32_t q = 0; q < PARTS; ++q) *(uvec4*)(rows_lds + (r * PARTS + q) * pitch + col * 2u) = parts[q];
            }
            __syncthreads();
            // rows of the instruction beyond those there are read the last one: what comes of them is not stored
            const unsigned char* x = rows_lds + min(l, rows * PARTS - 1u) * pitch + block * 64u;
            for (uint32_t s = share; s < here / 128u; s += p.splits) {
                const uint32_t step = c0 / 128u + s;
                const uvec4 c = *(const uvec4*)(codes + step * 64u);
                const uint32_t byte = scales[step * 4u];
                bf16x8 b[4];
                block_values(c, byte, b);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)(x + s * 256u + i * 16u), b[i], acc, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[wave][i][lane] = acc[i];
        __syncthreads();
        // sums[wave][i][lane]: row 4 * (lane / 16) + i of the instruction, column lane % 16
        for (uint32_t i = threadIdx.x; i < (kVWaves / p.splits) * 16u * rows; i += kVWaves * 64u) {
            const uint32_t col = i & 15u, r = (i >> 4) % rows, set = (i >> 4) / rows;
            const uint32_t n = (blockIdx.x * (kVWaves / p.splits) + set) * 16u + col;
            if (n >= p.N) continue;
            float v = 0.0f;
            for (int q = PARTS - 1; q >= 0; --q) {
                const uint32_t m = r * PARTS + q;
                for (uint32_t s = 0; s < p.splits; ++s) v += sums[set * p.splits + s][m & 3u][(m >> 2) * 16u + col];
            }
            put_row<DT>(p.y, (uint64_t)(r0 + r) * p.ldy + n, v);
        }
    }
}

}  // namespace

size_t vector_product_workspace(const VectorProduct&) { return 0; }

int launch_vector_product(const VectorProduct& a) {
    qesgd_mx4_layout W;
    if (const int rc = make_mx4_layout(a.N, a.K, &W); rc != QESGD_OK) return rc;
    VParams p{};
    p.x = a.x;
    p.ld = a.ld;
    p.T = (uint32_t)a.T;
    p.order = a.order;
    p.per = a.per;
    p.w = a.w;
    p.w_stride = a.w_stride;
    p.scales_off = W.scales_off;
    p.offsets = a.offsets;
    p.E = a.E;
    p.R = (uint32_t)a.R;
    p.N = (uint32_t)a.N;
    p.K = (uint32_t)a.K;
    p.row_codes = (uint32_t)W.row_codes;
    p.row_scales = (uint32_t)W.row_scales;
    p.y = a.y;
    p.ldy = a.ldy;
    const uint32_t steps = p.row_codes / 64u, parts = a.dtype == QESGD_F32 ? 3 : a.dtype == QESGD_F16 ? 2 : 1, rows = 16 / parts;
    p.splits = 1;
    while (p.splits < kVWaves && p.splits * 2 <= steps) p.splits *= 2;
    p.lds_rows = parts * (a.R < rows ? (uint32_t)a.R : rows);
    // 60 KB for the rows, so that two workgroups with their sums fit a CU
    const uint32_t unit = 128u * p.splits, most = (60u * 1024u / p.lds_rows - 16u) / 2u / unit * unit, all = (steps * 128u + unit - 1) / unit * unit;
    p.part_columns = most < unit ? unit : most < all ? most : all;
    const uint32_t bytes = p.lds_rows * (p.part_columns * 2u + 16u);
    const uint32_t across = 16u * (kVWaves / p.splits), blocks = (p.N + across - 1) / across;
    const dim3 grid(blocks, a.E);
    if (!grid_ok((uint64_t)blocks * a.E, kVWaves * 64)) return QESGD_ERR_DIM;
    by_type(a.dtype, [&](auto t) { k_mx4_vector_product<t.value><<<grid, kVWaves * 64, bytes, a.stream>>>(p); });
    return launched();
}

}  // namespace qesgd
