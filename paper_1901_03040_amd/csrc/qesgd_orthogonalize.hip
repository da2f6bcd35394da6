// Orthogonalising an update by Newton-Schulz products, with the momentum before it and the update behind it.
//
//   x = momentum step of g;  X = x / (||x||_F + eps);  a step:  G = X X^T,  P = a I + b G + c G G,  X = P X
//
// X is taken with its shorter side first (m x n, m <= n), so G and P are m x m; the transposed case only swaps the names.
//
// Arithmetic.  The iteration has to hold fp32 accuracy: small singular values grow by up to a^steps (485 for the usual
// coefficients), and rounding errors with them.  The card's fp32 matrix rate is a sixteenth of its fp16 rate, so every operand is
// held as hi + lo, two fp16 numbers with 22 bits between them, scaled by a power of two into fp16's range, and a product is
// hi hi + hi lo + lo hi with fp32 sums: three fp16 products, five times the fp32 rate, and as far from 64 bits as fp32 products are
// (2e-6 .. 3e-6 either way).  One fp16 product alone would cost three digits.
//
// Layout of an operand ("split"): rows along the contraction, padded with zeros to a multiple of 32; 32 numbers' hi (64 bytes),
// then their lo, so a step of the pipeline is one 128-byte line of each row.  Products have both operands' rows along the
// contraction, which takes X for X X^T and its transpose for P X: the last product's epilogue writes both.  G and P are symmetric:
// only tiles on and above the diagonal are computed, and the epilogue writes them twice.
#include <type_traits>

#include "qesgd_device.h"
#include "qesgd_matrix.h"
#include "qesgd_tile_product.h"

namespace qesgd {
namespace {

constexpr float kScaleX = 4096.0f;      // of X's entries (at most 1 at first; singular values near 1 keep them there): below 16
constexpr float kScaleG = 4096.0f;      // of G's
constexpr float kScaleP = 2048.0f;      // of P's: below 32

inline uint64_t split_pitch(uint64_t k) { return round_up_to(k, 32) * 4; }

// hi and lo of a scaled number.  What is below 2^-24 in scaled units is lost: 2^-36 of the largest entries.
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}
// Byte of number k of a row.
__device__ __forceinline__ uint64_t split_at(uint32_t k) { return (uint64_t)(k >> 5) * 128u + (k & 31u) * 2u; }

template <uint32_t DT>
__device__ __forceinline__ float fetch(const void* x, uint64_t at) {
    if (DT == QESGD_F32) return ((const float*)x)[at];
    if (DT == QESGD_F16) return (float)((const _Float16*)x)[at];
    return (float)((const __bf16*)x)[at];
}

struct SParams {                         // the passes before the iteration
    const void* x;
    float* momentum;
    double* partial;                     // [n][parts]
    uint64_t d;                          // rows * cols
    uint32_t rows, cols, parts;
    float mu, eps;
    bool nesterov;
    unsigned char* X;                    // rows along the longer side: m x n
    unsigned char* Xt;
    uint64_t X_bytes, Xt_bytes;          // of one matrix
    uint32_t X_pitch, Xt_pitch;
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Momentum, and the partial sums of squares of x in fp64 (any fp32 magnitude squares into range).  Bound by the stream of g and m.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_orthogonal_momentum(const SParams p) {
    const uint64_t base = (uint64_t)blockIdx.y * p.d;
    double sum = 0.0;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < p.d; i += (uint64_t)p.parts * 256u) {
        float v = fetch<DT>(p.x, base + i);
        if (p.momentum) {
            const float m = p.mu * p.momentum[base + i] + v;
            p.momentum[base + i] = m;
            v = p.nesterov ? v + p.mu * m : m;
        }
        sum += (double)v * (double)v;
    }
    __shared__ double part[4];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.partial[(uint64_t)blockIdx.y * p.parts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// X and its transpose, split, from a 64 x 64 tile of x.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_orthogonal_split(const SParams p) {
    __shared__ float tile[64][65];
    __shared__ double part[4];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < p.parts; i += 256u) sum += p.partial[(uint64_t)blockIdx.z * p.parts + i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    const double norm = sqrt(sum) + (double)p.eps;
    const double scale = norm > 0.0 ? (double)kScaleX / norm : 0.0;     // beyond fp32 where x is subnormal

    const uint32_t r0 = blockIdx.y * 64u, c0 = blockIdx.x * 64u;
    const uint64_t base = (uint64_t)blockIdx.z * p.d;
    const uint32_t tx = threadIdx.x & 63u, ty = threadIdx.x >> 6;
    for (uint32_t i = ty; i < 64u; i += 4u) {
        float v = 0.0f;
        if (r0 + i < p.rows && c0 + tx < p.cols) {
            const uint64_t at = base + (uint64_t)(r0 + i) * p.cols + c0 + tx;
            v = fetch<DT>(p.x, at);
            if (p.momentum) v = p.nesterov ? v + p.mu * p.momentum[at] : p.momentum[at];
        }
        tile[i][tx] = (float)((double)v * scale);
    }
    __syncthreads();
    // rows of x: those of X where rows <= cols, of its transpose otherwise
    const bool turned = p.rows > p.cols;
    unsigned char* rowwise = (turned ? p.Xt + blockIdx.z * p.Xt_bytes : p.X + blockIdx.z * p.X_bytes);
    unsigned char* colwise = (turned ? p.X + blockIdx.z * p.X_bytes : p.Xt + blockIdx.z * p.Xt_bytes);
    const uint32_t pr = turned ? p.Xt_pitch : p.X_pitch, pc = turned ? p.X_pitch : p.Xt_pitch;
    for (uint32_t i = ty; i < 64u; i += 4u) {
        _Float16 hi, lo;
        if (r0 + i < p.rows && (c0 + tx) * 4u < pr) {
            split(tile[i][tx], hi, lo);
            unsigned char* to = rowwise + (uint64_t)(r0 + i) * pr + split_at(c0 + tx);
            *(_Float16*)to = hi;
            *(_Float16*)(to + 64) = lo;
        }
        if (c0 + i < p.cols && (r0 + tx) * 4u < pc) {
            split(tile[tx][i], hi, lo);
            unsigned char* to = colwise + (uint64_t)(c0 + i) * pc + split_at(r0 + tx);
            *(_Float16*)to = hi;
            *(_Float16*)(to + 64) = lo;
        }
    }
}

enum { kGram = 0, kPoly = 1, kApply = 2, kFinal = 3 };

struct OParams {
    const unsigned char* a;              // M rows
    const unsigned char* b;              // N rows
    uint64_t a_bytes, b_bytes;           // of one matrix of the batch
    uint32_t M, N, steps, pitch;         // pitch of a and b: the same contraction
    uint32_t tiles_m, tiles_n, tiles;
    unsigned char* d1;                   // C, split
    unsigned char* d2;                   // its transpose, split
    uint64_t d1_bytes, d2_bytes;
    uint32_t d1_pitch, d2_pitch;
    float scale;                         // of the sums, into the output's scale
    float ca, cb;                        // kPoly: on the diagonal, and of G
    // kFinal: [n, M, N] outputs
    void* out;
    float* z;
    const float* w;
    float* u;
    float* zsum;
};

// Tile number t of the upper triangle, column by column.
__device__ __forceinline__ void upper_tile(uint32_t t, uint32_t& i, uint32_t& j) {
    j = (uint32_t)((__builtin_sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((j + 1u) * (j + 2u) / 2u <= t) ++j;
    while (j * (j + 1u) / 2u > t) --j;
    i = t - j * (j + 1u) / 2u;
}

template <class S, int KIND, uint32_t DT>
__global__ void __launch_bounds__(S::threads) k_orthogonal_product(const OParams p) {
    static_assert(S::BM == S::BN, "symmetric products take square tiles");
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t t = tile_of_workgroup(blockIdx.x, gridDim.x), z = blockIdx.y;
    uint32_t tm, tn;
    if (KIND == kGram || KIND == kPoly) {
        upper_tile(t, tm, tn);
    } else {
        tm = t % p.tiles_m;
        tn = t / p.tiles_m;
    }
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN;
    const unsigned char* a = p.a + z * p.a_bytes + (uint64_t)m0 * p.pitch;
    const unsigned char* b = p.b + z * p.b_bytes + (uint64_t)n0 * p.pitch;
    TileLoader<S::BM, S::threads> la;
    TileLoader<S::BN, S::threads> lb;
    la.init(p.pitch, p.M - m0);
    lb.init(p.pitch, p.N - n0);

    acc16 acc[S::FM][S::FN] = {};
    uint32_t at[4];                              // a lane's chunks of a row: hi of either half of the step, lo of either half
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) at[s] = (lane & 31u) * 128u + (((2u * s + h) ^ (lane & 7u)) * 16u);

    auto load = [&](uint32_t step, unsigned char* to) {
        la.load(a + (uint64_t)step * kStepBytes, to, false);
        lb.load(b + (uint64_t)step * kStepBytes, to + S::BM * kStepBytes, false);
    };
    auto compute = [&](const unsigned char* from) {
        const unsigned char* fa = from + wm * S::FM * 32 * kStepBytes;
        const unsigned char* fb = from + (S::BM + wn * S::FN * 32) * kStepBytes;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            half8 ah[S::FM], al[S::FM], bh[S::FN], bl[S::FN];
#pragma unroll
            for (int f = 0; f < S::FM; ++f) { ah[f] = *(const half8*)(fa + f * 4096 + at[s]); al[f] = *(const half8*)(fa + f * 4096 + at[s + 2]); }
#pragma unroll
            for (int f = 0; f < S::FN; ++f) { bh[f] = *(const half8*)(fb + f * 4096 + at[s]); bl[f] = *(const half8*)(fb + f * 4096 + at[s + 2]); }
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah[i], bh[j], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah[i], bl[j], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al[i], bh[j], acc[i][j], 0, 0, 0);
        }
    };

    load(0, lds0);
    for (uint32_t step = 0;;) {
        __syncthreads();
        if (step + 1 < p.steps) load(step + 1, lds1);
        compute(lds0);
        if (++step == p.steps) break;
        __syncthreads();
        if (step + 1 < p.steps) load(step + 1, lds0);
        compute(lds1);
        if (++step == p.steps) break;
    }

    // A lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r, r = 0..3.
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const uint32_t col = n0 + (wn * S::FN + j) * 32u + (lane & 31u);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t row = m0 + (wm * S::FM + i) * 32u + 8u * q + 4u * h;
                if (KIND == kFinal) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (row + r >= p.M || col >= p.N) continue;
                        const uint64_t o = ((uint64_t)z * p.M + row + r) * p.N + col;
                        const float v = acc[i][j][4 * q + r] * p.scale;
                        if (p.out) {
                            if (DT == QESGD_F32) ((float*)p.out)[o] = v;
                            else if (DT == QESGD_F16) ((_Float16*)p.out)[o] = (_Float16)v;
                            else ((__bf16*)p.out)[o] = (__bf16)v;
                        }
                        if (p.z) {
                            const float zv = p.z[o] + v;
                            p.z[o] = zv;
                            if (p.u) p.u[o] = p.w[o] + zv;
                            if (p.zsum) p.zsum[o] += zv;
                        }
                    }
                    continue;
                }
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * q + r] * p.scale;
                if (KIND == kPoly && col < p.N && row < p.M) {
                    // G[row.., col] = G[col, row..]: four in a row; its padding is there and zero
                    const unsigned char* g = p.a + z * p.a_bytes + (uint64_t)col * p.pitch + split_at(row);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float gv = (float)((const _Float16*)g)[r] + (float)((const _Float16*)(g + 64))[r];
                        v[r] = v[r] + p.cb * gv + (row + r == col ? p.ca : 0.0f);
                    }
                }
                _Float16 hi[4], lo[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) split(row + r < p.M && col < p.N ? v[r] : 0.0f, hi[r], lo[r]);
                if (col < p.N && row * 4u < p.d2_pitch) {
                    unsigned char* to = p.d2 + z * p.d2_bytes + (uint64_t)col * p.d2_pitch + split_at(row);
#pragma unroll
                    for (int r = 0; r < 4; ++r) { ((_Float16*)to)[r] = hi[r]; ((_Float16*)(to + 64))[r] = lo[r]; }
                }
                if (KIND == kApply || tm != tn) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (row + r < p.M && col * 4u < p.d1_pitch) {
                            unsigned char* to = p.d1 + z * p.d1_bytes + (uint64_t)(row + r) * p.d1_pitch + split_at(col);
                            *(_Float16*)to = hi[r];
                            *(_Float16*)(to + 64) = lo[r];
                        }
                    }
                }
            }
        }
}

// Workspace: partial sums, X, two of its transpose, G, P.
struct Plan {
    uint64_t m, n;                       // shorter and longer side
    uint32_t parts;
    uint64_t X_pitch, Xt_pitch, G_pitch, X_bytes, Xt_bytes, G_bytes;
    uint64_t X, Xt[2], G, P, total;
};

Plan make_plan(uint64_t rows, uint64_t cols, uint32_t count) {
    Plan p{};
    p.m = rows < cols ? rows : cols;
    p.n = rows < cols ? cols : rows;
    const uint64_t d = rows * cols;
    p.parts = (uint32_t)((d + 4095) / 4096 < 512 ? (d + 4095) / 4096 : 512);
    p.X_pitch = split_pitch(p.n);
    p.Xt_pitch = p.G_pitch = split_pitch(p.m);
    p.X_bytes = p.m * p.X_pitch;
    p.Xt_bytes = p.n * p.Xt_pitch;
    p.G_bytes = p.m * p.G_pitch;
    uint64_t at = round_up_to((uint64_t)count * p.parts * sizeof(double), 256);
    auto take = [&](uint64_t bytes) { const uint64_t here = at; at += round_up_to(bytes * count, 256); return here; };
    p.X = take(p.X_bytes);
    p.Xt[0] = take(p.Xt_bytes);
    p.Xt[1] = take(p.Xt_bytes);
    p.G = take(p.G_bytes);
    p.P = take(p.G_bytes);
    p.total = at;
    return p;
}

template <class S, int KIND, uint32_t DT>
int launch_product(OParams& p, uint32_t count, hipStream_t stream) {
    p.tiles_m = (p.M + S::BM - 1) / S::BM;
    p.tiles_n = (p.N + S::BN - 1) / S::BN;
    p.steps = p.pitch / kStepBytes;
    const uint64_t tiles = KIND == kGram || KIND == kPoly ? (uint64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (uint64_t)p.tiles_m * p.tiles_n;
    if (tiles >= (1ull << 31)) return QESGD_ERR_DIM;
    k_orthogonal_product<S, KIND, DT><<<dim3((uint32_t)tiles, count), S::threads, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

template <uint32_t DT>
int launch_type(const Orthogonalize& a) {
    typedef TileShape<2, 2, 2, 2> S;
    const Plan pl = make_plan(a.rows, a.cols, a.n);
    const bool turned = a.rows > a.cols;
    SParams s{};
    s.x = a.x;
    s.momentum = a.momentum;
    s.partial = (double*)a.workspace;
    s.d = a.rows * a.cols;
    s.rows = (uint32_t)a.rows;
    s.cols = (uint32_t)a.cols;
    s.parts = pl.parts;
    s.mu = a.mu;
    s.eps = a.eps;
    s.nesterov = a.nesterov;
    s.X = a.workspace + pl.X;
    s.Xt = a.workspace + pl.Xt[0];
    s.X_bytes = pl.X_bytes;
    s.Xt_bytes = pl.Xt_bytes;
    s.X_pitch = (uint32_t)pl.X_pitch;
    s.Xt_pitch = (uint32_t)pl.Xt_pitch;
    k_orthogonal_momentum<DT><<<dim3(pl.parts, a.n), 256, 0, a.stream>>>(s);
    k_orthogonal_split<DT><<<dim3((uint32_t)((a.cols + 63) / 64), (uint32_t)((a.rows + 63) / 64), a.n), 256, 0, a.stream>>>(s);

    for (uint32_t i = 0; i < a.steps; ++i) {
        const float ca = a.coeffs[3 * i], cb = a.coeffs[3 * i + 1], cc = a.coeffs[3 * i + 2];
        unsigned char* const Xt = a.workspace + pl.Xt[i & 1];
        OParams g{};
        g.a = g.b = a.workspace + pl.X;
        g.a_bytes = g.b_bytes = pl.X_bytes;
        g.M = g.N = (uint32_t)pl.m;
        g.pitch = (uint32_t)pl.X_pitch;
        g.d1 = g.d2 = a.workspace + pl.G;
        g.d1_bytes = g.d2_bytes = pl.G_bytes;
        g.d1_pitch = g.d2_pitch = (uint32_t)pl.G_pitch;
        g.scale = kScaleG / (kScaleX * kScaleX);
        int rc = launch_product<S, kGram, 0>(g, a.n, a.stream);
        if (rc != QESGD_OK) return rc;
        OParams q = g;
        q.a = q.b = a.workspace + pl.G;
        q.a_bytes = q.b_bytes = pl.G_bytes;
        q.pitch = (uint32_t)pl.G_pitch;
        q.d1 = q.d2 = a.workspace + pl.P;
        q.scale = cc * (kScaleP / (kScaleG * kScaleG));
        q.ca = ca * kScaleP;
        q.cb = cb * (kScaleP / kScaleG);
        rc = launch_product<S, kPoly, 0>(q, a.n, a.stream);
        if (rc != QESGD_OK) return rc;
        OParams x{};
        x.a = a.workspace + pl.P;
        x.a_bytes = pl.G_bytes;
        x.M = (uint32_t)pl.m;
        x.b = Xt;
        x.b_bytes = pl.Xt_bytes;
        x.N = (uint32_t)pl.n;
        x.pitch = (uint32_t)pl.G_pitch;
        if (i + 1 < a.steps) {
            x.d1 = a.workspace + pl.X;
            x.d1_bytes = pl.X_bytes;
            x.d1_pitch = (uint32_t)pl.X_pitch;
            x.d2 = a.workspace + pl.Xt[(i + 1) & 1];
            x.d2_bytes = pl.Xt_bytes;
            x.d2_pitch = (uint32_t)pl.Xt_pitch;
            x.scale = 1.0f / kScaleP;
            rc = launch_product<S, kApply, 0>(x, a.n, a.stream);
        } else {
            if (turned) {                // (P X)^T = Xt P, rows as the caller has them
                OParams y = x;
                y.a = x.b; y.a_bytes = x.b_bytes; y.M = x.N;
                y.b = x.a; y.b_bytes = x.a_bytes; y.N = x.M;
                x = y;
            }
            x.scale = a.alpha / (kScaleP * kScaleX);
            x.out = a.out;
            x.z = a.z;
            x.w = a.w;
            x.u = a.u;
            x.zsum = a.zsum;
            rc = launch_product<S, kFinal, DT>(x, a.n, a.stream);
        }
        if (rc != QESGD_OK) return rc;
    }
    return QESGD_OK;
}

}  // namespace

size_t orthogonalize_workspace(uint64_t rows, uint64_t cols, uint32_t n) { return make_plan(rows, cols, n).total; }

int launch_orthogonalize(const Orthogonalize& a) {
    switch (a.dtype) {
        case QESGD_F32: return launch_type<QESGD_F32>(a);
        case QESGD_BF16: return launch_type<QESGD_BF16>(a);
        default: return launch_type<QESGD_F16>(a);
    }
}

}  // namespace qesgd
