// Orthogonalising an update by Newton-Schulz products, with the momentum before it and the update behind it.
//
//   x = momentum step of g;  X = x / (||x||_F + eps);  a step:  G = X X^T,  P = a I + b G + c G G,  X = P X
//
// X is taken with its shorter side first (m x n, m <= n), so G and P are m x m; the transposed case only swaps the names.
//
// Arithmetic.  The iteration has to hold fp32 accuracy: small singular values grow by up to a^steps (485 for the usual
// coefficients), and rounding errors with them.  The card's fp32 matrix rate is a sixteenth of its fp16 rate, so every operand is
// held as hi + lo / 2048, two fp16 numbers with 22 bits between them, scaled by a power of two into fp16's range, and a product is
// hi hi + (hi lo + lo hi) / 2048 with fp32 sums, one for either part: three fp16 products, five times the fp32 rate.  One fp16
// product alone would cost three digits.  What a pair of fp16 numbers cannot do is fp32's range: a number has its 22 bits down to 2^-14
// in scaled units, 2^-28 or 2^-29 of the largest there can be, below that a bit less for every halving, and nothing is left below 2^-36.
// Without the 2048 that began at 2^-3: a matrix with one large number lost the others' digits, 1.5e-4 of them with a ratio of 1e-6, and after ten steps, which make the
// small ones large, of the whole result (now 1.5e-6 and 1e-6).
//
// Layout of an operand ("split"): rows along the contraction, padded with zeros to a multiple of 32; 32 numbers' hi (64 bytes),
// then their lo, so a step of the pipeline is one 128-byte line of each row.  Products have both operands' rows along the
// contraction, which takes X for X X^T and its transpose for P X: the last product's epilogue writes both.  G and P are symmetric:
// only tiles on and above the diagonal are computed, and the epilogue writes them twice.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "qesgd_device.h"
#include "qesgd_matrix.h"
#include "qesgd_tile_product.h"

namespace qesgd {
namespace {

constexpr double kMostX = 16384.0, kMostP = 262144.0;       // 2^14: what X, G and G P may reach, 2^18: P
constexpr double kMostPair = 256.0;              // and a product of two P, whose range is that of both
constexpr float kFirstX = 32768.0f;              // scale of the first X, whose entries are at most 1

// The power of two that takes numbers up to `bound`, or up to `most` where that is less, to at most 2^15, half of fp16's range: rounding
// may pass the bound.
inline double scale_for(double bound, double most) {
    const double b = bound < most ? std::max(bound, std::ldexp(1.0, -40)) : most;
    return std::ldexp(1.0, 15 - (int)std::ceil(std::log2(b)));
}

// How large the operands of each step can be, from the coefficients alone.  The singular values of the first X are at most 1, its
// Frobenius norm; those of the next at most the largest |a s + b s^3 + c s^5| on the way, G's are their squares, P's at most the largest
// |a + b s^2 + c s^4|, and no entry of a matrix is larger than its largest singular value.  So the operands' scales are known before
// the first kernel, whatever the matrix, and use fp16's range from its upper end.
//
// A matrix can be far from these bounds: of m equal singular values each is m^(-1/2), and polynomials that do not bring them together take 1 and that
// to numbers many digits apart.  The scales therefore end at 2^14 and 2^18, where numbers are still held to 2^-37 (P to 2^-33): with bounds of 2^40
// there a 200 x 333 matrix and three such polynomials had no digit left.
struct Scales {
    double X[QESGD_MAX_STEPS + 1], G[QESGD_MAX_STEPS + 1], P[QESGD_MAX_STEPS];
    double T[QESGD_MAX_STEPS], PP[QESGD_MAX_STEPS];       // G P, and the product of this step's P and the next one's: 0 beyond kMostPair
};

inline Scales scales_of(const float* coeffs, uint32_t steps) {
    Scales r{};
    double S = 1.0, before = 0.0;
    for (uint32_t i = 0; i < steps; ++i) {
        const double a = coeffs[3 * i], b = coeffs[3 * i + 1], c = coeffs[3 * i + 2];
        const double s = S * (1.0 + 1.0 / 65536.0), end = s * s;      // rounding moves singular values by less than that
        double next = 0.0, most = std::abs(a);
        const auto at = [&](double u) {
            if (!(u > 0.0 && u <= end)) return;
            const double v = std::abs(a + u * (b + u * c));
            most = std::max(most, v);
            next = std::max(next, std::sqrt(u) * v);
        };
        // The ends of the range, and where (a + b u + c u^2)' or (s (a + b s^2 + c s^4))' = a + 3 b u + 5 c u^2 is zero; without a b or a c, or
        // without real roots, some of these are no numbers and no places.
        const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(9.0 * b * b - 20.0 * a * c), b));
        at(end);
        at(-b / (2.0 * c));
        at(q / (5.0 * c));
        at(a / q);
        r.X[i] = i == 0 ? (double)kFirstX : scale_for(S, kMostX);
        r.G[i] = scale_for(S * S, kMostX);
        r.T[i] = scale_for(S * next, kMostX);
        r.P[i] = scale_for(most, kMostP);
        if (i > 0 && before * most <= kMostPair) r.PP[i - 1] = scale_for(before * most, kMostPair);
        before = most;
        S = std::min(next, std::ldexp(1.0, 70));                       // beyond what is taken, and far from the end of 64 bits
    }
    r.X[steps] = scale_for(S, kMostX);
    r.G[steps] = scale_for(S * S, kMostX);
    return r;
}

inline uint64_t split_pitch(uint64_t k) { return round_up_to(k, 32) * 4; }

// hi and lo of a scaled number.  What hi leaves is at most 2^-11 of it, so lo stays in range.
constexpr float kLo = 2048.0f;
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = (_Float16)((v - (float)hi) * kLo);
}
typedef _Float16 half4 __attribute__((ext_vector_type(4)));

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

// Four elements from `at` on, any of them at any element's address.
typedef vec4 vec4_any __attribute__((aligned(4)));
template <uint32_t DT>
__device__ __forceinline__ vec4 fetch4(const void* x, uint64_t at) {
    if constexpr (DT == QESGD_F32) {
        return *(const vec4_any*)((const float*)x + at);
    } else {
        typedef uint32_t pairs __attribute__((ext_vector_type(2)));
        typedef pairs pairs_any __attribute__((aligned(2)));
        const pairs v = *(const pairs_any*)((const unsigned short*)x + at);
        const uint32_t a = v[0], b = v[1];
        if (DT == QESGD_BF16) return vec4{__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u)};
        const auto half = [](uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (unsigned short)bits); };
        return vec4{half(a), half(a >> 16), half(b), half(b >> 16)};
    }
}

// Momentum, and the partial sums of squares of x in fp64 (any fp32 magnitude squares into range).  Bound by the stream of g and m: four
// elements a lane.  4096 x 25088: 580 us one by one, 223 us so = 5.5 TB/s; two, four and eight loads a lane on their way 233, 233, 246.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_orthogonal_momentum(const SParams p) {
    const uint64_t base = (uint64_t)blockIdx.y * p.d, quads = p.d / 4;
    double sum = 0.0;
    const auto one = [&](float v, float& m) {
        if (p.momentum) {
            m = p.mu * m + v;
            v = p.nesterov ? v + p.mu * m : m;
        }
        sum += (double)v * (double)v;
    };
    for (uint64_t q = (uint64_t)blockIdx.x * 256u + threadIdx.x; q < quads; q += (uint64_t)p.parts * 256u) {
        const uint64_t at = base + q * 4;
        const vec4 g = fetch4<DT>(p.x, at);
        vec4 m = {};
        if (p.momentum) m = *(const vec4_any*)(p.momentum + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float me = m[e];
            one(g[e], me);
            m[e] = me;
        }
        if (p.momentum) *(vec4_any*)(p.momentum + at) = m;
    }
    if (blockIdx.x == 0 && threadIdx.x < (p.d & 3u)) {
        const uint64_t at = base + quads * 4 + threadIdx.x;
        float m = p.momentum ? p.momentum[at] : 0.0f;
        one(fetch<DT>(p.x, at), m);
        if (p.momentum) p.momentum[at] = m;
    }
    __shared__ double part[4];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.partial[(uint64_t)blockIdx.y * p.parts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// X and its transpose, split, from a 64 x 64 tile of x.  A lane reads and stores four numbers of a row.
// 4096 x 25088: 355 us with one, 332 with four stored at once, 271 us so; 1000 x 2049 of bf16 12.6 and 9.0.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_orthogonal_split(const SParams p) {
    __shared__ __attribute__((aligned(16))) float tile[64][68];
    __shared__ double part[4];
    const uint32_t r0 = blockIdx.y * 64u, c0 = blockIdx.x * 64u;
    const uint64_t base = (uint64_t)blockIdx.z * p.d;
    const uint32_t k4 = (threadIdx.x & 15u) * 4u, i16 = threadIdx.x >> 4;
    vec4 v[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t r = r0 + i16 + 16u * i, c = c0 + k4;
        const uint64_t at = base + (uint64_t)r * p.cols + c;
        v[i] = vec4{};
        if (r < p.rows && c + 4u <= p.cols) {
            if (!p.momentum || p.nesterov) v[i] = fetch4<DT>(p.x, at);
            if (p.momentum) {
                const vec4 m = *(const vec4_any*)(p.momentum + at);
                v[i] = p.nesterov ? v[i] + p.mu * m : m;
            }
        } else if (r < p.rows) {
#pragma unroll
            for (uint32_t e = 0; e < 3; ++e) {
                if (c + e >= p.cols) break;
                float one = p.momentum && !p.nesterov ? 0.0f : fetch<DT>(p.x, at + e);
                if (p.momentum) one = p.nesterov ? one + p.mu * p.momentum[at + e] : p.momentum[at + e];
                v[i][e] = one;
            }
        }
    }
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < p.parts; i += 256u) sum += p.partial[(uint64_t)blockIdx.z * p.parts + i];
    sum = wave_sum(sum);
    if ((threadIdx.x & 63u) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (part[0] + part[1]) + (part[2] + part[3]);
    const double norm = sqrt(sum) + (double)p.eps;
    const double scale = norm > 0.0 ? (double)kFirstX / norm : 0.0;     // beyond fp32 where x is subnormal
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        vec4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (float)((double)v[i][e] * scale);
        *(vec4*)&tile[i16 + 16u * i][k4] = y;
    }
    __syncthreads();
    // rows of x: those of X where rows <= cols, of its transpose otherwise
    const bool turned = p.rows > p.cols;
    unsigned char* rowwise = (turned ? p.Xt + blockIdx.z * p.Xt_bytes : p.X + blockIdx.z * p.X_bytes);
    unsigned char* colwise = (turned ? p.X + blockIdx.z * p.X_bytes : p.Xt + blockIdx.z * p.Xt_bytes);
    const uint32_t pr = turned ? p.Xt_pitch : p.X_pitch, pc = turned ? p.X_pitch : p.Xt_pitch;
    const auto store4 = [](unsigned char* to, const vec4& x) {
        half4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 a, b;
            split(x[e], a, b);
            hi[e] = a;
            lo[e] = b;
        }
        *(half4*)to = hi;
        *(half4*)(to + 64) = lo;
    };
#pragma unroll
    for (uint32_t i0 = 0; i0 < 64; i0 += 16) {
        const uint32_t i = i0 + i16;
        if (r0 + i < p.rows && (c0 + k4) * 4u < pr) store4(rowwise + (uint64_t)(r0 + i) * pr + split_at(c0 + k4), *(const vec4*)&tile[i][k4]);
    }
    // a lane takes its column from four rows: neighbours are 4 rows apart, 4 * 68 words, 16 banks
#pragma unroll
    for (uint32_t i0 = 0; i0 < 64; i0 += 16) {
        const uint32_t i = i0 + i16;
        const vec4 x = {tile[k4][i], tile[k4 + 1][i], tile[k4 + 2][i], tile[k4 + 3][i]};
        if (c0 + i < p.cols && (r0 + k4) * 4u < pc) store4(colwise + (uint64_t)(c0 + i) * pc + split_at(r0 + k4), x);
    }
}

enum { kGram = 0, kPoly = 1, kApply = 2, kFinal = 3, kPartial = 4 };   // kGram: any symmetric product


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
    float* partial;                      // kPartial: [n, splits, M, M]
    uint32_t splits;
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

// The outputs of COUNT numbers: a lane holds column `col` and rows row + 8 q + r, r = 0..3.  Everything is read before the first store: the
// compiler cannot know that the outputs do not overlap, and would wait for each number in turn.
template <uint32_t DT, int COUNT, class ACC>
__device__ __forceinline__ void finish(const OParams& p, const ACC& acc, uint32_t batch, uint32_t row, uint32_t col) {
    if (col >= p.N) return;
    const uint64_t base = ((uint64_t)batch * p.M + row) * p.N + col;
    float z[COUNT], w[COUNT], s[COUNT];
    if (p.z) {
#pragma unroll
        for (int e = 0; e < COUNT; ++e) {
            const uint32_t r = 8u * (e >> 2) + (e & 3);
            const uint64_t o = row + r < p.M ? base + (uint64_t)r * p.N : base;
            if (row < p.M) {
                z[e] = p.z[o];
                if (p.u) w[e] = p.w[o];
                if (p.zsum) s[e] = p.zsum[o];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < COUNT; ++e) {
        const uint32_t r = 8u * (e >> 2) + (e & 3);
        if (row + r >= p.M) continue;
        const uint64_t o = base + (uint64_t)r * p.N;
        const float v = acc[e];
        if (p.out) {
            if (DT == QESGD_F32) ((float*)p.out)[o] = v;
            else if (DT == QESGD_F16) ((_Float16*)p.out)[o] = (_Float16)v;
            else ((__bf16*)p.out)[o] = (__bf16)v;
        }
        if (p.z) {
            const float zv = z[e] + v;
            p.z[o] = zv;
            if (p.u) p.u[o] = w[e] + zv;
            if (p.zsum) p.zsum[o] = s[e] + zv;
        }
    }
}

// A lane holds column lane & 31 of a fragment and rows 8 q + 4 h + r, r = 0..3 (h: the half of the wave).
__device__ __forceinline__ void store_partial(const OParams& p, const float (&v)[16], uint64_t which, uint32_t row, uint32_t col, uint32_t lane) {
    const uint32_t c = col + (lane & 31u), r0 = row + 4u * (lane >> 5);
    float* to = p.partial + (which * p.M + r0) * p.M + c;
    if (c < p.N)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t r = 8u * (e >> 2) + (e & 3);
            if (r0 + r < p.M) to[(uint64_t)r * p.M] = v[e];
        }
}

// P = a I + b G + c G G: the sums hold c G G already.  G[row.., col] = G[col, row..] lies four in a row; its padding is zero.
__device__ __forceinline__ void add_lower_terms(const OParams& p, float (&v)[16], uint32_t z, uint32_t row, uint32_t col, uint32_t lane) {
    const uint32_t c = col + (lane & 31u), r0 = row + 4u * (lane >> 5);
    if (c >= p.N) return;
    const unsigned char* g = p.a + z * p.a_bytes + (uint64_t)c * p.pitch;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t r = r0 + 8u * q;
        if (r >= p.M) continue;
        const half4 hi = *(const half4*)(g + split_at(r)), lo = *(const half4*)(g + split_at(r) + 64);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] += p.cb * ((float)hi[e] + (float)lo[e] * (1.0f / kLo)) + (r + e == c ? p.ca : 0.0f);
    }
}

// A fragment to the split rows of the transpose, and with `both` to its own.  Numbers outside the matrix are stored as the zeros
// that pad its rows.
__device__ __forceinline__ void store_split(const OParams& p, const float (&v)[16], uint32_t z, uint32_t row, uint32_t col, uint32_t lane, bool both) {
    const uint32_t c = col + (lane & 31u), h = lane >> 5;
    uint32_t w[2][8];                    // hi and lo; word 2 q + k holds rows 8 q + 4 h + 2 k and the next
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        _Float16 hi[2], lo[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t r = row + 8u * (k >> 1) + 4u * h + 2u * (k & 1) + e;
            split(r < p.M && c < p.N ? v[2 * k + e] : 0.0f, hi[e], lo[e]);
        }
        w[0][k] = (uint32_t)__builtin_bit_cast(unsigned short, hi[0]) | ((uint32_t)__builtin_bit_cast(unsigned short, hi[1]) << 16);
        w[1][k] = (uint32_t)__builtin_bit_cast(unsigned short, lo[0]) | ((uint32_t)__builtin_bit_cast(unsigned short, lo[1]) << 16);
    }
    // Rows of the transpose: the halves of the wave swap words, so that a lane has 16 numbers in a row.
    unsigned char* to = p.d2 + z * p.d2_bytes + (uint64_t)c * p.d2_pitch + split_at(row + 16u * h);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const auto x = __builtin_amdgcn_permlane32_swap(w[half][k], w[half][4 + k], false, false);
            o[4 * (k >> 1) + (k & 1)] = x[0];
            o[4 * (k >> 1) + (k & 1) + 2] = x[1];
        }
        if (c < p.N && (row + 16u * h) * 4u < p.d2_pitch) {
            *(uint4*)(to + half * 64) = make_uint4(o[0], o[1], o[2], o[3]);
            *(uint4*)(to + half * 64 + 16) = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
    if (!both) return;
    // Its own rows: the four lanes of a quad turn 4 x 4 numbers around, so that lane i of the quad has row i's four columns.
    const bool odd = (lane & 1u) != 0, low = (lane & 2u) == 0;
    const uint32_t pick = odd ? 0x03020706u : 0x05040100u;       // bytes 0..3: own word, 4..7: the neighbour's
    const uint32_t r0 = row + 4u * h + (lane & 3u), c4 = col + (lane & 28u);
    unsigned char* own = p.d1 + z * p.d1_bytes + (uint64_t)r0 * p.d1_pitch + split_at(c4);
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t a = w[half][2 * q], b = w[half][2 * q + 1];
            a = __builtin_amdgcn_perm((uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xB1, 0xF, 0xF, false), a, pick);
            b = __builtin_amdgcn_perm((uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, false), b, pick);
            const uint32_t got = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(low ? b : a), 0x4E, 0xF, 0xF, false);
            if (r0 + 8u * q < p.M && c4 * 4u < p.d1_pitch)
                *(uint2*)(own + (uint64_t)(8u * q) * p.d1_pitch + half * 64) = low ? make_uint2(a, got) : make_uint2(got, b);
        }
}

template <class S>
struct SplitOps {
    static constexpr int PARTS = 2;                            // 16 numbers of the contraction each
    static constexpr int LOADS = (S::BM + S::BN) * 8 / S::threads, PAIR_LOADS = 0;
    struct Frag { half8 ah[S::FM], bh[S::FN], bl[S::FN], al[S::FM]; };
    TileLoader<S::BM, S::threads> la;
    TileLoader<S::BN, S::threads> lb;
    const unsigned char *a, *b;
    uint32_t at_a, at_b;                                       // parts 2 and 3 of the row are lo of parts 0 and 1
    acc16 acc[S::FM][S::FN], low[S::FM][S::FN];                // of hi hi, and of hi lo + lo hi

    __device__ __forceinline__ void fetch(uint32_t step, unsigned char* to) {
        la.load(a + (uint64_t)step * kStepBytes, to, false);
        lb.load(b + (uint64_t)step * kStepBytes, to + S::BM * kStepBytes, false);
    }
    __device__ __forceinline__ void fetch_pair(uint32_t) {}
    __device__ __forceinline__ void arrive(uint32_t) {}
    __device__ __forceinline__ void next() {}
    __device__ __forceinline__ void read(Frag& f, const unsigned char* from, int part) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i) f.ah[i] = *(const half8*)(from + (at_a ^ (part * 32u)) + i * 4096);
#pragma unroll
        for (int j = 0; j < S::FN; ++j) f.bh[j] = *(const half8*)(from + (at_b ^ (part * 32u)) + j * 4096);
#pragma unroll
        for (int j = 0; j < S::FN; ++j) f.bl[j] = *(const half8*)(from + (at_b ^ (part * 32u + 64u)) + j * 4096);
#pragma unroll
        for (int i = 0; i < S::FM; ++i) f.al[i] = *(const half8*)(from + (at_a ^ (part * 32u + 64u)) + i * 4096);
    }
    __device__ __forceinline__ void multiply(const Frag& f, int) {
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ah[i], f.bh[j], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) low[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.ah[i], f.bl[j], low[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int j = 0; j < S::FN; ++j) low[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.al[i], f.bh[j], low[i][j], 0, 0, 0);
    }
};

// 4096 x 25088: X X^T in four pieces 1215 us, 1.04 PFLOP/s of fp16 products, P X 2212 us, 1.14, what a large library product reaches (the card lowers its
// clock); the last one, with z, u and zsum behind it, 2526 us; G G 275 us = 0.75, 528 tiles on 512 places.  512 x 4608, 2 of them: X X^T 13.4, G G 7.5, P X
// 30, the last 41 us.  With 64 x 64 tiles a step, 16 KB from L2 to LDS and 32 KB from there to the registers, takes 0.2 us: 3 or 8 buffers, or a second set of
// waves that shares the steps, change nothing, so small matrices stay 4.8 us + 0.2 us a step.
// Two waves a SIMD: two workgroups of 128 x 128 share a CU, which takes at most 256 registers a lane.
template <class S, int KIND, uint32_t DT>
__global__ void __launch_bounds__(S::threads, 2) k_orthogonal_product(const OParams p) {
    static_assert(S::BM == S::BN, "symmetric products take square tiles");
    __shared__ __attribute__((aligned(1024))) unsigned char lds0[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds1[(S::BM + S::BN) * kStepBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds2[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    __shared__ __attribute__((aligned(1024))) unsigned char lds3[S::BUFFERS > 2 ? (S::BM + S::BN) * kStepBytes : 16];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, h = lane >> 5;
    const uint32_t wm = wave / S::WN, wn = wave % S::WN;
    uint32_t t = tile_of_workgroup(blockIdx.x, gridDim.x), split_k = 0, first = 0, steps = p.steps;
    const uint32_t z = __builtin_amdgcn_readfirstlane(t / (p.tiles * p.splits));
    t -= z * (p.tiles * p.splits);
    uint32_t tm, tn;
    if (KIND == kPartial) {              // the tiles of one piece of the contraction follow one another
        split_k = __builtin_amdgcn_readfirstlane(t / p.tiles);
        t -= split_k * p.tiles;
        first = __builtin_amdgcn_readfirstlane(split_k * p.steps / p.splits);
        steps = __builtin_amdgcn_readfirstlane((split_k + 1u) * p.steps / p.splits) - first;
    }
    if (KIND == kGram || KIND == kPoly || KIND == kPartial) upper_tile(t, tm, tn);
    else banded_tile(t, p.tiles_m, p.tiles_n, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);     // the same in every lane, which the compiler loses over divisions and roots
    tn = __builtin_amdgcn_readfirstlane(tn);
    const uint32_t m0 = tm * S::BM, n0 = tn * S::BN;
    SplitOps<S> ops;
    ops.a = p.a + z * p.a_bytes + (uint64_t)m0 * p.pitch + (uint64_t)first * kStepBytes;
    ops.b = p.b + z * p.b_bytes + (uint64_t)n0 * p.pitch + (uint64_t)first * kStepBytes;
    ops.la.init(p.pitch, p.M - m0);
    ops.lb.init(p.pitch, p.N - n0);
    ops.at_a = wm * S::FM * 32 * kStepBytes + lane_place(lane);
    ops.at_b = (S::BM + wn * S::FN * 32) * kStepBytes + lane_place(lane);
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) ops.acc[i][j] = ops.low[i][j] = acc16{};
    if constexpr (S::BUFFERS == 2) {
        unsigned char* const buffers[2] = {lds0, lds1};
        run_steps(ops, steps, buffers);
    } else {
        unsigned char* const buffers[4] = {lds0, lds1, lds2, lds3};
        run_steps(ops, steps, buffers);
    }
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const uint32_t row = m0 + (wm * S::FM + i) * 32u, col = n0 + (wn * S::FN + j) * 32u;
            float v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __builtin_fmaf(ops.low[i][j][e], 1.0f / kLo, ops.acc[i][j][e]) * p.scale;
            if (KIND == kFinal) {
                finish<DT, 16>(p, v, z, row + 4u * h, col + (lane & 31u));
                continue;
            }
            if (KIND == kPartial) {
                store_partial(p, v, z * p.splits + split_k, row, col, lane);
                continue;
            }
            if (KIND == kPoly) add_lower_terms(p, v, z, row, col, lane);
            store_split(p, v, z, row, col, lane, KIND == kApply || tm != tn);
        }
}

// G from the partial sums of its contraction, added in order, 32 x 32 at a time, both halves.  A lane has one row's number of each of four
// rows and eight pieces in flight: the sums are few and far apart.  4096 x 4096 in three pieces 41 us, two of 512 x 512 in seven 5.
__global__ void __launch_bounds__(256) k_orthogonal_gram_sum(const OParams p) {
    __shared__ float tile[32][33];
    uint32_t ti, tj;
    upper_tile(blockIdx.x, ti, tj);
    const uint32_t r0 = ti * 32u, c0 = tj * 32u, z = blockIdx.y;
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5;
    const uint64_t all = (uint64_t)p.M * p.M;
    const float* from = p.partial + (uint64_t)z * p.splits * all;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float* at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + ty + 8u * i, c = c0 + tx;
        at[i] = from + (uint64_t)min(r, p.M - 1u) * p.M + min(c, p.M - 1u);
    }
    for (uint32_t k0 = 0; k0 < p.splits; k0 += 8) {
        float x[8][4];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[k][i] = at[i][(uint64_t)min(k0 + k, p.splits - 1u) * all];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += k0 + k < p.splits ? x[k][i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) tile[ty + 8 * i][tx] = r0 + ty + 8u * i < p.M && c0 + tx < p.M ? v[i] : 0.0f;
    __syncthreads();
    unsigned char* G = p.d1 + z * p.d1_bytes;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t i = ty + 8u * k;
        _Float16 hi, lo;
        if (r0 + i < p.M) {
            // below the diagonal, inside its tile, the mirror's number: both halves of a product are the same bits
            split(ti == tj && i > tx ? tile[tx][i] : tile[i][tx], hi, lo);
            unsigned char* to = G + (uint64_t)(r0 + i) * p.d1_pitch + split_at(c0 + tx);
            *(_Float16*)to = hi;
            *(_Float16*)(to + 64) = lo;
        }
        if (ti != tj && c0 + i < p.M) {
            split(tile[tx][i], hi, lo);
            unsigned char* to = G + (uint64_t)(c0 + i) * p.d1_pitch + split_at(r0 + tx);
            *(_Float16*)to = hi;
            *(_Float16*)(to + 64) = lo;
        }
    }
}

// A whole matrix in one workgroup: X, its transpose and one m x m matrix (G, then P in its place) stay in LDS as split rows for all
// steps, so a call is one launch and reads and writes its operands once.  Which shapes fit: small_layout().
//
// What bounds it is its chain of short phases, five barriers a step (six where the contraction is in pieces), so the work is cut into 16 x 16 tiles, whose matrix instruction takes
// a whole group of 32 numbers at once, and dealt to 16 waves.  A step: the tiles of G's upper half, where they are few the contraction
// in pieces to several waves whose sums one wave adds in order; P = a I + b G + c G G by the same waves; P X tile by tile, held in
// registers until every wave has read X.  Rows are groups of 128 bytes, chunks placed as in the pipeline.  64 x 64, 16 of them: 72 us as
// the launches of the general path, 31 us with 32 x 32 tiles on 8 waves, 23 us so: 7 us and 2.9 us a step, whether 16 matrices or one.  Vector
// instructions take 57% of a SIMD's cycles, LDS 35% of a CU's (two fifths of that bank conflicts), the matrix units 8%.
constexpr uint32_t kSmallWaves = 16, kSmallThreads = kSmallWaves * 64;
constexpr uint32_t kSmallHeld = 4;       // tiles of P X that a wave holds
constexpr uint32_t kSmallEach = kSmallHeld * 256 / 64;       // elements that a thread reads
typedef float acc4 __attribute__((ext_vector_type(4)));

struct SmallLayout {
    uint32_t mt, nt;                     // tiles along the sides
    uint32_t mg, ng;                     // groups of 32 along the sides
    uint32_t tiles, pieces;              // of G's upper half; of the contraction
    uint32_t Xt, G, partial, total;      // bytes: X lies at 0
};

// total = 0 where the matrix does not fit.
inline SmallLayout small_layout(uint64_t m, uint64_t n) {
    SmallLayout L{};
    if (m > 96 || n > 1024) return L;
    L.mt = (uint32_t)(m + 15) / 16;
    L.nt = (uint32_t)(n + 15) / 16;
    L.mg = (uint32_t)(m + 31) / 32;
    L.ng = (uint32_t)(n + 31) / 32;
    L.tiles = L.mt * (L.mt + 1) / 2;
    L.pieces = L.tiles < kSmallWaves ? kSmallWaves / L.tiles : 1;
    if (L.pieces > L.ng) L.pieces = L.ng;
    L.Xt = L.mt * 16 * L.ng * 128;
    L.G = L.Xt + L.nt * 16 * L.mg * 128;
    L.partial = L.G + L.mt * 16 * L.mg * 128;
    L.total = L.partial + (L.pieces - 1) * L.tiles * 1024;
    if (L.total > kLdsBytes - 8 * kSmallWaves || L.mt * L.nt > kSmallHeld * kSmallWaves) L.total = 0;
    return L;
}

struct SmallParams {
    SParams s;
    OParams o;                           // of the last product
    SmallLayout L;
    uint32_t steps;
    struct Step { float g, a, b, c, y; } step[QESGD_MAX_STEPS];       // of the sums, into the scales of G, P and the next X
};

// Byte of number k's hi in a row (its lo: the place with 64 flipped, chunk c + 4 instead of c).
__device__ __forceinline__ uint32_t place_of(uint32_t row, uint32_t pitch, uint32_t k) {
    return row * pitch + (k >> 5) * 128u + ((((k & 31u) >> 3) ^ ((row >> 1) & 7u)) * 16u) + (k & 7u) * 2u;
}
// A wave's vector instruction takes four cycles and sixteen waves share a CU, so places are put together from few: rows of a tile
// are 16 apart from the next tile's, which leaves the swizzle (row / 2 & 7) alone.
struct SmallPlaces {
    uint32_t read, col, row, pitch;
    // lane: row lane & 15, numbers 8 (lane / 16) .. + 7 of a group (read); row lane & 15, numbers 4 (lane / 16) .. + 3 (col);
    // rows 4 (lane / 16) .. + 3, number lane & 15 (row)
    __device__ __forceinline__ SmallPlaces(uint32_t lane, uint32_t pitch_) : pitch(pitch_) {
        read = place_of(lane & 15u, pitch, 8u * (lane >> 4));
        col = place_of(lane & 15u, pitch, 4u * (lane >> 4));
        row = place_of(4u * (lane >> 4), pitch, lane & 15u);
    }
};
__device__ __forceinline__ half8 read8(const unsigned char* p) { return *(const half8*)p; }

// acc += A B^T over `groups` groups from g on, `by` apart; A and B: the tiles' first rows.  A lane's operand is one chunk of its row.
__device__ __forceinline__ acc4 small_product(const unsigned char* A, uint32_t a, const unsigned char* B, uint32_t b, uint32_t g, uint32_t groups, uint32_t by) {
    acc4 acc = {0.0f, 0.0f, 0.0f, 0.0f}, low = acc;
    const unsigned char *ah = A + a, *al = A + (a ^ 64u), *bh = B + b, *bl = B + (b ^ 64u);
    for (; g < groups; g += by) {
        const half8 vah = read8(ah + g * 128u), vbh = read8(bh + g * 128u), vbl = read8(bl + g * 128u), val = read8(al + g * 128u);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vah, vbh, acc, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_16x16x32_f16(vah, vbl, low, 0, 0, 0);
        low = __builtin_amdgcn_mfma_f32_16x16x32_f16(val, vbh, low, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(low[r], 1.0f / kLo, acc[r]);
    return acc;
}
// Tile (tr, tc): a lane holds column lane & 15 and rows 4 (lane / 16) .. + 3.  Its transpose goes to by_col, and with by_row itself there.
__device__ __forceinline__ void put_tile(unsigned char* by_row, const SmallPlaces& pr, unsigned char* by_col, const SmallPlaces& pc, uint32_t tr,
                                         uint32_t tc, const acc4& v) {
    half4 hi, lo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        _Float16 a, b;
        split(v[r], a, b);
        hi[r] = a;
        lo[r] = b;
    }
    unsigned char* c = by_col + tc * 16u * pc.pitch + (tr >> 1) * 128u;
    const uint32_t at = pc.col ^ ((tr & 1u) * 32u);
    *(half4*)(c + at) = hi;
    *(half4*)(c + (at ^ 64u)) = lo;
    if (by_row) {
        unsigned char* w = by_row + tr * 16u * pr.pitch + (tc >> 1) * 128u;
        const uint32_t at0 = pr.row ^ ((tc & 1u) * 32u);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            const uint32_t at1 = (at0 ^ ((r >> 1) * 16u));                  // rows 2 and 3: the next swizzle
            *(_Float16*)(w + at1 + r * pr.pitch) = hi[r];
            *(_Float16*)(w + (at1 ^ 64u) + r * pr.pitch) = lo[r];
        }
    }
}

template <uint32_t DT>
__global__ void __launch_bounds__(kSmallThreads) k_orthogonal_small(const SmallParams p) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char X[];       // mt * 16 rows
    __shared__ double sums[kSmallWaves];
    const SmallLayout& L = p.L;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), z = blockIdx.x, lane = threadIdx.x & 63u;
    SmallPlaces px(lane, L.ng * 128u), pg(lane, L.mg * 128u);
    unsigned char* const Xt = X + L.Xt;                       // nt * 16 rows
    unsigned char* const G = X + L.G;                         // mt * 16 rows
    acc4* const partial = (acc4*)(X + L.partial);

    // Lane i has the factors of step i: a load from the arguments in every step, which nothing hides, took 0.2 us of each.
    static_assert(QESGD_MAX_STEPS <= 64 && (QESGD_MAX_STEPS & (QESGD_MAX_STEPS - 1u)) == 0 && sizeof(SmallParams::Step) == 5 * sizeof(float), "one step a lane");
    float factors[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) factors[i] = ((const float*)&p.step[lane & (QESGD_MAX_STEPS - 1u)])[i];

    // the momentum and the norm, as in k_orthogonal_momentum; what a thread has read it keeps
    const uint64_t base = (uint64_t)z * p.s.d;
    const uint32_t d = (uint32_t)p.s.d;
    float x[kSmallEach];
#pragma unroll
    for (uint32_t k = 0; k < kSmallEach; ++k) {
        const uint32_t i = k * kSmallThreads + threadIdx.x;
        x[k] = i < d ? fetch<DT>(p.s.x, base + i) : 0.0f;
    }
    if (p.s.momentum) {
        float m[kSmallEach];
#pragma unroll
        for (uint32_t k = 0; k < kSmallEach; ++k) {
            const uint32_t i = k * kSmallThreads + threadIdx.x;
            m[k] = i < d ? p.s.momentum[base + i] : 0.0f;
        }
#pragma unroll
        for (uint32_t k = 0; k < kSmallEach; ++k) {
            const uint32_t i = k * kSmallThreads + threadIdx.x;
            m[k] = p.s.mu * m[k] + x[k];
            if (i < d) p.s.momentum[base + i] = m[k];
            x[k] = p.s.nesterov ? x[k] + p.s.mu * m[k] : m[k];
        }
    }
    double sum = 0.0;
#pragma unroll
    for (uint32_t k = 0; k < kSmallEach; ++k) sum += (double)x[k] * (double)x[k];
    if (((p.s.rows | p.s.cols) & 31u) != 0)                   // zeros behind the ends
        for (uint32_t i = threadIdx.x * 16u; i < L.partial; i += kSmallThreads * 16u) *(uint4*)(X + i) = make_uint4(0, 0, 0, 0);
    sum = wave_sum(sum);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (uint32_t i = 0; i < kSmallWaves; ++i) sum += sums[i];
    const double norm = sqrt(sum) + (double)p.s.eps;
    const double scale = norm > 0.0 ? (double)kFirstX / norm : 0.0;
    const bool turned = p.s.rows > p.s.cols;
    {
        uint32_t r = threadIdx.x / p.s.cols, c = threadIdx.x - r * p.s.cols;
        const uint32_t dr = kSmallThreads / p.s.cols, dc = kSmallThreads - dr * p.s.cols;
#pragma unroll
        for (uint32_t k = 0; k < kSmallEach; ++k) {
            if (k * kSmallThreads + threadIdx.x < d) {
                _Float16 hi, lo;
                split((float)((double)x[k] * scale), hi, lo);
                const uint32_t at = place_of(turned ? c : r, px.pitch, turned ? r : c), bt = place_of(turned ? r : c, pg.pitch, turned ? c : r);
                *(_Float16*)(X + at) = hi;
                *(_Float16*)(X + (at ^ 64u)) = lo;
                *(_Float16*)(Xt + bt) = hi;
                *(_Float16*)(Xt + (bt ^ 64u)) = lo;
            }
            r += dr;
            c += dc;
            if (c >= p.s.cols) { c -= p.s.cols; ++r; }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();

    // A wave has up to two tiles of G (21 at most), or a piece of one, and up to kSmallHeld of P X.
    const bool split_up = L.pieces > 1;
    const uint32_t piece = split_up ? __builtin_amdgcn_readfirstlane(wave / L.tiles) : 0;
    uint32_t ti[2], tj[2], it[kSmallHeld], jt[kSmallHeld];
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
        upper_tile(min(wave + k * kSmallWaves - piece * L.tiles, L.tiles - 1), ti[k], tj[k]);
        ti[k] = __builtin_amdgcn_readfirstlane(ti[k]);
        tj[k] = __builtin_amdgcn_readfirstlane(tj[k]);
    }
#pragma unroll
    for (uint32_t k = 0; k < kSmallHeld; ++k) {
        jt[k] = __builtin_amdgcn_readfirstlane((wave + k * kSmallWaves) / L.mt);
        it[k] = wave + k * kSmallWaves - jt[k] * L.mt;
    }
    const uint32_t l = lane & 15u, quad = lane >> 4;
    acc4 y[kSmallHeld] = {};
    for (uint32_t step = 0;; ++step) {
        // sums with these are formed where they are used: kept over the steps, they spill
        asm volatile("" : "+v"(px.read), "+v"(px.col), "+v"(pg.read), "+v"(pg.col), "+v"(pg.row));
        SmallParams::Step f;
#pragma unroll
        for (int i = 0; i < 5; ++i) ((float*)&f)[i] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_uint(factors[i]), (int)step));
        acc4 g[2] = {};
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            if (k == 0 ? wave < L.tiles * L.pieces : wave + kSmallWaves < L.tiles) {
                g[k] = small_product(X + ti[k] * 16u * px.pitch, px.read, X + tj[k] * 16u * px.pitch, px.read, piece, L.ng, L.pieces);
                if (piece > 0) partial[(wave - L.tiles) * 64u + lane] = g[k];
            }
        }
        if (split_up) __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            if (wave + k * kSmallWaves < L.tiles) {
                for (uint32_t i = 1; i < L.pieces; ++i) g[k] += partial[((i - 1) * L.tiles + wave) * 64u + lane];
                g[k] *= f.g;
                put_tile(ti[k] != tj[k] ? G : nullptr, pg, G, pg, ti[k], tj[k], g[k]);
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            if (wave + k * kSmallWaves < L.tiles) {
                const acc4 gg = small_product(G + ti[k] * 16u * pg.pitch, pg.read, G + tj[k] * 16u * pg.pitch, pg.read, 0, L.mg, 1);
                const bool diagonal = ti[k] == tj[k];
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r)
                    g[k][r] = gg[r] * f.c + f.b * g[k][r] + (diagonal && quad * 4u + r == l ? f.a : 0.0f);
            }
        }
        __syncthreads();                                      // G has been read
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k)
            if (wave + k * kSmallWaves < L.tiles) put_tile(ti[k] != tj[k] ? G : nullptr, pg, G, pg, ti[k], tj[k], g[k]);
        __syncthreads();
        const bool last = step + 1 == p.steps;
#pragma unroll
        for (uint32_t k = 0; k < kSmallHeld; ++k) {
            const unsigned char *P = G + it[k] * 16u * pg.pitch, *T = Xt + jt[k] * 16u * pg.pitch;
            // numbers of a row of the caller's matrix along the lanes where the result leaves: P X as it is, or its transpose
            const bool straight = last && !turned;
            if (jt[k] < L.nt) y[k] = small_product(straight ? P : T, pg.read, straight ? T : P, pg.read, 0, L.mg, 1);
        }
        if (last) break;
        __syncthreads();                                      // the transpose has been read
#pragma unroll
        for (uint32_t k = 0; k < kSmallHeld; ++k) {
            y[k] *= f.y;
            if (jt[k] < L.nt) put_tile(Xt, pg, X, px, jt[k], it[k], y[k]);
        }
        __syncthreads();
    }
#pragma unroll
    for (uint32_t k = 0; k < kSmallHeld; ++k)
        if (jt[k] < L.nt) finish<DT, 4>(p.o, y[k] * p.o.scale, z, (turned ? jt[k] : it[k]) * 16u + quad * 4u, (turned ? it[k] : jt[k]) * 16u + l);
}

// Which tiles, and how many pieces of the contraction, from how long the workgroups take on 256 CUs.  Unit: a step of 512 workgroups
// with 128 x 128 tiles, two a CU, 1.1 us of a full chip, and 3 us for a launch.  A last round of up to 256 has a CU each and takes 0.70 of that.  64 x 64: 0.38 (a
// quarter of the work; each step reads twice as much for it).  P X with 64 x 64: 0.12 for a last round of up to 256, because its stores and outputs
// run under other workgroups' products.  Larger tiles have no registers for two sums of each number: 256 x 256 with one sum took 13.4 ms where these take
// 14.1 at 4096 x 25088 and 1572 / 1607 us at 2048 x 8192, 256 x 128 tiles 14.2.  Five steps, us, by this rule / with 64 x 64 alone / with 128 x 128 alone:
//   512 x 4608, 2 of them 267 / 267 / 426;  1024 x 8192 488 / 523 / 681;  2048 x 2048 812 / 840 / 826;  2048 x 8192 1607 / 1909 / 1626;  3000 x
//   3000 2228 / 2445 / 2230;  1024 x 1024, 12 of them 1094 / 1254 / 1094;  4096 x 6000 5944 / 7852 / 5947;  4096 x 25088 14106 / 19925 / 14108
struct Cut {
    uint32_t edge, pieces;
    double us;                           // by this reckoning
};

double cut_cost(uint64_t groups, uint32_t edge, bool upper) {
    const uint64_t slots = 512, left = groups % slots;
    const double full = edge == 128 ? 1.0 : 0.38, half = edge == 128 ? 0.70 : upper ? 0.27 : 0.12;
    return (double)(groups / slots) * full + (left == 0 ? 0.0 : left <= 256 ? half : full);
}

// M x N (upper = M x M, the upper half) over `steps` steps, `count` of them; more than one piece only for upper.
Cut choose_cut(uint64_t M, uint64_t N, uint64_t steps, uint64_t count, bool upper, uint32_t most_pieces) {
    Cut best{64, 1, 1e300};
    for (uint32_t edge : {64u, 128u}) {
        const uint64_t tm = (M + edge - 1) / edge, tn = (N + edge - 1) / edge, tiles = (upper ? tm * (tm + 1) / 2 : tm * tn) * count;
        for (uint32_t pieces = 1; pieces <= most_pieces && pieces * 4ull <= steps + 3ull; ++pieces) {
            // A piece has about four steps or more: ceil(steps / 4) pieces at most, the shortest of which has three (two, of five steps
            // in two pieces); the pipeline takes any number.  The sums of the pieces cost a launch, and are written and read at about 4 TB/s.
            const double sums = pieces == 1 ? 0.0 : 3.0 + (double)pieces * (double)count * (double)(M * M) * 2e-6;
            const double cost = 3.0 + cut_cost(tiles * pieces, edge, upper) * (double)((steps + pieces - 1) / pieces) * 1.1 + sums;
            if (cost < best.us) best = Cut{edge, pieces, cost};
        }
    }
    return best;
}

// Workspace: partial sums, X, two of its transpose, G, P, for pairs of steps two more like them, and the pieces' sums.
struct Plan {
    uint64_t m, n;                       // shorter and longer side
    uint32_t parts;
    uint64_t X_pitch, Xt_pitch, G_pitch, X_bytes, Xt_bytes, G_bytes;
    uint64_t X, Xt[2], G, P, T, P2, partial, total;
    Cut gram, square, apply;             // X X^T, products of m x m matrices, P X
    bool pairs;
};

Plan make_plan(uint64_t rows, uint64_t cols, uint32_t count) {
    Plan p{};
    p.m = rows < cols ? rows : cols;
    p.n = rows < cols ? cols : rows;
    const uint64_t d = rows * cols;
    p.parts = (uint32_t)std::min<uint64_t>((d + 4095) / 4096, 1024);
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
    p.gram = choose_cut(p.m, p.m, p.X_pitch / kStepBytes, count, true, 16);
    p.square = choose_cut(p.m, p.m, p.G_pitch / kStepBytes, count, true, 1);
    p.apply = choose_cut(p.m, p.n, p.G_pitch / kStepBytes, count, false, 1);
    // Two steps at once: G of the second is P G P, and one product takes X through both, P' P X: three products of m x m matrices in the
    // place of X X^T and P X.  Singly / in pairs, us: 128 x 1024 97 / 101, 512 x 4608, 2 of them 327 / 284, 768 x 1536 197 / 198, 1000 x 2049
    // 304 / 284, 2048 x 3000 1014 / 1027, 2048 x 8192 1965 / 1643, 4096 x 6000 5820 / 5566, 4096 x 25088 19874 / 14143.  For matrices of noise and
    // strong directions the errors are those of single steps where n is much larger than m, and grow up to three times for square matrices, hence not below n = 2 m; where one
    // direction holds nearly all of the norm, five times at 520 x 4160 (5e-6, and 2.4e-6 with fp32 products).
    p.pairs = p.n >= 2 * p.m && p.gram.us + p.apply.us > 3.0 * p.square.us;
    if (p.pairs) {
        p.T = take(p.G_bytes);
        p.P2 = take(p.G_bytes);
    }
    p.partial = at;
    if (p.gram.pieces > 1) take(p.gram.pieces * p.m * p.m * 4);
    p.total = at;
    return p;
}

int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

template <class S, int KIND, uint32_t DT>
int launch_product_as(OParams& p, uint32_t count, hipStream_t stream) {
    constexpr bool symmetric = KIND == kGram || KIND == kPoly || KIND == kPartial;
    p.tiles_m = (p.M + S::BM - 1) / S::BM;
    p.tiles_n = (p.N + S::BN - 1) / S::BN;
    const uint64_t tiles = symmetric ? (uint64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (uint64_t)p.tiles_m * p.tiles_n;
    if (!grid_ok(tiles * p.splits * count, S::threads)) return QESGD_ERR_DIM;
    p.tiles = (uint32_t)tiles;
    k_orthogonal_product<S, KIND, DT><<<p.tiles * p.splits * count, S::threads, 0, stream>>>(p);
    return launched();
}

typedef TileShape<2, 2, 2, 2, 2> Tile128;
typedef TileShape<2, 2, 1, 1, 4> Tile64;

template <int KIND, uint32_t DT>
int launch_product(OParams& p, const Cut& cut, uint32_t count, hipStream_t stream) {
    p.steps = p.pitch / kStepBytes;
    p.splits = cut.pieces;
    switch (cut.edge) {
        case 128: return launch_product_as<Tile128, KIND, DT>(p, count, stream);
        default: return launch_product_as<Tile64, KIND, DT>(p, count, stream);
    }
}

template <uint32_t DT>
int launch_type(const Orthogonalize& a) {
    SParams s{};
    s.x = a.x;
    s.momentum = a.momentum;
    s.d = a.rows * a.cols;
    s.rows = (uint32_t)a.rows;
    s.cols = (uint32_t)a.cols;
    s.mu = a.mu;
    s.eps = a.eps;
    s.nesterov = a.nesterov;
    const Scales sc = scales_of(a.coeffs, a.steps);
    const SmallLayout small = small_layout(std::min(a.rows, a.cols), std::max(a.rows, a.cols));
    if (small.total) {
        SmallParams p{};
        p.s = s;
        p.L = small;
        p.steps = a.steps;
        for (uint32_t i = 0; i < a.steps; ++i) {
            const double X = sc.X[i], G = sc.G[i], P = sc.P[i];
            p.step[i] = {(float)(G / (X * X)), (float)(a.coeffs[3 * i] * P), (float)(a.coeffs[3 * i + 1] * (P / G)), (float)(a.coeffs[3 * i + 2] * (P / (G * G))),
                         (float)(sc.X[i + 1] / (P * X))};
        }
        p.o.M = (uint32_t)a.rows;
        p.o.N = (uint32_t)a.cols;
        p.o.scale = (float)(a.alpha / (sc.P[a.steps - 1] * sc.X[a.steps - 1]));
        p.o.out = a.out;
        p.o.z = a.z;
        p.o.w = a.w;
        p.o.u = a.u;
        p.o.zsum = a.zsum;
        k_orthogonal_small<DT><<<a.n, kSmallThreads, small.total, a.stream>>>(p);
        return launched();
    }

    const Plan pl = make_plan(a.rows, a.cols, a.n);
    const bool turned = a.rows > a.cols;
    s.partial = (double*)a.workspace;
    s.parts = pl.parts;
    s.X = a.workspace + pl.X;
    s.Xt = a.workspace + pl.Xt[0];
    s.X_bytes = pl.X_bytes;
    s.Xt_bytes = pl.Xt_bytes;
    s.X_pitch = (uint32_t)pl.X_pitch;
    s.Xt_pitch = (uint32_t)pl.Xt_pitch;
    k_orthogonal_momentum<DT><<<dim3(pl.parts, a.n), 256, 0, a.stream>>>(s);
    if (const int rc = launched(); rc != QESGD_OK) return rc;
    k_orthogonal_split<DT><<<dim3((uint32_t)((a.cols + 63) / 64), (uint32_t)((a.rows + 63) / 64), a.n), 256, 0, a.stream>>>(s);
    if (const int rc = launched(); rc != QESGD_OK) return rc;

    const auto at = [&](uint64_t offset) { return a.workspace + offset; };
    // d = A B of symmetric matrices that commute; scale: d's over A's and B's
    const auto square = [&](uint64_t A, uint64_t B, uint64_t d, double scale) {
        OParams o{};
        o.a = at(A);
        o.b = at(B);
        o.a_bytes = o.b_bytes = o.d1_bytes = o.d2_bytes = pl.G_bytes;
        o.M = o.N = (uint32_t)pl.m;
        o.pitch = o.d1_pitch = o.d2_pitch = (uint32_t)pl.G_pitch;
        o.d1 = o.d2 = at(d);
        o.scale = (float)scale;
        return o;
    };
    const auto poly = [&](uint32_t step, uint64_t d) {
        const double G = sc.G[step], P = sc.P[step];
        OParams o = square(pl.G, pl.G, d, a.coeffs[3 * step + 2] * (P / (G * G)));
        o.ca = (float)(a.coeffs[3 * step] * P);
        o.cb = (float)(a.coeffs[3 * step + 1] * (P / G));
        return launch_product<kPoly, 0>(o, pl.square, a.n, a.stream);
    };
    uint32_t which = 0;                  // of the two transposes
    // An odd step stays alone, in the middle: five steps as 2 1 2 are as exact as one by one (matrices of noise and strong directions, 128 x
    // 1024: 1.5e-6 either way), as 2 2 1 half as exact.
    const uint32_t alone = pl.pairs && (a.steps & 1u) ? 2u * ((a.steps / 2u + 1u) / 2u) : a.steps;
    for (uint32_t i = 0; i < a.steps;) {
        const double X = sc.X[i];
        OParams g = square(0, 0, pl.G, sc.G[i] / (X * X));
        g.a = g.b = at(pl.X);
        g.a_bytes = g.b_bytes = pl.X_bytes;
        g.pitch = (uint32_t)pl.X_pitch;
        int rc;
        if (pl.gram.pieces > 1) {
            g.partial = (float*)at(pl.partial);
            rc = launch_product<kPartial, 0>(g, pl.gram, a.n, a.stream);
            if (rc != QESGD_OK) return rc;
            const uint32_t t = (g.M + 31u) / 32u;
            k_orthogonal_gram_sum<<<dim3(t * (t + 1) / 2, a.n), 256, 0, a.stream>>>(g);
            rc = launched();
        } else {
            rc = launch_product<kGram, 0>(g, pl.gram, a.n, a.stream);
        }
        const bool pair = pl.pairs && i != alone && i + 1 < a.steps && sc.PP[i] > 0.0;
        if (rc == QESGD_OK) rc = poly(i++, pl.P);
        uint64_t P = pl.P;
        double scale_p = sc.P[i - 1];
        if (pair) {
            OParams o;
            const double G = sc.G[i - 1], T = sc.T[i - 1], G2 = sc.G[i], P2 = sc.P[i], PP = sc.PP[i - 1];
            if (rc == QESGD_OK) rc = launch_product<kGram, 0>(o = square(pl.G, pl.P, pl.T, T / (G * scale_p)), pl.square, a.n, a.stream);
            if (rc == QESGD_OK) rc = launch_product<kGram, 0>(o = square(pl.T, pl.P, pl.G, G2 / (T * scale_p)), pl.square, a.n, a.stream);
            if (rc == QESGD_OK) rc = poly(i++, pl.P2);
            if (rc == QESGD_OK) rc = launch_product<kGram, 0>(o = square(pl.P2, pl.P, pl.T, PP / (P2 * scale_p)), pl.square, a.n, a.stream);
            P = pl.T;
            scale_p = PP;
        }
        if (rc != QESGD_OK) return rc;
        OParams x{};
        x.a = at(P);
        x.a_bytes = pl.G_bytes;
        x.M = (uint32_t)pl.m;
        x.b = at(pl.Xt[which]);
        x.b_bytes = pl.Xt_bytes;
        x.N = (uint32_t)pl.n;
        x.pitch = (uint32_t)pl.G_pitch;
        if (i < a.steps) {
            which ^= 1u;
            x.d1 = at(pl.X);
            x.d1_bytes = pl.X_bytes;
            x.d1_pitch = (uint32_t)pl.X_pitch;
            x.d2 = at(pl.Xt[which]);
            x.d2_bytes = pl.Xt_bytes;
            x.d2_pitch = (uint32_t)pl.Xt_pitch;
            x.scale = (float)(sc.X[i] / (scale_p * X));
            rc = launch_product<kApply, 0>(x, pl.apply, a.n, a.stream);
        } else {
            if (turned) {                // (P X)^T = Xt P, rows as the caller has them
                std::swap(x.a, x.b);
                std::swap(x.a_bytes, x.b_bytes);
                std::swap(x.M, x.N);
            }
            x.scale = (float)(a.alpha / (scale_p * X));
            x.out = a.out;
            x.z = a.z;
            x.w = a.w;
            x.u = a.u;
            x.zsum = a.zsum;
            rc = launch_product<kFinal, DT>(x, pl.apply, a.n, a.stream);
        }
        if (rc != QESGD_OK) return rc;
    }
    return QESGD_OK;
}

}  // namespace

size_t orthogonalize_workspace(uint64_t rows, uint64_t cols, uint32_t n) {
    if (small_layout(rows < cols ? rows : cols, rows < cols ? cols : rows).total) return 0;
    return make_plan(rows, cols, n).total;
}

int launch_orthogonalize(const Orthogonalize& a) {
    switch (a.dtype) {
        case QESGD_F32: return launch_type<QESGD_F32>(a);
        case QESGD_BF16: return launch_type<QESGD_BF16>(a);
        default: return launch_type<QESGD_F16>(a);
    }
}

}  // namespace qesgd
