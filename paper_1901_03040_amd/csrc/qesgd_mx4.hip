// The microscaled 4-bit form of matrices: quantisation along the rows, along the columns or both from one read,
// and its inverse fused with the mean over the workers and the update.
//
// Block of 32 coordinates with largest magnitude m: scale 2^e, element q of {0, .5, 1, 1.5, 2, 3, 4, 6} with a sign.
//   nearest     e = floor(log2 m) - 2, q = |v| / 2^e to nearest even, at most 6
//   stochastic  e = the smallest with m <= 6 * 2^e, q one of the two neighbours of a = |v| / 2^e: up iff r + T >= 2^16,
//               T = trunc(f * 2^16), f the fraction of the way; E[q] = a to 2^-16 of a step
// a is exact (a power of two only moves the exponent; what falls below fp32's range is far below the grid).
#include <type_traits>

#include "qesgd_device.h"
#include "qesgd_matrix.h"

namespace qesgd {
namespace {

typedef uint32_t uvec4 __attribute__((ext_vector_type(4)));
typedef uint32_t uvec2 __attribute__((ext_vector_type(2)));
typedef float fvec2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
// 128-bit accesses at any element's address: the rows of a matrix start where they start
typedef uvec4 uvec4_any __attribute__((aligned(2)));
typedef vec4 vec4_any __attribute__((aligned(4)));

// Byte e + 127 of a block from the bits of its largest magnitude; 255 where that is infinite or a NaN.  The exponent field
// less 2 is floor(log2 m) - 2 + 127; adding 0x3FFFFF first carries into it iff the significand is over 1.5, i.e. m > 6 * 2^e.
// Subnormal m, and zero, end at e = -127; e = 126 (m > 1.5 * 2^127, stochastic) is held at 125, where 6 is the end of the range.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int32_t e = (int32_t)((top + (STOCHASTIC ? 0x3FFFFFu : 0u)) >> 23) - 2;
    const uint32_t b = (uint32_t)(e < 0 ? 0 : e > 252 ? 252 : e);
    return top >= 0x7F800000u ? 255u : b;
}

// The fp32 bits of a magnitude of 16 bits.
template <uint32_t DT>
__device__ __forceinline__ uint32_t half_bits(uint32_t half) {
    if (DT == QESGD_BF16) return half << 16;
    return __float_as_uint((float)__builtin_bit_cast(_Float16, (unsigned short)half));
}

// Eight consecutive elements of a lane as they come from memory.
template <uint32_t DT>
struct Eight {
    typename std::conditional<DT == QESGD_F32, float[8], uvec4>::type v;

    __device__ __forceinline__ float at(int i) const {
        if constexpr (DT == QESGD_F32) return v[i];
        else if (DT == QESGD_BF16) return __uint_as_float((i & 1) ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
        else return (float)__builtin_bit_cast(_Float16, (unsigned short)((i & 1) ? v[i >> 1] >> 16 : v[i >> 1]));
    }
    // Bits of the largest magnitude, as integers: a NaN counts as the largest.
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (DT == QESGD_F32) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            return m;
        } else {
            ushort2v m = __builtin_bit_cast(ushort2v, v[0] & 0x7FFF7FFFu);
#pragma unroll
            for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, v[i] & 0x7FFF7FFFu));
            return half_bits<DT>(max((uint32_t)m[0], (uint32_t)m[1]));
        }
    }
    // From element `from` on, of which the first n (0..8) exist; the others are 0.
    __device__ __forceinline__ void load(const void* x, uint64_t from, uint32_t n) {
        if constexpr (DT == QESGD_F32) {
            const float* p = (const float*)x + from;
            if (n == 8) {
                const vec4 a = *(const vec4_any*)p, b = *(const vec4_any*)(p + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
            }
        } else {
            const unsigned short* p = (const unsigned short*)x + from;
            if (n == 8) {
                v = *(const uvec4_any*)p;
            } else {
                v = uvec4{0, 0, 0, 0};
#pragma unroll
                for (uint32_t i = 0; i < 7; ++i)
                    if (i < n) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
            }
        }
    }
};

// Two 16-bit elements to byte BYTE of a word of codes.
template <uint32_t DT, int BYTE>
__device__ __forceinline__ uint32_t convert2(uint32_t word, uint32_t pair, float scale) {
    if constexpr (DT == QESGD_BF16) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, __builtin_bit_cast(bf16x2, pair), scale, BYTE);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(word, __builtin_bit_cast(f16x2, pair), scale, BYTE);
}

// Codes of eight coordinates that share the scale byte sb, as one word.  `group`: number of their Philox call.
template <uint32_t DT, bool STOCHASTIC>
__device__ __forceinline__ uint32_t encode8(const Eight<DT>& x, uint32_t sb, uint64_t group, uint32_t worker, uint32_t round,
                                            uint32_t key0, uint32_t key1) {
    uint32_t word = 0;
    if (!STOCHASTIC) {
        // the conversions divide by the power of two in the scale's exponent field, round to nearest even and end at 6
        const float scale = __uint_as_float(sb << 23);
        if constexpr (DT == QESGD_F32) {
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x.v[0], x.v[1], scale, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x.v[2], x.v[3], scale, 1);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x.v[4], x.v[5], scale, 2);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x.v[6], x.v[7], scale, 3);
        } else {
            const uint32_t w0 = x.v[0], w1 = x.v[1], w2 = x.v[2], w3 = x.v[3];
            word = convert2<DT, 0>(word, w0, scale);
            word = convert2<DT, 1>(word, w1, scale);
            word = convert2<DT, 2>(word, w2, scale);
            word = convert2<DT, 3>(word, w3, scale);
        }
    } else {
        uint32_t rnd[4];
        philox4x32_10((uint32_t)group, (uint32_t)(group >> 32), worker, round, key0, key1, rnd);
        const float inv = __uint_as_float((254u - sb) << 23);              // 2^-e
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t r = variate16(rnd, i);
            const float v = x.at(i), a = fminf(__builtin_fabsf(v) * inv, 6.0f);          // over 6 only at e = 125
            // from 1 on the code is the exponent and the first bit of the significand (252 + code, and 252 is 4 modulo 8), and T its
            // next 16 bits: adding r there carries into the code iff r + T >= 2^16; below, the grid is a multiple of 1/2
            const uint32_t high = ((__float_as_uint(a) + (r << 6)) >> 22 & 7u) ^ 4u;
            const uint32_t low = ((uint32_t)(a * 131072.0f) + r) >> 16;
            word |= ((a < 1.0f ? low : high) | (__float_as_uint(v) >> 28 & 8u)) << (4 * i);
        }
    }
    return sb == 255u ? 0u : word;
}

// Over the four lanes of a quad, which share a block.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, false));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, false));
}
// The four quads of a row of 16 lanes: their bytes as one word, in every lane.
__device__ __forceinline__ uint32_t row_bytes(uint32_t byte, uint32_t lane) {
    uint32_t w = byte << (8u * ((lane >> 2) & 3u));
    w |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x124, 0xF, 0xF, false);   // row_ror:4
    w |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x128, 0xF, 0xF, false);   // row_ror:8
    return w;
}

struct QParams {
    const void* x;
    uint64_t ld, x_stride, rows, cols;
    uint64_t slots;                   // rows * wide
    uint32_t groups;                  // wide / 128
    uint32_t groups_t;                // the same of the transposed form
    unsigned char* packed;
    uint64_t packed_stride, scales_off;
    unsigned char* packed_t;
    uint64_t packed_t_stride, scales_t_off;
    uint32_t key0, key1, round, worker0;
    uint32_t xcd_group;
};

// Slots: the padded matrix, row after row.  A lane owns 8 consecutive ones (one Philox call, one word of codes), a quad a block,
// a wave kQChunks chunks of 512.  FLAT: the matrix is one row (a vector, or rows that need no padding and follow one another).
//
// Bound by its one read of x where rounding is cheap: 4096 x 25088 bf16 nearest 44 us = 5.9 TB/s, 16 vectors of 25.6 M f32 stochastic
// 331 us = 5.6 TB/s.  Stochastic 16-bit elements are bound by the vector instructions (a Philox call for 16 bytes): 5 matrices of 2737 x 2681
// 31 us = 3.0 TB/s.  One, two and four chunks a wave: 45.6 / 43.6 / 45.4, 340 / 331 / 330, 31.8 / 31.2 / 31.6 us.
constexpr uint32_t kQWaves = 4, kQChunks = 2;

template <uint32_t DT, bool STOCHASTIC, bool FLAT>
__global__ void __launch_bounds__(kQWaves * 64) k_mx4_quantize(const QParams p) {
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t wave0 = ((uint64_t)xcd_tile(blockIdx.x, gridDim.x, p.xcd_group) * kQWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) *
                           (kQChunks * kChunk);
    if (wave0 >= p.slots) return;
    const uint32_t k = blockIdx.y;
    const uint64_t x0 = (uint64_t)k * p.x_stride;
    Eight<DT> v[kQChunks];
    if (FLAT && wave0 + kQChunks * kChunk <= p.cols) {
        if constexpr (DT == QESGD_F32) {
            if ((((uintptr_t)p.x | (p.x_stride << 2)) & 15u) == 0) {
                vec4 a[kQChunks], b[kQChunks];
                load_halves_as<kQChunks, false>((const float*)p.x + x0 + wave0 + half_offset(lane), a, b);
#pragma unroll
                for (uint32_t c = 0; c < kQChunks; ++c) halves_to_lane(a[c], b[c], v[c].v);
            } else {
#pragma unroll
                for (uint32_t c = 0; c < kQChunks; ++c) v[c].load(p.x, x0 + wave0 + c * kChunk + lane * kLaneElems, 8u);
            }
        } else {
#pragma unroll
            for (uint32_t c = 0; c < kQChunks; ++c) v[c].load(p.x, x0 + wave0 + c * kChunk + lane * kLaneElems, 8u);
        }
    } else {
        const uint32_t group0 = (uint32_t)(wave0 >> 7), row0 = FLAT ? 0u : group0 / p.groups;       // uniform
#pragma unroll
        for (uint32_t c = 0; c < kQChunks; ++c) {
            const uint64_t slot = wave0 + c * kChunk + lane * kLaneElems;
            uint64_t row = 0, col = slot;
            if (!FLAT) {
                // the wave's 4 kQChunks groups of 128 end at most so many rows
                uint32_t r = row0, g = group0 - row0 * p.groups + c * 4u + (lane >> 4);
                if (p.groups >= 4u * kQChunks) {
                    const uint32_t over = g >= p.groups ? 1u : 0u;
                    r += over;
                    g -= over ? p.groups : 0u;
                } else {
                    const uint32_t more = g / p.groups;
                    r += more;
                    g -= more * p.groups;
                }
                row = r;
                col = (uint64_t)g * 128u + (lane & 15u) * 8u;
            }
            const uint32_t n = slot >= p.slots || col >= p.cols ? 0u : p.cols - col < 8 ? (uint32_t)(p.cols - col) : 8u;
            v[c].load(p.x, x0 + row * p.ld + col, n);
        }
    }
    unsigned char* out = p.packed + (uint64_t)k * p.packed_stride;
#pragma unroll
    for (uint32_t c = 0; c < kQChunks; ++c) {
        const uint64_t slot = wave0 + c * kChunk + lane * kLaneElems;
        const uint32_t sb = scale_byte<STOCHASTIC>(quad_max(v[c].top()));
        const uint32_t word = encode8<DT, STOCHASTIC>(v[c], sb, slot >> 3, p.worker0 + k, p.round, p.key0, p.key1);
        const uint32_t scales = row_bytes(sb, lane);
        if (slot < p.slots) {                                  // slots come in 128s: a row of lanes is in or out
            *(uint32_t*)(out + (slot >> 1)) = word;
            if ((lane & 15u) == 0) *(uint32_t*)(out + p.scales_off + (slot >> 5)) = scales;
        }
    }
}

// Both forms, or the transposed one alone, of a 128 x 128 tile.  The rows' form is made while the tile is read (a wave takes four
// rows at a time, a quad a block); the raw elements go to LDS, and then a lane takes 32 rows of one column.  8192 x 4096 bf16: nearest 26 us
// (4.0 TB/s of reads and writes), stochastic 52 us, which is its arithmetic: two Philox calls for 8 elements.  256 / 512 threads: 25.0 / 26.2 us
// there, 512 x 512 f32, which waits for its loads, 5.3 / 4.6.
constexpr uint32_t kTile = 128, kBothThreads = 512;

template <uint32_t DT, bool STOCHASTIC>
__global__ void __launch_bounds__(kBothThreads) k_mx4_quantize_both(const QParams p) {
    typedef typename std::conditional<DT == QESGD_F32, float, unsigned short>::type elem;
    // 32 rows, then 64 bytes of room: the four blocks of a column that a quad reads at once lie in different banks
    constexpr uint32_t kRoom = 64 / sizeof(elem);
    __shared__ __attribute__((aligned(16))) elem tile[kTile * kTile + 4 * kRoom];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, k = blockIdx.y;
    const uint32_t tr = blockIdx.x / p.groups, tc = blockIdx.x - tr * p.groups;
    const uint64_t r0 = (uint64_t)tr * kTile, c0 = (uint64_t)tc * kTile;
    const uint64_t x0 = (uint64_t)k * p.x_stride;
    const uint32_t col = (lane & 15u) * 8u;
    const uint32_t n = c0 + col >= p.cols ? 0u : p.cols - c0 - col < 8 ? (uint32_t)(p.cols - c0 - col) : 8u;
    Eight<DT> v[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint64_t row = r0 + i * 32u + wave * 4u + (lane >> 4);
        v[i].load(p.x, x0 + row * p.ld + c0 + col, row < p.rows ? n : 0u);
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t r = i * 32u + wave * 4u + (lane >> 4);
        const uint64_t row = r0 + r;
        elem* to = tile + r * kTile + (r >> 5) * kRoom + col;
        if constexpr (DT == QESGD_F32) {
            *(vec4*)to = vec4{v[i].v[0], v[i].v[1], v[i].v[2], v[i].v[3]};
            *(vec4*)(to + 4) = vec4{v[i].v[4], v[i].v[5], v[i].v[6], v[i].v[7]};
        } else {
            *(uvec4*)to = v[i].v;
        }
        if (p.packed) {
            const uint64_t slot = row * ((uint64_t)p.groups * 128u) + c0 + col;
            const uint32_t sb = scale_byte<STOCHASTIC>(quad_max(v[i].top()));
            const uint32_t word = encode8<DT, STOCHASTIC>(v[i], sb, slot >> 3, p.worker0 + k, p.round, p.key0, p.key1);
            const uint32_t scales = row_bytes(sb, lane);
            if (row < p.rows) {
                unsigned char* out = p.packed + (uint64_t)k * p.packed_stride;
                *(uint32_t*)(out + (slot >> 1)) = word;
                if ((lane & 15u) == 0) *(uint32_t*)(out + p.scales_off + (slot >> 5)) = scales;
            }
        }
    }
    __syncthreads();
    // A lane takes 32 rows of a column: one of 32-bit elements, or of 16-bit ones either of the pair that a word of LDS holds.
    const uint32_t block = lane & 3u, word_col = DT == QESGD_F32 ? threadIdx.x >> 2 : (threadIdx.x >> 2) & 63u;
    const uint32_t side = DT == QESGD_F32 ? 0u : threadIdx.x >> 8;
    const uint32_t* from = (const uint32_t*)tile + block * (32u * kTile + kRoom) * sizeof(elem) / 4u + word_col;
    uint32_t raw[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) raw[j] = from[j * (kTile * sizeof(elem) / 4u)];
    Eight<DT> y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (DT == QESGD_F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[j].v[e] = __uint_as_float(raw[j * 8 + e]);
        } else {
            // the lower (upper) halves of two rows' words, as a pair along the column
            const uint32_t pick = side ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[j].v[e] = __builtin_amdgcn_perm(raw[j * 8 + 2 * e + 1], raw[j * 8 + 2 * e], pick);
        }
    }
    const uint32_t c = DT == QESGD_F32 ? word_col : word_col * 2u + side;
    const uint32_t sb = scale_byte<STOCHASTIC>(max(max(y[0].top(), y[1].top()), max(y[2].top(), y[3].top())));
    const uint64_t slot = (c0 + c) * ((uint64_t)p.groups_t * 128u) + r0 + block * 32u;
    uvec4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = encode8<DT, STOCHASTIC>(y[j], sb, (slot >> 3) + j, p.worker0 + k, p.round, p.key0, p.key1);
    uint32_t scales = sb << (8u * block);
    scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0xB1, 0xF, 0xF, false);
    scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x4E, 0xF, 0xF, false);
    if (c0 + c < p.cols) {
        unsigned char* out = p.packed_t + (uint64_t)k * p.packed_t_stride;
        *(uvec4*)(out + (slot >> 1)) = w;
        if (block == 0) *(uint32_t*)(out + p.scales_t_off + (slot >> 5)) = scales;
    }
}

struct AParams {
    const unsigned char* packed;
    uint64_t packed_stride, scales_off;
    uint64_t slots, cols;
    uint32_t groups, K;
    const float* w;
    float* zbar;
    float* u;
    float* zsum;
    float inv_k, k;
    bool pow2;
    uint32_t xcd_group;
};

// A lane owns 8 slots again: a word of codes and a scale byte per worker, decoded by the conversion that multiplies by a power of
// two (exact); workers are added in order from +0.  Bound by the streams: 16 workers of 25.6 M 106 us = 6.9 TB/s.
template <bool FLAT>
__global__ void __launch_bounds__(256) k_mx4_aggregate_update(const AParams p) {
    const uint32_t lane = threadIdx.x & 63u;
    const uint64_t slot0 = ((uint64_t)xcd_tile(blockIdx.x, gridDim.x, p.xcd_group) * 4u + (threadIdx.x >> 6)) * kChunk;
    const uint64_t slot = slot0 + lane * kLaneElems;
    if (slot >= p.slots) return;
    uint64_t at = slot;
    uint32_t n = 8;
    const bool whole = FLAT && slot0 + kChunk <= p.cols;       // uniform
    if (!whole) {
        uint64_t row = 0, col = slot;
        if (!FLAT) {
            const uint32_t g = (uint32_t)(slot >> 7);
            row = g / p.groups;
            col = (uint64_t)(g - (uint32_t)row * p.groups) * 128u + (slot & 127u);
        }
        n = col >= p.cols ? 0u : p.cols - col < 8 ? (uint32_t)(p.cols - col) : 8u;
        at = row * p.cols + col;
    }
    const unsigned char* codes = p.packed + (slot >> 1);
    const unsigned char* scales = p.packed + p.scales_off + (slot >> 5);
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t k = 0;
    auto add = [&](uint32_t word, uint32_t byte) {
        const float s = __uint_as_float(byte << 23);            // the conversion reads the exponent field; 255 gives NaN
        const fvec2 q0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 0), q1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 1);
        const fvec2 q2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 2), q3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, s, 3);
        acc[0] += q0[0]; acc[1] += q0[1]; acc[2] += q1[0]; acc[3] += q1[1];
        acc[4] += q2[0]; acc[5] += q2[1]; acc[6] += q3[0]; acc[7] += q3[1];
    };
    for (; k + 4 <= p.K; k += 4) {
        uint32_t word[4], byte[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            word[j] = *(const uint32_t*)(codes + (k + j) * p.packed_stride);
            byte[j] = scales[(k + j) * p.packed_stride];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) add(word[j], byte[j]);
    }
    for (; k < p.K; ++k) add(*(const uint32_t*)(codes + k * p.packed_stride), scales[k * p.packed_stride]);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = p.pow2 ? acc[i] * p.inv_k : acc[i] / p.k;

    if (whole) {
        const uint64_t h = slot0 + half_offset(lane);
        vec4 za, zb;
        lane_to_halves(acc, za, zb);
        if (p.zbar) { store_stream(p.zbar + h, za); store_stream(p.zbar + h + kChunk / 2, zb); }
        if (p.u) {
            store_stream(p.u + h, load_stream(p.w + h) + za);
            store_stream(p.u + h + kChunk / 2, load_stream(p.w + h + kChunk / 2) + zb);
        }
        if (p.zsum) {
            store_stream(p.zsum + h, load_stream(p.zsum + h) + za);
            store_stream(p.zsum + h + kChunk / 2, load_stream(p.zsum + h + kChunk / 2) + zb);
        }
    } else if (n == 8) {
        const vec4 za = {acc[0], acc[1], acc[2], acc[3]}, zb = {acc[4], acc[5], acc[6], acc[7]};
        if (p.zbar) { *(vec4_any*)(p.zbar + at) = za; *(vec4_any*)(p.zbar + at + 4) = zb; }
        if (p.u) {
            const vec4 a = *(const vec4_any*)(p.w + at) + za, b = *(const vec4_any*)(p.w + at + 4) + zb;
            *(vec4_any*)(p.u + at) = a;
            *(vec4_any*)(p.u + at + 4) = b;
        }
        if (p.zsum) {
            const vec4 a = *(const vec4_any*)(p.zsum + at) + za, b = *(const vec4_any*)(p.zsum + at + 4) + zb;
            *(vec4_any*)(p.zsum + at) = a;
            *(vec4_any*)(p.zsum + at + 4) = b;
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 7; ++i) {
            if (i >= n) break;
            if (p.zbar) p.zbar[at + i] = acc[i];
            if (p.u) p.u[at + i] = p.w[at + i] + acc[i];
            if (p.zsum) p.zsum[at + i] += acc[i];
        }
    }
}

int finish_launch() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return QESGD_OK;
    set_last_hip_error((int)e);
    return QESGD_ERR_HIP;
}

template <uint32_t DT, bool STOCHASTIC>
int launch_quantize_as(const Mx4Quantize& a, QParams& p, bool flat) {
    if (p.packed_t) {
        const uint64_t tiles = ((a.rows + kTile - 1) / kTile) * p.groups;
        if (!grid_ok(tiles, kBothThreads)) return QESGD_ERR_DIM;
        k_mx4_quantize_both<DT, STOCHASTIC><<<dim3((uint32_t)tiles, a.K), kBothThreads, 0, a.stream>>>(p);
        return finish_launch();
    }
    constexpr uint64_t tile = kQWaves * kQChunks * kChunk;
    const uint64_t tiles = (p.slots + tile - 1) / tile;
    if (!grid_ok(tiles, kQWaves * 64)) return QESGD_ERR_DIM;
    p.xcd_group = xcd_group_log2(tile);
    const dim3 grid((uint32_t)tiles, a.K);
    if (flat) k_mx4_quantize<DT, STOCHASTIC, true><<<grid, kQWaves * 64, 0, a.stream>>>(p);
    else k_mx4_quantize<DT, STOCHASTIC, false><<<grid, kQWaves * 64, 0, a.stream>>>(p);
    return finish_launch();
}

template <uint32_t DT>
int launch_quantize_type(const Mx4Quantize& a, QParams& p, bool flat) {
    return a.stochastic ? launch_quantize_as<DT, true>(a, p, flat) : launch_quantize_as<DT, false>(a, p, flat);
}

}  // namespace

int launch_mx4_quantize(const Mx4Quantize& a) {
    qesgd_mx4_layout L{}, T{};
    int rc = make_mx4_layout(a.rows, a.cols, &L);
    if (rc == QESGD_OK && a.packed_t) rc = make_mx4_layout(a.cols, a.rows, &T);
    if (rc != QESGD_OK) return rc;
    QParams p{};
    p.x = a.x;
    p.ld = a.ld;
    p.x_stride = a.x_stride;
    p.rows = a.rows;
    p.cols = a.cols;
    p.groups = (uint32_t)(L.row_codes / 64);
    p.groups_t = (uint32_t)(T.row_codes / 64);
    p.slots = a.rows * L.row_codes * 2;
    p.packed = a.packed;
    p.packed_stride = a.packed_stride;
    p.scales_off = L.scales_off;
    p.packed_t = a.packed_t;
    p.packed_t_stride = a.packed_t_stride;
    p.scales_t_off = T.scales_off;
    p.key0 = (uint32_t)a.seed;
    p.key1 = (uint32_t)(a.seed >> 32);
    p.round = a.round;
    p.worker0 = a.worker0;
    const bool flat = !a.packed_t && (a.rows == 1 || (a.cols % kMx4Pad == 0 && a.ld == a.cols));
    if (flat) p.cols = a.rows * a.cols;
    switch (a.dtype) {
        case QESGD_F32: return launch_quantize_type<QESGD_F32>(a, p, flat);
        case QESGD_BF16: return launch_quantize_type<QESGD_BF16>(a, p, flat);
        default: return launch_quantize_type<QESGD_F16>(a, p, flat);
    }
}

int launch_mx4_aggregate(const Mx4Aggregate& a) {
    qesgd_mx4_layout L;
    const int rc = make_mx4_layout(a.rows, a.cols, &L);
    if (rc != QESGD_OK) return rc;
    AParams p{};
    p.packed = a.packed;
    p.packed_stride = a.packed_stride;
    p.scales_off = L.scales_off;
    p.slots = a.rows * L.row_codes * 2;
    p.groups = (uint32_t)(L.row_codes / 64);
    p.K = a.K;
    p.w = a.w;
    p.zbar = a.zbar;
    p.u = a.u;
    p.zsum = a.zsum;
    p.pow2 = (a.K & (a.K - 1)) == 0;
    p.k = (float)a.K;
    p.inv_k = 1.0f / (float)a.K;
    const bool flat = a.rows == 1 || a.cols % kMx4Pad == 0;
    p.cols = flat ? a.rows * a.cols : a.cols;
    const uint64_t tiles = (p.slots + 4 * kChunk - 1) / (4 * kChunk);
    if (!grid_ok(tiles, 256)) return QESGD_ERR_DIM;
    p.xcd_group = xcd_group_log2(4 * kChunk);
    if (flat) k_mx4_aggregate_update<true><<<(uint32_t)tiles, 256, 0, a.stream>>>(p);
    else k_mx4_aggregate_update<false><<<(uint32_t)tiles, 256, 0, a.stream>>>(p);
    return finish_launch();
}

}  // namespace qesgd
