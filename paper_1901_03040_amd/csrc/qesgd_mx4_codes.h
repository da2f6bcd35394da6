// Elements of matrices to 4-bit microscaled codes: what the quantising kernels share (not installed).
//
// Block of 32 coordinates with largest magnitude m: scale 2^e, element q of {0, .5, 1, 1.5, 2, 3, 4, 6} with a sign.
//   nearest     e = floor(log2 m) - 2, q = |v| / 2^e to nearest even, at most 6
//   stochastic  e = the smallest with m <= 6 * 2^e, q one of the two neighbours of a = |v| / 2^e: up iff r + T >= 2^16,
//               T = trunc(f * 2^16), f the fraction of the way; E[q] = a to 2^-16 of a step
// a is exact (a power of two only moves the exponent; what falls below fp32's range is far below the grid).
#pragma once

#include <type_traits>

#include "qesgd_device.h"
#include "qesgd_matrix.h"

namespace qesgd {

typedef uint32_t uvec4 __attribute__((ext_vector_type(4)));
typedef uint32_t uvec2 __attribute__((ext_vector_type(2)));
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
    // From element `from` on; zeros where there is none.
    __device__ __forceinline__ void load_whole(const void* x, uint64_t from, bool there) {
        if constexpr (DT == QESGD_F32) {
            vec4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
            if (there) {
                const float* p = (const float*)x + from;
                a = *(const vec4_any*)p;
                b = *(const vec4_any*)(p + 4);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
            v = uvec4{0, 0, 0, 0};
            if (there) v = *(const uvec4_any*)((const unsigned short*)x + from);
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

// From here on fp32 results that do not fit are cut off: what encode8 wants of subnormal numbers.  All else that the quantising kernels compute in fp32 is exact.
__device__ __forceinline__ void round_down() { __builtin_amdgcn_s_setreg(1 | (2 - 1) << 11, 3); }     // the two bits of the mode register for fp32

// Codes of eight coordinates that share the scale byte sb, as one word.  `group`: number of their Philox call.  STOCHASTIC: after round_down.
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
        // Times 2^-126, the least normal number, an element's code is bits 22 to 24, which above 1 are the exponent and the first bit of the significand and
        // below, as the number is subnormal, a multiple of 1/2; T is the 16 bits under them, cut off and not rounded (see round_down),
        // and adding r there carries into the code iff r + T >= 2^16.
        const auto append = [&](float v, uint32_t r) {
            const uint32_t code = __float_as_uint(v) + (r << 6);
            word = __builtin_amdgcn_alignbit(word, (code & 0x80000000u) | (code << 6 & ~0x80000000u), 28);         // the sign and those bits behind the word
        };
        const float inv = __builtin_ldexpf(1.0f, 1 - (int)sb);             // 2^-e 2^-126, a subnormal number from e = 1 on
        if (__builtin_expect(__ballot(sb > 150u) == 0, 1)) {
#pragma unroll
            for (int i = 7; i >= 0; --i) append(x.at(i) * inv, variate16(rnd, i));
        } else {
            // beyond e = 23 that is too small for a number; and where e stays at 125, what lies over 6 ends there
            const float by = __uint_as_float((254u - sb) << 23);
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const float v = x.at(i);
                append(__builtin_copysignf(fminf(__builtin_fabsf(v) * by, 6.0f) * 0x1p-126f, v), variate16(rnd, i));
            }
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

}  // namespace qesgd
