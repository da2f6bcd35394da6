// The weighted sum of a token's rows, and its gradients.
//
//   out[t] = sum_j gates[t, j] rows[slot(t, j)];  drows[slot(t, j)] = gates[t, j] dy[t];  dgates[t, j] = <dy[t], rows[slot(t, j)]>
//
// Sums in fp32, in order of j and, for the products with dy, lane by lane and then over the lanes, always in the same order.
#include "qesgd_experts.h"
#include "qesgd_launch.h"
#include "qesgd_mx4_codes.h"

namespace qesgd {
namespace {

struct CParams {
    const void* rows;
    uint64_t ld;
    uint32_t R;
    const int32_t* slots;
    const float* gates;
    uint32_t T, k;
    uint32_t N, vectors;              // of a row: sixteen bytes each, the last one as long as the row is
    void* out;
    uint64_t ld_out;
    const void* dy;
    uint64_t ld_dy;
    void* drows;
    uint64_t ld_d;
    float* dgates;
};

// Sixteen bytes of a row, or the n elements that are left of it.
template <uint32_t DT>
struct Piece {
    static constexpr uint32_t V = DT == QESGD_F32 ? 4 : 8;
    uvec4 v;

    __device__ __forceinline__ void load(const void* x, uint64_t at, uint32_t n) {
        if constexpr (DT == QESGD_F32) {
            const float* p = (const float*)x + at;
            if (n >= V) {
                v = __builtin_bit_cast(uvec4, *(const vec4_any*)p);
            } else {
                v = uvec4{0, 0, 0, 0};
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) v[i] = __float_as_uint(p[i]);
            }
        } else {
            const unsigned short* p = (const unsigned short*)x + at;
            if (n >= V) {
                v = *(const uvec4_any*)p;
            } else {
                v = uvec4{0, 0, 0, 0};
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
            }
        }
    }
    __device__ __forceinline__ float at(int i) const {
        if (DT == QESGD_F32) return __uint_as_float(v[i]);
        if (DT == QESGD_BF16) return __uint_as_float((i & 1) ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
        return (float)__builtin_bit_cast(_Float16, (unsigned short)((i & 1) ? v[i >> 1] >> 16 : v[i >> 1]));
    }
    __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            if constexpr (DT == QESGD_F32) v[i] = __float_as_uint(x[i]);
            else if constexpr (DT == QESGD_BF16) v[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
            else v[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * i], (_Float16)x[2 * i + 1]});
        }
    }
    __device__ __forceinline__ void store(void* x, uint64_t at, uint32_t n) const {
        if constexpr (DT == QESGD_F32) {
            float* p = (float*)x + at;
            if (n >= V) {
                *(vec4_any*)p = __builtin_bit_cast(vec4, v);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) p[i] = __uint_as_float(v[i]);
            }
        } else {
            unsigned short* p = (unsigned short*)x + at;
            if (n >= V) {
                *(uvec4_any*)p = v;
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) p[i] = (unsigned short)(v[i >> 1] >> (16 * (i & 1)));
            }
        }
    }
};

// A thread a piece of a token's row.
template <uint32_t DT>
__global__ void __launch_bounds__(256) k_combine(const CParams p) {
    constexpr uint32_t V = Piece<DT>::V;
    const uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    const uint64_t t = i / p.vectors;
    if (t >= p.T) return;
    const uint32_t col = (uint32_t)(i - t * p.vectors) * V, n = p.N - col;
    float sum[V];
#pragma unroll
    for (uint32_t e = 0; e < V; ++e) sum[e] = 0.0f;
    for (uint32_t j = 0; j < p.k; ++j) {
        const uint64_t pair = t * p.k + j;
        const uint32_t slot = p.slots ? (uint32_t)p.slots[pair] : (uint32_t)pair;
        if (slot >= p.R) continue;
        const float g = p.gates ? p.gates[pair] : 1.0f;
        Piece<DT> x;
        x.load(p.rows, slot * p.ld + col, n);
#pragma unroll
        for (uint32_t e = 0; e < V; ++e) sum[e] += g * x.at(e);
    }
    Piece<DT> y;
    y.set(sum);
    y.store(p.out, t * p.ld_out + col, n);
}

// W waves a token; KM: at least k.
template <uint32_t DT, int W, int KM>
__global__ void __launch_bounds__(256) k_combine_backward(const CParams p) {
    constexpr uint32_t V = Piece<DT>::V, tokens = 4 / W;
    __shared__ float sums[4][KM];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint64_t t = (uint64_t)blockIdx.x * tokens + wave / W;
    const bool there = t < p.T;
    float dot[KM], gate[KM];
    uint32_t slot[KM];
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        dot[j] = 0.0f;
        gate[j] = 0.0f;
        slot[j] = 0xFFFFFFFFu;
        if (there && (uint32_t)j < p.k) {
            const uint64_t pair = t * p.k + j;
            slot[j] = p.slots ? (uint32_t)p.slots[pair] : (uint32_t)pair;
            if (p.drows) gate[j] = p.gates[pair];
        }
    }
    if (there) {
        for (uint32_t c = (wave % W) * 64u + lane; c < p.vectors; c += W * 64u) {
            const uint32_t col = c * V, n = p.N - col;
            Piece<DT> d, x[KM];
            d.load(p.dy, t * p.ld_dy + col, n);
            if (p.dgates) {
#pragma unroll
                for (int j = 0; j < KM; ++j)
                    if (slot[j] < p.R) x[j].load(p.rows, slot[j] * p.ld + col, n);
#pragma unroll
                for (int j = 0; j < KM; ++j)
                    if (slot[j] < p.R) {
#pragma unroll
                        for (uint32_t e = 0; e < V; ++e) dot[j] += d.at(e) * x[j].at(e);
                    }
            }
            if (p.drows) {
#pragma unroll
                for (int j = 0; j < KM; ++j)
                    if (slot[j] < p.R) {
                        float v[V];
#pragma unroll
                        for (uint32_t e = 0; e < V; ++e) v[e] = gate[j] * d.at(e);
                        Piece<DT> y;
                        y.set(v);
                        y.store(p.drows, slot[j] * p.ld_d + col, n);
                    }
            }
        }
    }
    if (!p.dgates) return;
#pragma unroll
    for (int j = 0; j < KM; ++j) {
        for (int m = 1; m < 64; m <<= 1) dot[j] += __shfl_xor(dot[j], m);
        if (lane == 0) sums[wave][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < tokens * KM) {
        const uint32_t of = threadIdx.x / KM, j = threadIdx.x % KM;
        const uint64_t token = (uint64_t)blockIdx.x * tokens + of;
        if (token < p.T && j < p.k) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) v += sums[of * W + w][j];
            p.dgates[token * p.k + j] = v;
        }
    }
}

CParams params(const Combine& a) {
    CParams p{};
    p.rows = a.rows;
    p.ld = a.ld;
    p.R = (uint32_t)a.R;
    p.slots = a.slots;
    p.gates = a.gates;
    p.T = (uint32_t)a.T;
    p.k = a.k;
    p.N = (uint32_t)a.N;
    const uint32_t V = 16 / dtype_bytes(a.dtype);
    p.vectors = (p.N + V - 1) / V;
    p.out = a.out;
    p.ld_out = a.ld_out;
    p.dy = a.dy;
    p.ld_dy = a.ld_dy;
    p.drows = a.drows;
    p.ld_d = a.ld_d;
    p.dgates = a.dgates;
    return p;
}

}  // namespace

int launch_combine(const Combine& a) {
    const CParams p = params(a);
    const uint64_t groups = ((uint64_t)p.T * p.vectors + 255) / 256;
    if (!grid_ok(groups, 256)) return QESGD_ERR_DIM;
    by_type(a.dtype, [&](auto t) { k_combine<t.value><<<(uint32_t)groups, 256, 0, a.stream>>>(p); });
    return launched();
}

int launch_combine_backward(const Combine& a) {
    const CParams p = params(a);
    const bool wide = p.vectors > 128;
    const uint64_t groups = wide ? p.T : (p.T + 3) / 4;
    if (!grid_ok(groups, 256)) return QESGD_ERR_DIM;
    const auto by_choices = [&](auto f) {
        using std::integral_constant;
        if (p.k <= 2) f(integral_constant<int, 2>{});
        else if (p.k <= 4) f(integral_constant<int, 4>{});
        else if (p.k <= 8) f(integral_constant<int, 8>{});
        else f(integral_constant<int, 16>{});
    };
    by_type(a.dtype, [&](auto t) {
        by_choices([&](auto km) {
            if (wide) k_combine_backward<t.value, 4, km.value><<<(uint32_t)groups, 256, 0, a.stream>>>(p);
            else k_combine_backward<t.value, 1, km.value><<<(uint32_t)groups, 256, 0, a.stream>>>(p);
        });
    });
    return launched();
}

}  // namespace qesgd
