// The weighted sum of a token's rows, and its gradients.
//
//   out[t] = sum_j gates[t, j] rows[slot(t, j)];  drows[slot(t, j)] = gates[t, j] dy[t];  dgates[t, j] = <dy[t], rows[slot(t, j)]>
//
// Sums in fp32, in order of j and, for the products with dy, lane by lane and then over the lanes, always in the same order.  Rows in fp32 beside results of 16 bits, which are then
// rounded once, or of the results' type.  Bound by the bytes: 16384 tokens x 2 rows x 4096 bf16, two sets in turn, sum 75 us = 5.4 TB/s (the same rows again 61), gradients 102 us =
// 6.6 TB/s; with rows of fp32 113 = 5.9 and 158 = 6.0.  A call of 517 x 3 x 1001 is a launch and three trips to memory, 5 us.
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
    uint32_t block0;                  // of the launch, where the gradients take several
};

// Sixteen bytes of a row, or the n elements that are left of it.
template <uint32_t DT>
struct Piece {
    static constexpr uint32_t V = DT == QESGD_F32 ? 4 : 8;
    uvec4 v;

    // STREAM: non-temporal
    template <bool STREAM>
    __device__ __forceinline__ void load(const void* x, uint64_t at, uint32_t n) {
        if constexpr (DT == QESGD_F32) {
            const float* p = (const float*)x + at;
            if (n >= V) {
                if (STREAM) v = __builtin_bit_cast(uvec4, __builtin_nontemporal_load((const vec4_any*)p));
                else v = __builtin_bit_cast(uvec4, *(const vec4_any*)p);
            } else {
                v = uvec4{0, 0, 0, 0};
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) v[i] = __float_as_uint(p[i]);
            }
        } else {
            const unsigned short* p = (const unsigned short*)x + at;
            if (n >= V) {
                if (STREAM) v = __builtin_nontemporal_load((const uvec4_any*)p);
                else v = *(const uvec4_any*)p;
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
    template <bool STREAM>
    __device__ __forceinline__ void store(void* x, uint64_t at, uint32_t n) const {
        if constexpr (DT == QESGD_F32) {
            float* p = (float*)x + at;
            if (n >= V) {
                if (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(vec4, v), (vec4_any*)p);
                else *(vec4_any*)p = __builtin_bit_cast(vec4, v);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) p[i] = __uint_as_float(v[i]);
            }
        } else {
            unsigned short* p = (unsigned short*)x + at;
            if (n >= V) {
                if (STREAM) __builtin_nontemporal_store(v, (uvec4_any*)p);
                else *(uvec4_any*)p = v;
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V - 1; ++i)
                    if (i < n) p[i] = (unsigned short)(v[i >> 1] >> (16 * (i & 1)));
            }
        }
    }
};

// As many elements of a row of type RT as sixteen bytes of type DT hold: one piece, or two where the rows are fp32 beside results of 16 bits.
template <uint32_t DT, uint32_t RT>
struct RowPiece {
    static constexpr uint32_t V = Piece<RT>::V, P = Piece<DT>::V / V;
    Piece<RT> part[P];

    template <bool STREAM>
    __device__ __forceinline__ void load(const void* x, uint64_t at, uint32_t n) {
#pragma unroll
        for (uint32_t i = 0; i < P; ++i) part[i].template load<STREAM>(x, at + i * V, n > i * V ? n - i * V : 0u);
    }
    __device__ __forceinline__ float at(uint32_t i) const { return part[i / V].at((int)(i % V)); }
};

// A thread a piece of a token's row.  STREAM: out is written non-temporally.
template <uint32_t DT, uint32_t RT, bool STREAM>
__global__ void __launch_bounds__(256) k_combine(const CParams p) {
    constexpr uint32_t V = Piece<DT>::V;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, token = i / p.vectors;         // a launch has fewer than 2^32 threads
    if (token >= p.T) return;
    const uint64_t t = token;
    const uint32_t col = (i - token * p.vectors) * V, n = p.N - col;
    float sum[V];
#pragma unroll
    for (uint32_t e = 0; e < V; ++e) sum[e] = 0.0f;
    for (uint32_t j = 0; j < p.k; ++j) {
        const uint64_t pair = t * p.k + j;
        const uint32_t slot = p.slots ? (uint32_t)p.slots[pair] : (uint32_t)pair;
        if (slot >= p.R) continue;
        const float g = p.gates ? p.gates[pair] : 1.0f;
        RowPiece<DT, RT> x;
        x.template load<false>(p.rows, slot * p.ld + col, n);
#pragma unroll
        for (uint32_t e = 0; e < V; ++e) sum[e] += g * x.at(e);
    }
    Piece<DT> y;
    y.set(sum);
    y.template store<STREAM>(p.out, t * p.ld_out + col, n);
}

// Policies of the backward pass: rows' gradients written non-temporally, and rows read so too.
enum { kKept = 0, kStreamOut = 1, kStreamBoth = 2 };

// L lanes a token (256: a workgroup); KM: at least k.
template <uint32_t DT, uint32_t RT, uint32_t L, int KM, int POLICY>
__global__ void __launch_bounds__(256) k_combine_backward(const CParams p) {
    constexpr uint32_t V = Piece<DT>::V, tokens = 256 / L;
    constexpr bool OUT = POLICY != kKept, IN = POLICY == kStreamBoth;
    __shared__ float sums[4][KM];
    const uint32_t lane = threadIdx.x % L;
    const uint64_t t = (uint64_t)(p.block0 + blockIdx.x) * tokens + threadIdx.x / L;
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
        for (uint32_t c = lane; c < p.vectors; c += L) {
            const uint32_t col = c * V, n = p.N - col;
            Piece<DT> d;
            RowPiece<DT, RT> x[KM];
            d.template load<false>(p.dy, t * p.ld_dy + col, n);
            if (p.dgates) {
#pragma unroll
                for (int j = 0; j < KM; ++j)
                    if (slot[j] < p.R) x[j].template load<IN>(p.rows, slot[j] * p.ld + col, n);
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
                        y.template store<OUT>(p.drows, slot[j] * p.ld_d + col, n);
                    }
            }
        }
    }
    if (!p.dgates) return;
    constexpr uint32_t W = L < 64 ? L : 64;
#pragma unroll
    for (int j = 0; j < KM; ++j)
#pragma unroll
        for (uint32_t m = 1; m < W; m <<= 1) dot[j] += __shfl_xor(dot[j], (int)m);
    if (L <= 64) {
#pragma unroll
        for (int j = 0; j < KM; ++j)
            if (there && lane == (uint32_t)j % W && (uint32_t)j < p.k) p.dgates[t * p.k + j] = dot[j];
        return;
    }
#pragma unroll
    for (int j = 0; j < KM; ++j)
        if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6][j] = dot[j];
    __syncthreads();
    if (threadIdx.x < p.k) p.dgates[t * p.k + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
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

// A result of whole lines, of a call that moves more than the memory-side cache keeps for the next one, is written non-temporally, us without / with:
// 16384 tokens x 2 rows x 4096 bf16 78 / 58, gradients 134 / 131, and 112 with the rows read so too, where they alone are more than that cache; 8192 tokens 30 / 30, 68 / 51 and
// 58; 65536 x 1 x 1024 40 / 40, 77 / 59 and 63; small calls the same.
constexpr uint64_t kStreamMoved = 128ull << 20, kStreamRows = 256ull << 20;
static bool whole_lines(const void* p, uint64_t ld, uint32_t dtype) { return ((uintptr_t)p | ld * dtype_bytes(dtype)) % 128 == 0; }

// f(types of the results and of the rows, as constants): the same, or rows of fp32.
template <class F>
static void by_types(const Combine& a, F&& f) {
    by_type(a.dtype, [&](auto t) {
        if (a.rows_dtype == t.value) f(t, t);
        else f(t, std::integral_constant<uint32_t, QESGD_F32>{});
    });
}

int launch_combine(const Combine& a) {
    const CParams p = params(a);
    const uint64_t groups = ((uint64_t)p.T * p.vectors + 255) / 256, moved = a.N * (a.T * a.k * dtype_bytes(a.rows_dtype) + a.T * dtype_bytes(a.dtype));
    if (!grid_ok(groups, 256)) return QESGD_ERR_DIM;
    const bool stream = moved >= kStreamMoved && whole_lines(a.out, a.ld_out, a.dtype);
    by_types(a, [&](auto t, auto r) {
        if (stream) k_combine<t.value, r.value, true><<<(uint32_t)groups, 256, 0, a.stream>>>(p);
        else k_combine<t.value, r.value, false><<<(uint32_t)groups, 256, 0, a.stream>>>(p);
    });
    return launched();
}

int launch_combine_backward(const Combine& a) {
    CParams p = params(a);
    // lanes of a token: a workgroup for long rows, for short ones no more than have work
    const uint32_t lanes = p.vectors > 128 ? 256 : p.vectors > 16 ? 64 : p.vectors > 8 ? 16 : 8;
    const uint64_t tokens = 256 / lanes, groups = (p.T + tokens - 1) / tokens, pairs = a.T * a.k, rows = a.N * pairs * dtype_bytes(a.rows_dtype);
    const bool stream = a.drows && rows + a.N * pairs * dtype_bytes(a.dtype) >= kStreamMoved && whole_lines(a.drows, a.ld_d, a.dtype);
    int rc = QESGD_OK;
    const auto go = [&](auto t, auto r, auto l, auto km) {
        constexpr uint32_t DT = t.value, RT = r.value, L = l.value;
        constexpr int KM = km.value;
        const auto launch = [&](auto policy) {
            rc = by_launches(groups, 256, [&](uint32_t first, uint32_t count) {
                p.block0 = first;
                k_combine_backward<DT, RT, L, KM, policy.value><<<count, 256, 0, a.stream>>>(p);
            });
        };
        // rows of up to 256 bytes are not streamed: a call of them has to have a million
        if (L == 256 && stream && rows >= kStreamRows) launch(std::integral_constant<int, L == 256 ? kStreamBoth : kKept>{});
        else if (L >= 64 && stream) launch(std::integral_constant<int, L >= 64 ? kStreamOut : kKept>{});
        else launch(std::integral_constant<int, kKept>{});
    };
    const auto by_choices = [&](auto t, auto r, auto l) {
        using std::integral_constant;
        if (p.k <= 2) go(t, r, l, integral_constant<int, 2>{});
        else if (p.k <= 4) go(t, r, l, integral_constant<int, 4>{});
        else if (p.k <= 8) go(t, r, l, integral_constant<int, 8>{});
        else go(t, r, l, integral_constant<int, 16>{});
    };
    by_types(a, [&](auto t, auto r) {
        using std::integral_constant;
        switch (lanes) {
            case 8: by_choices(t, r, integral_constant<uint32_t, 8>{}); break;
            case 16: by_choices(t, r, integral_constant<uint32_t, 16>{}); break;
            case 64: by_choices(t, r, integral_constant<uint32_t, 64>{}); break;
            default: by_choices(t, r, integral_constant<uint32_t, 256>{}); break;
        }
    });
    return rc;
}

}  // namespace qesgd
