// Internal declarations of the operators for layers of experts: the router, products by groups of rows, products of single rows (not installed).
#pragma once

#include "qesgd_matrix.h"

namespace qesgd {

constexpr uint64_t kMaxPairs = 1ull << 28;               // T * k: their numbers, and four bytes each, stay within 32 bits
constexpr uint64_t kMaxLogits = 1ull << 36;

struct Route {
    const void* logits;
    uint32_t dtype;
    uint64_t ld, T;
    uint32_t E, k;
    bool all;                       // gates over all logits
    int32_t* experts;
    float* gates;
    int32_t* offsets;
    int32_t* order;
    int32_t* slots;
    uint32_t* workspace;
    hipStream_t stream;
};
struct RouteBackward {
    const void* logits;             // nullable unless all
    uint32_t dtype;
    uint64_t ld, T;
    uint32_t E, k;
    bool all;
    const int32_t* experts;
    const float* gates;
    const float* dgates;
    void* dlogits;
    uint64_t ld_d;
    hipStream_t stream;
};
size_t route_workspace(uint64_t T, uint32_t E, uint32_t k);
int launch_route(const Route& a);
int launch_route_backward(const RouteBackward& a);

struct Combine {
    const void* rows;
    uint32_t dtype, rows_dtype;     // of the rest; of rows: the same or fp32
    uint64_t ld, R;
    const int32_t* slots;           // nullable
    const float* gates;             // nullable
    uint64_t T;
    uint32_t k;
    uint64_t N;
    void* out;
    uint64_t ld_out;
    // backward
    const void* dy;
    uint64_t ld_dy;
    void* drows;                    // nullable
    uint64_t ld_d;
    float* dgates;                  // nullable
    hipStream_t stream;
};
int launch_combine(const Combine& a);
int launch_combine_backward(const Combine& a);

struct GroupQuantize {
    const void* x;
    uint32_t dtype;
    uint64_t ld, T;
    const int32_t* order;           // nullable
    uint32_t per;
    const int32_t* offsets;
    uint32_t E;
    uint64_t R, cols;
    bool stochastic;
    uint64_t seed;
    uint32_t round, worker;
    unsigned char* packed;          // nullable
    unsigned char* packed_t;        // nullable
    hipStream_t stream;
};
int launch_quantize_groups(const GroupQuantize& a);

struct GroupProduct {
    const unsigned char* a;
    const unsigned char* b;
    uint64_t b_stride;
    const int32_t* offsets;
    uint32_t E;
    uint64_t R, N, K;
    void* c;
    uint32_t dtype;
    uint64_t ldc;
    float* workspace;
    hipStream_t stream;
};
size_t grouped_product_workspace(const GroupProduct& a);
int launch_grouped_product(const GroupProduct& a);
// a, b: the forms along the groups' rows; c: [E, N, K]
size_t grouped_gradient_workspace(const GroupProduct& a);
int launch_grouped_gradient(const GroupProduct& a);

// A result in rows of `cols` numbers, ldc apart, from the sums of the pieces of its contraction, [pieces, sums]; offsets: the groups whose rows count, or null for all.
struct PieceSum {
    const float* partial;
    uint32_t pieces;
    uint64_t sums;
    const int32_t* offsets;
    uint32_t E, R, cols;
    void* c;
    uint64_t ldc;
};
int launch_piece_sum(const PieceSum& p, uint32_t dtype, hipStream_t stream);

struct VectorProduct {
    const void* x;
    uint32_t dtype, rows_dtype;     // of x; of y: the same or fp32
    uint64_t ld, T;
    const int32_t* order;           // nullable
    uint32_t per;
    const unsigned char* w;
    uint64_t w_stride;
    const int32_t* offsets;         // nullable: one group
    uint32_t E;
    uint64_t R, N, K;
    void* y;
    uint64_t ldy;
    float* workspace;
    hipStream_t stream;
};
size_t vector_product_workspace(const VectorProduct& a);
int launch_vector_product(const VectorProduct& a);

// n / d for n < 2^31 as the upper half of n * factor, shifted, d >= 2 (Granlund and Montgomery's division by a constant).
inline void divide_by(uint32_t d, uint32_t& factor, uint32_t& shift) {
    uint32_t log = 0;
    while ((1u << log) < d) ++log;
    factor = (uint32_t)((1ull << (31u + log)) / d + 1u);
    shift = log ? log - 1u : 0u;
}

inline uint64_t grouped_columns(uint64_t R, uint64_t E) { return (R + (kMx4Pad - 1) * (E < R ? E : R)) / kMx4Pad * kMx4Pad; }

}  // namespace qesgd
