// Internal declarations of the operators for matrix parameters: 4-bit microscaled codes, their mean and
// product, and the orthogonalised update (not installed).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qesgd.h"

namespace qesgd {

inline uint64_t round_up_to(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }
inline uint32_t dtype_bytes(uint32_t dtype) { return dtype == QESGD_F32 ? 4u : 2u; }

// ---- microscaled 4-bit codes ------------------------------------------------

constexpr uint64_t kMx4Block = 32;                       // coordinates that share a scale
constexpr uint64_t kMx4Pad = 128;                        // columns are padded to a multiple of this
constexpr uint64_t kMx4MaxSlots = 1ull << 38;            // padded coordinates of one matrix: 128 of them are numbered in 32 bits
constexpr uint64_t kMx4MaxLaunch = 1ull << 34;           // of a call that launches eight or more of them a thread: half of what follows

// A launch numbers its threads in 32 bits.
inline bool grid_ok(uint64_t groups, uint64_t threads) { return groups < (1ull << 31) && groups * threads < (1ull << 32); }

struct Mx4Quantize {
    const void* x;
    uint32_t dtype;
    uint64_t ld, x_stride;          // elements between rows, between workers
    uint64_t rows, cols;
    uint32_t K;
    bool stochastic;
    uint64_t seed;
    uint32_t round, worker0;
    unsigned char* packed;          // nullable
    uint64_t packed_stride;
    unsigned char* packed_t;        // nullable: the form of the transposed matrix
    uint64_t packed_t_stride;
    hipStream_t stream;
};

struct Mx4Aggregate {
    const unsigned char* packed;
    uint64_t packed_stride;
    uint32_t K;
    uint64_t rows, cols;
    const float* w;
    float* zbar;
    float* u;
    float* zsum;
    hipStream_t stream;
};

struct Mx4Product {
    const unsigned char* a;
    const unsigned char* b;
    uint64_t M, N, K;
    void* c;
    uint32_t dtype;
    uint64_t ldc;
    float* workspace;
    hipStream_t stream;
    uint32_t edge, pieces;          // of mx4_product_plan
};

int make_mx4_layout(uint64_t rows, uint64_t cols, qesgd_mx4_layout* out);
int launch_mx4_quantize(const Mx4Quantize& a);
int launch_mx4_aggregate(const Mx4Aggregate& a);
// Chooses the kernel for (M, N, K); the bytes of workspace that it needs.
size_t mx4_product_plan(Mx4Product& a);
int launch_mx4_product(const Mx4Product& a);

// ---- orthogonalised update ----------------------------------------------------

struct Orthogonalize {
    const void* x;                  // [n, rows, cols]
    uint32_t dtype;                 // of x and out
    uint64_t rows, cols;
    uint32_t n;
    float* momentum;                // nullable, f32
    float mu;
    bool nesterov;
    const float* coeffs;            // host, 3 * steps
    uint32_t steps;
    float eps, alpha;
    void* out;                      // nullable where z is given
    float* z;                       // nullable; the rest is f32 and goes with it
    const float* w;
    float* u;
    float* zsum;
    unsigned char* workspace;
    hipStream_t stream;
};

size_t orthogonalize_workspace(uint64_t rows, uint64_t cols, uint32_t n);
int launch_orthogonalize(const Orthogonalize& a);

}  // namespace qesgd
