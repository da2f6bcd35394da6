// Host side of the C ABI for matrix parameters: shape arithmetic and argument checks, all of them before the
// first HIP call of an entry point.
#include <cmath>

#include "qesgd_matrix.h"

namespace qesgd {

static bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }

int make_mx4_layout(uint64_t rows, uint64_t cols, qesgd_mx4_layout* out) {
    if (rows == 0 || cols == 0 || rows >= (1ull << 40) || cols >= (1ull << 38)) return QESGD_ERR_DIM;
    const uint64_t wide = round_up_to(cols, kMx4Pad);
    if (wide > kMx4MaxSlots / rows) return QESGD_ERR_DIM;
    qesgd_mx4_layout L{};
    L.rows = rows;
    L.cols = cols;
    L.row_codes = wide / 2;
    L.row_scales = wide / kMx4Block;
    L.codes_off = 0;
    L.scales_off = round_up_to(rows * L.row_codes, 256);
    L.bytes = L.scales_off + round_up_to(rows * L.row_scales, 256);
    L.payload_bytes = rows * (L.row_codes + L.row_scales);
    *out = L;
    return QESGD_OK;
}

static bool dtype_ok(uint32_t t) { return t == QESGD_F32 || t == QESGD_BF16 || t == QESGD_F16; }

// d elements, n_matrices of them rows x cols each, as a count that 64-bit offsets in bytes can carry.
static bool count_ok(uint64_t rows, uint64_t cols, uint64_t n) {
    return rows != 0 && cols != 0 && n != 0 && rows < (1ull << 40) && cols < (1ull << 40) / rows + 1 &&
           rows * cols < (1ull << 40) / n + 1 && rows * cols * n < (1ull << 40);
}

// Sides of a matrix that the iteration and the product take: row numbers, and byte offsets inside a tile's rows, stay within 32 bits.
constexpr uint64_t kMaxSide = 1ull << 20;

static int orthogonal_check(const Orthogonalize& a, size_t workspace_bytes) {
    if (!a.x || !a.coeffs) return QESGD_ERR_NULL;
    if (!count_ok(a.rows, a.cols, a.n) || a.rows > kMaxSide || a.cols > kMaxSide || a.n > 65535u) return QESGD_ERR_DIM;
    if (!dtype_ok(a.dtype)) return QESGD_ERR_DTYPE;
    if (a.steps == 0 || a.steps > QESGD_MAX_STEPS) return QESGD_ERR_STEPS;
    for (uint32_t i = 0; i < 3 * a.steps; ++i)
        if (!std::isfinite(a.coeffs[i])) return QESGD_ERR_COEFF;
    if (!(a.eps >= 0.0f) || !std::isfinite(a.eps) || !std::isfinite(a.alpha) || !std::isfinite(a.mu)) return QESGD_ERR_COEFF;
    if (!aligned(a.x, 16) || !aligned(a.momentum, 16) || !aligned(a.out, 16) || !aligned(a.z, 16) || !aligned(a.w, 16) ||
        !aligned(a.u, 16) || !aligned(a.zsum, 16) || !aligned(a.workspace, 256))
        return QESGD_ERR_ALIGN;
    const size_t need = orthogonalize_workspace(a.rows, a.cols, a.n);
    if (need > 0 && (!a.workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    return QESGD_OK;
}

}  // namespace qesgd

using namespace qesgd;

extern "C" {

int qesgd_mx4_layout_query(uint64_t rows, uint64_t cols, qesgd_mx4_layout* out) {
    if (!out) return QESGD_ERR_NULL;
    return make_mx4_layout(rows, cols, out);
}

int qesgd_mx4_quantize_pack(const void* x, uint32_t dtype, uint64_t ld, uint64_t x_stride, uint64_t rows, uint64_t cols,
                            uint32_t K, uint32_t mode, uint64_t seed, uint32_t round, uint32_t worker,
                            void* packed, uint64_t packed_stride, void* packed_t, uint64_t packed_t_stride, void* stream) {
    if (!x || (!packed && !packed_t)) return QESGD_ERR_NULL;
    qesgd_mx4_layout L, T;
    int rc = make_mx4_layout(rows, cols, &L);
    if (rc == QESGD_OK && packed_t) rc = make_mx4_layout(cols, rows, &T);
    if (rc != QESGD_OK) return rc;
    if (rows * L.row_codes * 2 > kMx4MaxLaunch || (packed_t && cols * T.row_codes * 2 > kMx4MaxLaunch)) return QESGD_ERR_DIM;
    if (!dtype_ok(dtype)) return QESGD_ERR_DTYPE;
    if (K == 0 || K > QESGD_MAX_WORKERS) return QESGD_ERR_WORKERS;
    if (mode != QESGD_MX4_NEAREST && mode != QESGD_MX4_STOCHASTIC) return QESGD_ERR_MODE;
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(packed, 256) || !aligned(packed_t, 256)) return QESGD_ERR_ALIGN;
    if (rows > 1 && (ld < cols || ld >= (1ull << 40) / rows)) return QESGD_ERR_STRIDE;
    if (K > 1) {
        const uint64_t span = rows > 1 ? (rows - 1) * ld + cols : cols;
        if (x_stride < span || x_stride >= (1ull << 41)) return QESGD_ERR_STRIDE;
        if (packed && (packed_stride < L.bytes || packed_stride % 256 != 0)) return QESGD_ERR_STRIDE;
        if (packed_t && (packed_t_stride < T.bytes || packed_t_stride % 256 != 0)) return QESGD_ERR_STRIDE;
    }
    Mx4Quantize a{};
    a.x = x;
    a.dtype = dtype;
    a.ld = rows > 1 ? ld : cols;
    a.x_stride = x_stride;
    a.rows = rows;
    a.cols = cols;
    a.K = K;
    a.stochastic = mode == QESGD_MX4_STOCHASTIC;
    a.seed = seed;
    a.round = round;
    a.worker0 = worker;
    a.packed = (unsigned char*)packed;
    a.packed_stride = packed_stride;
    a.packed_t = (unsigned char*)packed_t;
    a.packed_t_stride = packed_t_stride;
    a.stream = (hipStream_t)stream;
    return launch_mx4_quantize(a);
}

int qesgd_mx4_unpack_aggregate_update(const void* packed_slab, uint64_t packed_stride, uint32_t K, uint64_t rows, uint64_t cols,
                                      const float* w_snap, float* zbar_out, float* u_out, float* zsum_inout, void* stream) {
    if (!packed_slab || (!zbar_out && !u_out && !zsum_inout)) return QESGD_ERR_NULL;
    if ((u_out != nullptr) != (w_snap != nullptr)) return QESGD_ERR_NULL;
    qesgd_mx4_layout L;
    const int rc = make_mx4_layout(rows, cols, &L);
    if (rc != QESGD_OK) return rc;
    if (rows * L.row_codes * 2 > kMx4MaxLaunch) return QESGD_ERR_DIM;
    if (K == 0 || K > QESGD_MAX_WORKERS) return QESGD_ERR_WORKERS;
    if (!aligned(packed_slab, 256) || !aligned(w_snap, 16) || !aligned(zbar_out, 16) || !aligned(u_out, 16) || !aligned(zsum_inout, 16))
        return QESGD_ERR_ALIGN;
    if (K > 1 && (packed_stride < L.bytes || packed_stride % 256 != 0)) return QESGD_ERR_STRIDE;
    Mx4Aggregate a{};
    a.packed = (const unsigned char*)packed_slab;
    a.packed_stride = packed_stride;
    a.K = K;
    a.rows = rows;
    a.cols = cols;
    a.w = w_snap;
    a.zbar = zbar_out;
    a.u = u_out;
    a.zsum = zsum_inout;
    a.stream = (hipStream_t)stream;
    return launch_mx4_aggregate(a);
}

static bool product_dims_ok(uint64_t M, uint64_t N, uint64_t K) {
    return M != 0 && N != 0 && K != 0 && M <= kMaxSide && N <= kMaxSide && K <= kMaxSide;
}

size_t qesgd_mx4_product_workspace_bytes(uint64_t M, uint64_t N, uint64_t K) {
    if (!product_dims_ok(M, N, K)) return 0;
    Mx4Product p{};
    p.M = M;
    p.N = N;
    p.K = K;
    return mx4_product_plan(p);
}

int qesgd_mx4_product(const void* a_packed, const void* b_packed, uint64_t M, uint64_t N, uint64_t K, void* c, uint32_t dtype,
                      uint64_t ldc, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a_packed || !b_packed || !c) return QESGD_ERR_NULL;
    if (!product_dims_ok(M, N, K)) return QESGD_ERR_DIM;
    if (!dtype_ok(dtype)) return QESGD_ERR_DTYPE;
    if (!aligned(a_packed, 256) || !aligned(b_packed, 256) || !aligned(c, 16) || !aligned(workspace, 16)) return QESGD_ERR_ALIGN;
    if (M > 1 && (ldc < N || ldc >= (1ull << 40) / M)) return QESGD_ERR_STRIDE;
    Mx4Product p{};
    p.M = M;
    p.N = N;
    p.K = K;
    const size_t need = mx4_product_plan(p);
    if (need > 0 && (!workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    p.a = (const unsigned char*)a_packed;
    p.b = (const unsigned char*)b_packed;
    p.c = c;
    p.dtype = dtype;
    p.ldc = M > 1 ? ldc : N;
    p.workspace = (float*)workspace;
    p.stream = (hipStream_t)stream;
    return launch_mx4_product(p);
}

size_t qesgd_orthogonalize_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t n) {
    if (!count_ok(rows, cols, n) || rows > kMaxSide || cols > kMaxSide || n > 65535u) return 0;
    return orthogonalize_workspace(rows, cols, n);
}

int qesgd_orthogonalize(const void* x, uint32_t dtype, uint64_t rows, uint64_t cols, uint32_t n, const float* coeffs, uint32_t steps,
                        float eps, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!out) return QESGD_ERR_NULL;
    Orthogonalize a{};
    a.x = x;
    a.dtype = dtype;
    a.rows = rows;
    a.cols = cols;
    a.n = n;
    a.coeffs = coeffs;
    a.steps = steps;
    a.eps = eps;
    a.alpha = 1.0f;
    a.out = out;
    a.workspace = (unsigned char*)workspace;
    a.stream = (hipStream_t)stream;
    const int rc = orthogonal_check(a, workspace_bytes);
    return rc != QESGD_OK ? rc : launch_orthogonalize(a);
}

int qesgd_orthogonal_update(const float* g, uint64_t rows, uint64_t cols, uint32_t n, float* momentum_inout, float mu, uint32_t nesterov,
                            const float* coeffs, uint32_t steps, float eps, float alpha, float* step_out, float* z_inout,
                            const float* w_snap, float* u_out, float* zsum_inout, void* workspace, size_t workspace_bytes,
                            void* stream) {
    if (!step_out && !z_inout) return QESGD_ERR_NULL;
    if ((u_out != nullptr) != (w_snap != nullptr) || (!z_inout && (u_out || zsum_inout))) return QESGD_ERR_NULL;
    Orthogonalize a{};
    a.x = g;
    a.dtype = QESGD_F32;
    a.rows = rows;
    a.cols = cols;
    a.n = n;
    a.momentum = momentum_inout;
    a.mu = mu;
    a.nesterov = nesterov != 0;
    a.coeffs = coeffs;
    a.steps = steps;
    a.eps = eps;
    a.alpha = alpha;
    a.out = step_out;
    a.z = z_inout;
    a.w = w_snap;
    a.u = u_out;
    a.zsum = zsum_inout;
    a.workspace = (unsigned char*)workspace;
    a.stream = (hipStream_t)stream;
    const int rc = orthogonal_check(a, workspace_bytes);
    return rc != QESGD_OK ? rc : launch_orthogonalize(a);
}

}  // extern "C"
