// Host side of the C ABI for layers of experts: argument checks, all of them before the first HIP call of an entry point.
#include "qesgd_experts.h"

using namespace qesgd;

namespace {

constexpr uint64_t kMaxSide = 1ull << 20;

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p % a) == 0; }
bool dtype_ok(uint32_t t) { return t == QESGD_F32 || t == QESGD_BF16 || t == QESGD_F16; }
bool experts_ok(uint32_t E) { return E != 0 && E <= QESGD_MAX_EXPERTS; }
bool choices_ok(uint32_t E, uint32_t k) { return experts_ok(E) && k != 0 && k <= E && k <= QESGD_MAX_CHOICES; }
bool side_ok(uint64_t v) { return v != 0 && v <= kMaxSide; }
// The type of the experts' rows beside results of dtype; takes the mark off dtype.
uint32_t rows_type(uint32_t& dtype) {
    const bool wide = dtype & QESGD_ROWS_F32;
    dtype &= ~QESGD_ROWS_F32;
    return wide ? (uint32_t)QESGD_F32 : dtype;
}
// rows of `row` elements, ld apart
bool rows_ok(uint64_t rows, uint64_t row, uint64_t ld) { return rows < 2 || (ld >= row && ld < (1ull << 40) / rows); }
bool slab_ok(uint64_t E, uint64_t stride, uint64_t bytes) { return E < 2 || (stride >= bytes && stride % 256 == 0 && stride < (1ull << 48)); }

// The checks that forward and backward of the router share.
int route_check(uint32_t dtype, uint64_t ld, uint64_t T, uint32_t E, uint32_t k, uint32_t gate_kind) {
    if (!choices_ok(E, k)) return QESGD_ERR_EXPERTS;
    if (T == 0 || T > kMaxPairs / k || T > kMaxLogits / E) return QESGD_ERR_DIM;
    if (!dtype_ok(dtype)) return QESGD_ERR_DTYPE;
    if (gate_kind != QESGD_GATE_ALL && gate_kind != QESGD_GATE_CHOSEN) return QESGD_ERR_MODE;
    return rows_ok(T, E, ld) ? QESGD_OK : QESGD_ERR_STRIDE;
}

int combine_check(uint32_t dtype, uint64_t R, const int32_t* slots, uint64_t T, uint32_t k, uint64_t N) {
    constexpr uint64_t most = 1ull << 28;
    if (k == 0 || k > QESGD_MAX_CHOICES) return QESGD_ERR_EXPERTS;
    if (T == 0 || T > most || R == 0 || R > most || N == 0 || N > most || T * k >= (1ull << 31) || T > (1ull << 38) / N) return QESGD_ERR_DIM;
    if (!slots && T * k > R) return QESGD_ERR_DIM;
    return dtype_ok(dtype) ? QESGD_OK : QESGD_ERR_DTYPE;
}

int grouped_check(const GroupProduct& a) {
    if (!experts_ok(a.E)) return QESGD_ERR_EXPERTS;
    if (!side_ok(a.R) || !side_ok(a.N) || !side_ok(a.K)) return QESGD_ERR_DIM;
    if (!dtype_ok(a.dtype)) return QESGD_ERR_DTYPE;
    if (!aligned(a.a, 256) || !aligned(a.b, 256) || !aligned(a.offsets, 4) || !aligned(a.c, dtype_bytes(a.dtype)) || !aligned(a.workspace, 16))
        return QESGD_ERR_ALIGN;
    return QESGD_OK;
}

GroupProduct sizes(uint64_t R, uint64_t N, uint64_t K, uint32_t E) {
    GroupProduct a{};
    a.R = R;
    a.N = N;
    a.K = K;
    a.E = E;
    return a;
}
bool sizes_ok(uint64_t R, uint64_t N, uint64_t K, uint32_t E) { return experts_ok(E) && side_ok(R) && side_ok(N) && side_ok(K); }

}  // namespace

extern "C" {

size_t qesgd_route_workspace_bytes(uint64_t T, uint32_t E, uint32_t k) {
    if (!choices_ok(E, k) || T == 0 || T > kMaxPairs / k || T > kMaxLogits / E) return 0;
    return route_workspace(T, E, k);
}

int qesgd_route(const void* logits, uint32_t dtype, uint64_t ld, uint64_t T, uint32_t E, uint32_t k, uint32_t gate_kind,
                int32_t* experts, float* gates, int32_t* offsets, int32_t* order, int32_t* slots,
                void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !experts || !gates || !offsets || !order || !slots) return QESGD_ERR_NULL;
    if (const int rc = route_check(dtype, ld, T, E, k, gate_kind); rc != QESGD_OK) return rc;
    if (!aligned(logits, dtype_bytes(dtype)) || !aligned(experts, 4) || !aligned(gates, 4) || !aligned(offsets, 4) || !aligned(order, 4) ||
        !aligned(slots, 4) || !aligned(workspace, 16))
        return QESGD_ERR_ALIGN;
    const size_t need = route_workspace(T, E, k);
    if (need > 0 && (!workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    Route a{};
    a.logits = logits;
    a.dtype = dtype;
    a.ld = T > 1 ? ld : E;
    a.T = T;
    a.E = E;
    a.k = k;
    a.all = gate_kind == QESGD_GATE_ALL;
    a.experts = experts;
    a.gates = gates;
    a.offsets = offsets;
    a.order = order;
    a.slots = slots;
    a.workspace = (uint32_t*)workspace;
    a.stream = (hipStream_t)stream;
    return launch_route(a);
}

int qesgd_route_backward(const void* logits, uint32_t dtype, uint64_t ld, uint64_t T, uint32_t E, uint32_t k, uint32_t gate_kind,
                         const int32_t* experts, const float* gates, const float* dgates, void* dlogits, uint64_t ld_d, void* stream) {
    if (!experts || !gates || !dgates || !dlogits || (!logits && gate_kind != QESGD_GATE_CHOSEN)) return QESGD_ERR_NULL;
    if (const int rc = route_check(dtype, logits ? ld : ld_d, T, E, k, gate_kind); rc != QESGD_OK) return rc;
    if (!rows_ok(T, E, ld_d)) return QESGD_ERR_STRIDE;
    if (!aligned(logits, dtype_bytes(dtype)) || !aligned(dlogits, dtype_bytes(dtype)) || !aligned(experts, 4) || !aligned(gates, 4) || !aligned(dgates, 4))
        return QESGD_ERR_ALIGN;
    RouteBackward a{};
    a.logits = logits;
    a.dtype = dtype;
    a.ld = T > 1 ? ld : E;
    a.T = T;
    a.E = E;
    a.k = k;
    a.all = gate_kind == QESGD_GATE_ALL;
    a.experts = experts;
    a.gates = gates;
    a.dgates = dgates;
    a.dlogits = dlogits;
    a.ld_d = T > 1 ? ld_d : E;
    a.stream = (hipStream_t)stream;
    return launch_route_backward(a);
}

int qesgd_combine(const void* rows, uint32_t dtype, uint64_t ld, uint64_t R, const int32_t* slots, const float* gates, uint64_t T, uint32_t k,
                  uint64_t N, void* out, uint64_t ld_out, void* stream) {
    if (!rows || !out) return QESGD_ERR_NULL;
    const uint32_t rows_dtype = rows_type(dtype);
    if (const int rc = combine_check(dtype, R, slots, T, k, N); rc != QESGD_OK) return rc;
    if (!aligned(rows, dtype_bytes(rows_dtype)) || !aligned(out, dtype_bytes(dtype)) || !aligned(slots, 4) || !aligned(gates, 4)) return QESGD_ERR_ALIGN;
    if (!rows_ok(R, N, ld) || !rows_ok(T, N, ld_out)) return QESGD_ERR_STRIDE;
    Combine a{};
    a.rows = rows;
    a.dtype = dtype;
    a.rows_dtype = rows_dtype;
    a.ld = R > 1 ? ld : N;
    a.R = R;
    a.slots = slots;
    a.gates = gates;
    a.T = T;
    a.k = k;
    a.N = N;
    a.out = out;
    a.ld_out = T > 1 ? ld_out : N;
    a.stream = (hipStream_t)stream;
    return launch_combine(a);
}

int qesgd_combine_backward(const void* dy, uint32_t dtype, uint64_t ld_dy, const void* rows, uint64_t ld, uint64_t R, const int32_t* slots,
                           const float* gates, uint64_t T, uint32_t k, uint64_t N, void* drows, uint64_t ld_d, float* dgates, void* stream) {
    if (!dy || (!drows && !dgates) || (dgates && !rows) || (drows && !gates)) return QESGD_ERR_NULL;
    const uint32_t given = rows_type(dtype), rows_dtype = dgates ? given : dtype;      // without dgates nothing is read of the rows
    if (const int rc = combine_check(dtype, R, slots, T, k, N); rc != QESGD_OK) return rc;
    if (dgates && drows == rows && rows_dtype != dtype) return QESGD_ERR_DTYPE;
    if (!aligned(dy, dtype_bytes(dtype)) || !aligned(rows, dtype_bytes(rows_dtype)) || !aligned(drows, dtype_bytes(dtype)) || !aligned(slots, 4) ||
        !aligned(gates, 4) || !aligned(dgates, 4))
        return QESGD_ERR_ALIGN;
    if (!rows_ok(T, N, ld_dy) || (dgates && !rows_ok(R, N, ld)) || (drows && !rows_ok(R, N, ld_d))) return QESGD_ERR_STRIDE;
    Combine a{};
    a.rows = rows;
    a.dtype = dtype;
    a.rows_dtype = rows_dtype;
    a.ld = R > 1 ? ld : N;
    a.R = R;
    a.slots = slots;
    a.gates = gates;
    a.T = T;
    a.k = k;
    a.N = N;
    a.dy = dy;
    a.ld_dy = T > 1 ? ld_dy : N;
    a.drows = drows;
    a.ld_d = R > 1 ? ld_d : N;
    a.dgates = dgates;
    a.stream = (hipStream_t)stream;
    return launch_combine_backward(a);
}

uint64_t qesgd_mx4_grouped_columns(uint64_t R, uint32_t E) { return side_ok(R) && experts_ok(E) ? grouped_columns(R, E) : 0; }

int qesgd_mx4_quantize_groups(const void* x, uint32_t dtype, uint64_t ld, uint64_t T, const int32_t* order, uint32_t per, const int32_t* offsets,
                              uint32_t E, uint64_t R, uint64_t cols, uint32_t mode, uint64_t seed, uint32_t round, uint32_t worker,
                              void* packed, void* packed_t, void* stream) {
    if (!x || !offsets || (!packed && !packed_t)) return QESGD_ERR_NULL;
    if (!experts_ok(E)) return QESGD_ERR_EXPERTS;
    if (!side_ok(R) || !side_ok(T) || !side_ok(cols) || !side_ok(per)) return QESGD_ERR_DIM;
    qesgd_mx4_layout L, T_;
    int rc = make_mx4_layout(R, cols, &L);
    if (rc == QESGD_OK) rc = make_mx4_layout(cols, grouped_columns(R, E), &T_);
    if (rc != QESGD_OK) return rc;
    if (R * L.row_codes * 2 > kMx4MaxLaunch || (packed_t && cols * T_.row_codes * 2 > kMx4MaxLaunch)) return QESGD_ERR_DIM;
    if (!dtype_ok(dtype)) return QESGD_ERR_DTYPE;
    if (mode != QESGD_MX4_NEAREST && mode != QESGD_MX4_STOCHASTIC) return QESGD_ERR_MODE;
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(order, 4) || !aligned(offsets, 4) || !aligned(packed, 256) || !aligned(packed_t, 256))
        return QESGD_ERR_ALIGN;
    if (!rows_ok(T, cols, ld)) return QESGD_ERR_STRIDE;
    GroupQuantize a{};
    a.x = x;
    a.dtype = dtype;
    a.ld = T > 1 ? ld : cols;
    a.T = T;
    a.order = order;
    a.per = order ? per : 1;        // row r of x, not one of its pairs
    a.offsets = offsets;
    a.E = E;
    a.R = R;
    a.cols = cols;
    a.stochastic = mode == QESGD_MX4_STOCHASTIC;
    a.seed = seed;
    a.round = round;
    a.worker = worker;
    a.packed = (unsigned char*)packed;
    a.packed_t = (unsigned char*)packed_t;
    a.stream = (hipStream_t)stream;
    return launch_quantize_groups(a);
}

size_t qesgd_mx4_grouped_product_workspace_bytes(uint64_t R, uint64_t N, uint64_t K, uint32_t E) {
    return sizes_ok(R, N, K, E) ? grouped_product_workspace(sizes(R, N, K, E)) : 0;
}

int qesgd_mx4_grouped_product(const void* a_packed, const void* b_slab, uint64_t b_stride, const int32_t* offsets, uint32_t E, uint64_t R,
                              uint64_t N, uint64_t K, void* c, uint32_t dtype, uint64_t ldc, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a_packed || !b_slab || !offsets || !c) return QESGD_ERR_NULL;
    GroupProduct a = sizes(R, N, K, E);
    a.a = (const unsigned char*)a_packed;
    a.b = (const unsigned char*)b_slab;
    a.b_stride = b_stride;
    a.offsets = offsets;
    a.c = c;
    a.dtype = dtype;
    a.ldc = R > 1 ? ldc : N;
    a.workspace = (float*)workspace;
    a.stream = (hipStream_t)stream;
    if (const int rc = grouped_check(a); rc != QESGD_OK) return rc;
    qesgd_mx4_layout B;
    if (const int rc = make_mx4_layout(N, K, &B); rc != QESGD_OK) return rc;
    if (!rows_ok(R, N, ldc) || !slab_ok(E, b_stride, B.bytes)) return QESGD_ERR_STRIDE;
    const size_t need = grouped_product_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    return launch_grouped_product(a);
}

size_t qesgd_mx4_grouped_gradient_workspace_bytes(uint64_t R, uint64_t N, uint64_t K, uint32_t E) {
    return sizes_ok(R, N, K, E) ? grouped_gradient_workspace(sizes(R, N, K, E)) : 0;
}

int qesgd_mx4_grouped_gradient(const void* a_packed_t, const void* b_packed_t, const int32_t* offsets, uint32_t E, uint64_t R, uint64_t N,
                               uint64_t K, void* d, uint32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!a_packed_t || !b_packed_t || !offsets || !d) return QESGD_ERR_NULL;
    GroupProduct a = sizes(R, N, K, E);
    a.a = (const unsigned char*)a_packed_t;
    a.b = (const unsigned char*)b_packed_t;
    a.offsets = offsets;
    a.c = d;
    a.dtype = dtype;
    a.ldc = K;
    a.workspace = (float*)workspace;
    a.stream = (hipStream_t)stream;
    if (const int rc = grouped_check(a); rc != QESGD_OK) return rc;
    const size_t need = grouped_gradient_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    return launch_grouped_gradient(a);
}

static bool vector_sizes_ok(uint64_t R, uint64_t N, uint64_t K, uint32_t E) { return sizes_ok(R, N, K, E); }

size_t qesgd_mx4_vector_product_workspace_bytes(uint64_t R, uint64_t N, uint64_t K, uint32_t E) {
    if (!vector_sizes_ok(R, N, K, E)) return 0;
    VectorProduct a{};
    a.R = R;
    a.N = N;
    a.K = K;
    a.E = E;
    return vector_product_workspace(a);
}

int qesgd_mx4_vector_product(const void* x, uint32_t dtype, uint64_t ld, uint64_t T, const int32_t* order, uint32_t per, const void* w_slab,
                             uint64_t w_stride, const int32_t* offsets, uint32_t E, uint64_t R, uint64_t N, uint64_t K, void* y, uint64_t ldy,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !w_slab || !y || (!offsets && E > 1)) return QESGD_ERR_NULL;
    if (!experts_ok(E)) return QESGD_ERR_EXPERTS;
    if (!vector_sizes_ok(R, N, K, E) || !side_ok(T) || !side_ok(per)) return QESGD_ERR_DIM;
    const uint32_t rows_dtype = rows_type(dtype);
    if (!dtype_ok(dtype)) return QESGD_ERR_DTYPE;
    if (!aligned(x, dtype_bytes(dtype)) || !aligned(y, dtype_bytes(rows_dtype)) || !aligned(order, 4) || !aligned(offsets, 4) || !aligned(w_slab, 256) ||
        !aligned(workspace, 16))
        return QESGD_ERR_ALIGN;
    qesgd_mx4_layout W;
    if (const int rc = make_mx4_layout(N, K, &W); rc != QESGD_OK) return rc;
    if (!rows_ok(T, K, ld) || !rows_ok(R, N, ldy) || !slab_ok(E, w_stride, W.bytes)) return QESGD_ERR_STRIDE;
    VectorProduct a{};
    a.x = x;
    a.dtype = dtype;
    a.rows_dtype = rows_dtype;
    a.ld = T > 1 ? ld : K;
    a.T = T;
    a.order = order;
    a.per = order ? per : 1;        // row r of x, not one of its pairs
    a.w = (const unsigned char*)w_slab;
    a.w_stride = w_stride;
    a.offsets = offsets;
    a.E = E;
    a.R = R;
    a.N = N;
    a.K = K;
    a.y = y;
    a.ldy = R > 1 ? ldy : N;
    a.workspace = (float*)workspace;
    a.stream = (hipStream_t)stream;
    const size_t need = vector_product_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return QESGD_ERR_WORKSPACE;
    return launch_vector_product(a);
}

}  // extern "C"
