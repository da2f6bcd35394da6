"""The host side of the operators for matrix parameters under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, g++): layouts,
sizes and checks at the ends of their ranges, the launchers replaced by stubs."""
import os

import pytest

from test_sanitizers import ROOT, _build_and_run

DRIVER = r"""
#include "qesgd_matrix.h"
namespace qesgd {
static int launches = 0;
static Mx4Quantize q; static Mx4Aggregate g; static Mx4Product p; static Orthogonalize o;
int launch_mx4_quantize(const Mx4Quantize& a) { q = a; ++launches; return QESGD_OK; }
int launch_mx4_aggregate(const Mx4Aggregate& a) { g = a; ++launches; return QESGD_OK; }
size_t mx4_product_plan(Mx4Product& a) { a.edge = 64; a.pieces = a.K > 4096 ? 4 : 1; return a.pieces > 1 ? a.pieces * a.M * a.N * 4 : 0; }
int launch_mx4_product(const Mx4Product& a) { p = a; ++launches; return QESGD_OK; }
size_t orthogonalize_workspace(uint64_t rows, uint64_t cols, uint32_t n) { return rows * cols < 4096 ? 0 : rows * cols * n; }
int launch_orthogonalize(const Orthogonalize& a) { o = a; ++launches; return QESGD_OK; }
}
#include <cstdio>
#include <memory>
int main() {
    using namespace qesgd;
    const uint64_t sides[] = {0, 1, 31, 127, 128, 129, 4097, 1ull << 20, (1ull << 20) + 1, (1ull << 31) - 1, 1ull << 31, (1ull << 32) + 5,
                              (1ull << 38) - 1, 1ull << 38, (1ull << 40) - 1, 1ull << 40, ~0ull};
    const uint64_t strides[] = {0, 1, 128, 4096, 1ull << 20, (1ull << 40) - 256, 1ull << 41, ~0ull - 255, ~0ull};
    void* x = (void*)0x10000; void* pk = (void*)0x20000; void* pt = (void*)0x30000; float* z = (float*)0x40000;
    float co[3 * QESGD_MAX_STEPS] = {};
    unsigned long long taken = 0, refused = 0;
    auto count = [&](int rc, int before) {
        if (rc == QESGD_OK) ++taken; else ++refused;
        return launches - before == (rc == QESGD_OK ? 1 : 0);           // what is refused launches nothing
    };
    for (uint64_t r : sides) for (uint64_t c : sides) {
        qesgd_mx4_layout L;
        if (qesgd_mx4_layout_query(r, c, &L) == QESGD_OK) {
            if (L.bytes % 256 || L.scales_off % 256 || L.bytes < L.payload_bytes || L.payload_bytes != r * (L.row_codes + L.row_scales)) return 2;
            if (L.row_codes * 2 < c || L.row_codes * 2 >= c + 128 || L.row_scales * 16 != L.row_codes) return 3;
        }
        for (uint64_t ld : strides) for (uint32_t K : {0u, 1u, 2u, 64u, 65u}) for (uint64_t ps : strides) for (int form = 0; form < 4; ++form) {
            int before = launches;
            const int rc = qesgd_mx4_quantize_pack(x, K % 3, ld, ps, r, c, K, K & 1, 1, 2, 3, form & 1 ? pk : nullptr, ps, form & 2 ? pt : nullptr, ps, nullptr);
            if (!count(rc, before)) return 4;
            if (rc == QESGD_OK && ((r > 1 && q.ld < c) || (K > 1 && q.x_stride < (r - 1) * q.ld + c))) return 5;
        }
        for (uint64_t ps : strides) for (uint32_t K : {0u, 1u, 2u, 64u, 65u}) {
            int before = launches;
            if (!count(qesgd_mx4_unpack_aggregate_update(pk, ps, K, r, c, z, z, z, nullptr, nullptr), before)) return 6;
        }
        for (uint64_t k : sides) for (uint64_t ldc : strides) {
            int before = launches;
            const size_t need = qesgd_mx4_product_workspace_bytes(r, c, k);
            if (!count(qesgd_mx4_product(pk, pt, r, c, k, z, QESGD_BF16, ldc, x, need, nullptr), before)) return 7;
            before = launches;
            if (need > 0 && qesgd_mx4_product(pk, pt, r, c, k, z, QESGD_BF16, ldc, x, need - 1, nullptr) == QESGD_OK) return 8;
            if (need > 0 && qesgd_mx4_product(pk, pt, r, c, k, z, QESGD_BF16, ldc, nullptr, need, nullptr) == QESGD_OK) return 9;
            if (launches != before) return 10;
        }
        for (uint32_t n : {0u, 1u, 5u, 65535u, 65536u, ~0u}) for (uint32_t steps : {0u, 1u, QESGD_MAX_STEPS, QESGD_MAX_STEPS + 1, ~0u}) {
            // as many coefficients as the call reads, to the byte
            const uint32_t room = steps && steps <= QESGD_MAX_STEPS ? 3 * steps : 1;
            auto own = std::unique_ptr<float[]>(new float[room]());
            int before = launches;
            const size_t need = qesgd_orthogonalize_workspace_bytes(r, c, n);
            if (!count(qesgd_orthogonalize(x, QESGD_F16, r, c, n, own.get(), steps, 0.0f, z, pk, need, nullptr), before)) return 11;
            before = launches;
            if (!count(qesgd_orthogonal_update(z, r, c, n, z, 0.9f, 7, own.get(), steps, 1e-7f, -1.0f, z, z, z, z, z, pk, need, nullptr), before)) return 12;
        }
    }
    int before = launches;
    if (qesgd_mx4_quantize_pack(x, 0, 128, 0, 8, 128, 1, 2, 0, 0, 0, pk, 0, nullptr, 0, nullptr) != QESGD_ERR_MODE) return 13;
    if (qesgd_mx4_quantize_pack((char*)x + 2, 0, 128, 0, 8, 128, 1, 0, 0, 0, 0, pk, 0, nullptr, 0, nullptr) != QESGD_ERR_ALIGN) return 14;
    if (qesgd_orthogonalize(x, 9, 8, 8, 1, co, 1, 0.0f, z, nullptr, 0, nullptr) != QESGD_ERR_DTYPE) return 15;
    if (qesgd_orthogonalize(x, 0, 8, 8, 1, co, 1, -1.0f, z, nullptr, 0, nullptr) != QESGD_ERR_COEFF) return 16;
    if (launches != before) return 17;
    std::printf("matrix sanitizer calls: %llu taken, %llu refused\n", taken, refused);
    return taken && refused ? 0 : 18;
}
"""


def test_host_side_under_address_and_ub_sanitizers(tmp_path):
    if not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("HIP headers not available")
    csrc = os.path.join(ROOT, "paper_1901_03040_amd", "csrc")
    out = _build_and_run(tmp_path, "matrix_san", DRIVER,
                         ["-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{os.path.join(ROOT, 'include')}", f"-I{csrc}",
                          "-Wno-deprecated-declarations", os.path.join(csrc, "qesgd_matrix_api.cpp")])
    assert "matrix sanitizer calls" in out
