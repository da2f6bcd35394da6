"""The host side of the operators for layers of experts under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, g++): checks at the
ends of their ranges, the launchers replaced by stubs that look at what they are given."""
import os

import pytest

from test_sanitizers import ROOT, _build_and_run

DRIVER = r"""
#include "qesgd_experts.h"
namespace qesgd {
static int launches = 0;
static bool wrong = false;
int make_mx4_layout(uint64_t rows, uint64_t cols, qesgd_mx4_layout* out) {
    if (rows == 0 || cols == 0 || rows >= (1ull << 40) || cols >= (1ull << 38)) return QESGD_ERR_DIM;
    const uint64_t wide = round_up_to(cols, kMx4Pad);
    if (wide > kMx4MaxSlots / rows) return QESGD_ERR_DIM;
    qesgd_mx4_layout L{};
    L.row_codes = wide / 2;
    L.row_scales = wide / 32;
    L.scales_off = round_up_to(rows * L.row_codes, 256);
    L.bytes = L.scales_off + round_up_to(rows * L.row_scales, 256);
    *out = L;
    return QESGD_OK;
}
size_t route_workspace(uint64_t T, uint32_t E, uint32_t k) { return T * k > 1000 ? (size_t)E * 64 : 0; }
int launch_route(const Route& a) { ++launches; wrong |= a.k > a.E || a.T * a.k > kMaxPairs || a.ld < a.E; return QESGD_OK; }
int launch_route_backward(const RouteBackward& a) { ++launches; wrong |= a.T * a.E > kMaxLogits || a.ld_d < a.E; return QESGD_OK; }
int launch_combine(const Combine& a) { ++launches; wrong |= a.ld < a.N || a.ld_out < a.N || (!a.slots && a.T * a.k > a.R); return QESGD_OK; }
int launch_combine_backward(const Combine& a) { ++launches; wrong |= a.ld_dy < a.N; return QESGD_OK; }
int launch_quantize_groups(const GroupQuantize& a) { ++launches; wrong |= a.ld < a.cols || a.R * a.cols > kMx4MaxLaunch; return QESGD_OK; }
size_t grouped_product_workspace(const GroupProduct& a) { return a.K > 4096 ? a.R * a.N * 8 : 0; }
size_t grouped_gradient_workspace(const GroupProduct& a) { return a.R > 4096 ? a.E * 16 : 0; }
int launch_grouped_product(const GroupProduct& a) { ++launches; wrong |= a.ldc < a.N; return QESGD_OK; }
int launch_grouped_gradient(const GroupProduct&) { ++launches; return QESGD_OK; }
size_t vector_product_workspace(const VectorProduct& a) { return a.K > 4096 ? a.R * a.N * 4 : 0; }
int launch_vector_product(const VectorProduct& a) { ++launches; wrong |= a.ldy < a.N || a.ld < a.K || (!a.offsets && a.E > 1); return QESGD_OK; }
}
#include <cstdio>
int main() {
    using namespace qesgd;
    const uint64_t sides[] = {0, 1, 127, 129, 4097, 1ull << 20, (1ull << 20) + 1, 1ull << 28, (1ull << 31) - 1, (1ull << 32) + 5, 1ull << 40, ~0ull};
    const uint64_t strides[] = {0, 1, 4096, 1ull << 20, 1ull << 39, 1ull << 48, ~0ull - 255, ~0ull};
    const uint32_t counts[] = {0, 1, 2, 16, 17, 1024, 1025, ~0u};
    void* x = (void*)0x10000; void* p = (void*)0x20000; float* f = (float*)0x30000; int32_t* i = (int32_t*)0x40000;
    unsigned long long taken = 0, refused = 0;
    auto count = [&](int rc, int before) {
        if (rc == QESGD_OK) ++taken; else ++refused;
        return launches - before == (rc == QESGD_OK ? 1 : 0);
    };
    for (uint64_t a : sides) for (uint64_t s : strides) for (uint32_t E : counts) for (uint32_t k : counts) {
        int b = launches;
        size_t need = qesgd_route_workspace_bytes(a, E, k);
        if (!count(qesgd_route(x, QESGD_F16, s, a, E, k, k & 1, i, f, i, i, i, p, need, nullptr), b)) return 2;
        b = launches;
        if (!count(qesgd_route_backward(x, QESGD_F32, s, a, E, k, 0, i, f, f, f, s, nullptr), b)) return 3;
        b = launches;
        if (!count(qesgd_combine(x, QESGD_BF16, s, a, E & 1 ? i : nullptr, nullptr, a, k, E, x, s, nullptr), b)) return 4;
        b = launches;
        if (!count(qesgd_combine_backward(x, QESGD_F32, s, x, s, a, i, f, E, k, a, x, s, f, nullptr), b)) return 5;
    }
    for (uint64_t r : sides) for (uint64_t n : sides) for (uint64_t k : sides) for (uint64_t s : strides) for (uint32_t E : counts) {
        const uint64_t columns = qesgd_mx4_grouped_columns(r, E);
        if (columns && (columns % 128 || columns < r || columns >= r + 127ull * E + 128)) return 6;
        int b = launches;
        if (!count(qesgd_mx4_quantize_groups(x, QESGD_F32, s, n, nullptr, (uint32_t)k, i, E, r, k, 1, 1, 2, 3, p, p, nullptr), b)) return 7;
        b = launches;
        size_t need = qesgd_mx4_grouped_product_workspace_bytes(r, n, k, E);
        if (!count(qesgd_mx4_grouped_product(p, p, s, i, E, r, n, k, f, QESGD_BF16, s, x, need, nullptr), b)) return 8;
        if (need > 0 && qesgd_mx4_grouped_product(p, p, s, i, E, r, n, k, f, QESGD_BF16, s, x, need - 1, nullptr) == QESGD_OK) return 9;
        b = launches;
        need = qesgd_mx4_grouped_gradient_workspace_bytes(r, n, k, E);
        if (!count(qesgd_mx4_grouped_gradient(p, p, i, E, r, n, k, f, QESGD_F32, x, need, nullptr), b)) return 10;
        b = launches;
        need = qesgd_mx4_vector_product_workspace_bytes(r, n, k, E);
        if (!count(qesgd_mx4_vector_product(x, QESGD_F32, s, n, i, 1, p, s, E > 1 ? i : nullptr, E, r, n, k, f, s, x, need, nullptr), b)) return 11;
        if (need > 0 && qesgd_mx4_vector_product(x, QESGD_F32, s, n, i, 1, p, s, i, E, r, n, k, f, s, nullptr, need, nullptr) == QESGD_OK) return 12;
    }
    std::printf("expert sanitizer calls: %llu taken, %llu refused\n", taken, refused);
    return taken && refused && !wrong ? 0 : 18;
}
"""


def test_host_side_under_address_and_ub_sanitizers(tmp_path):
    if not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("HIP headers not available")
    csrc = os.path.join(ROOT, "paper_1901_03040_amd", "csrc")
    out = _build_and_run(tmp_path, "expert_san", DRIVER,
                         ["-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{os.path.join(ROOT, 'include')}", f"-I{csrc}",
                          "-Wno-deprecated-declarations", os.path.join(csrc, "qesgd_experts_api.cpp")])
    assert "expert sanitizer calls" in out
