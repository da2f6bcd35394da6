"""4-bit microscaled codes, no GPU: the reference's own values, the packed layout, and what the entry points refuse."""
import numpy as np
import pytest

import matrix_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    binding.lib()
    return binding


def test_reference_known_blocks():
    x = np.zeros((1, 32))
    x[0, :9] = [6, -6, 0.25, 0.75, 1.25, 2.5, 5, 3.5, -0.0]
    code, scale = R.quantize(x)
    assert scale[0, 0] == 127                                       # floor(log2 6) - 2 = 0
    assert code[0, :9].tolist() == [7, 15, 0, 2, 2, 4, 6, 6, 8]     # ties to the even code
    x[0, 0] = 7.0                                                   # nearest cuts off at 6, stochastic takes the next scale
    assert R.quantize(x)[1][0, 0] == 127 and R.quantize(x)[0][0, 0] == 7
    assert R.quantize(x, True)[1][0, 0] == 128
    x[0, 3] = np.inf
    code, scale = R.quantize(x)
    assert scale[0, 0] == 255 and not code.any() and np.isnan(R.values(code, scale, 32)).all()
    assert R.quantize(np.full((1, 5), 2.0 ** -140))[1][0, 0] == 0   # held at e = -127


def test_reference_stochastic_is_unbiased():
    rng = np.random.default_rng(1)
    x = np.repeat(rng.standard_normal((1, 128)), 4000, 0)
    q = R.values(*R.quantize(x, True, 5, 2, 1), 128)
    step = np.ldexp(2.0, R.quantize(x[:1], True)[1].astype(int) - 127).repeat(32, 1)    # widest gap of the grid
    # a mean of 4000 draws within 5 sigma; a draw's sigma is at most half the gap
    assert (np.abs(q.mean(0) - x[0]) <= 5 * step[0] / 2 / np.sqrt(4000) + step[0] / 65536).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (7, 1000), (4096, 25088), (1, 25_557_032), (1 << 20, 100)])
def test_layout(B, rows, cols):
    lay = B.qesgd_mx4_layout_query(rows, cols)
    wide = R.up(cols, 128)
    assert (lay.rows, lay.cols, lay.row_codes, lay.row_scales) == (rows, cols, wide // 2, wide // 32)
    assert lay.codes_off == 0 and lay.scales_off == R.up(rows * wide // 2, 256)
    assert lay.bytes == lay.scales_off + R.up(rows * wide // 32, 256)
    assert lay.payload_bytes == rows * (wide // 2 + wide // 32)


def test_layout_errors(B):
    for rows, cols in [(0, 1), (1, 0), (1 << 40, 1), (1, 1 << 38), (1 << 32, 1 << 7), (1 << 31, 129)]:
        with pytest.raises(B.QesgdError) as e:
            B.qesgd_mx4_layout_query(rows, cols)
        assert e.value.code == B.ERR_DIM
    B.qesgd_mx4_layout_query(1 << 31, 128)
    assert B.lib().qesgd_mx4_layout_query(1, 1, None) == B.ERR_NULL


def quantize_rc(B, x=0x10000, dtype=0, ld=300, x_stride=1 << 20, rows=100, cols=300, K=1, mode=0, packed=0x20000, ps=1 << 20,
                packed_t=None, pts=0):
    return B.lib().qesgd_mx4_quantize_pack(x, dtype, ld, x_stride, rows, cols, K, mode, 1, 0, 0, packed, ps, packed_t, pts, None)


def test_quantize_refusals(B):
    """Addresses that are none: every call is turned down before a launch."""
    assert quantize_rc(B, x=None) == B.ERR_NULL
    assert quantize_rc(B, packed=None) == B.ERR_NULL
    assert quantize_rc(B, rows=0) == B.ERR_DIM
    assert quantize_rc(B, cols=0) == B.ERR_DIM
    assert quantize_rc(B, rows=1 << 33, cols=128, ld=128) == B.ERR_DIM
    assert quantize_rc(B, rows=1 << 32, cols=1, ld=1, packed=None, packed_t=0x20000) == B.ERR_DIM
    assert quantize_rc(B, dtype=3) == B.ERR_DTYPE
    assert quantize_rc(B, K=0) == B.ERR_WORKERS
    assert quantize_rc(B, K=65) == B.ERR_WORKERS
    assert quantize_rc(B, mode=2) == B.ERR_MODE
    assert quantize_rc(B, x=0x10002) == B.ERR_ALIGN
    assert quantize_rc(B, x=0x10001, dtype=1) == B.ERR_ALIGN
    assert quantize_rc(B, packed=0x20040) == B.ERR_ALIGN
    assert quantize_rc(B, packed_t=0x20040) == B.ERR_ALIGN
    assert quantize_rc(B, ld=299) == B.ERR_STRIDE
    assert quantize_rc(B, ld=1 << 39) == B.ERR_STRIDE
    assert quantize_rc(B, K=2, x_stride=29_999) == B.ERR_STRIDE
    assert quantize_rc(B, K=2, ps=256) == B.ERR_STRIDE
    assert quantize_rc(B, K=2, ps=(1 << 20) + 16) == B.ERR_STRIDE
    assert quantize_rc(B, K=2, packed_t=0x30000, pts=256) == B.ERR_STRIDE
    assert B.lib().qesgd_last_hip_error() == 0


def test_aggregate_refusals(B):
    f = B.lib().qesgd_mx4_unpack_aggregate_update
    pk, w, z, u, zs = 0x20000, 0x30000, 0x40000, 0x50000, 0x60000
    assert f(None, 1 << 20, 2, 10, 100, w, z, u, zs, None) == B.ERR_NULL
    assert f(pk, 1 << 20, 2, 10, 100, None, None, None, None, None) == B.ERR_NULL
    assert f(pk, 1 << 20, 2, 10, 100, None, z, u, None, None) == B.ERR_NULL
    assert f(pk, 1 << 20, 2, 10, 100, w, z, None, None, None) == B.ERR_NULL
    assert f(pk, 1 << 20, 2, 0, 100, w, z, u, zs, None) == B.ERR_DIM
    assert f(pk, 1 << 20, 0, 10, 100, w, z, u, zs, None) == B.ERR_WORKERS
    assert f(pk, 1 << 20, 65, 10, 100, w, z, u, zs, None) == B.ERR_WORKERS
    assert f(pk + 128, 1 << 20, 2, 10, 100, w, z, u, zs, None) == B.ERR_ALIGN
    assert f(pk, 1 << 20, 2, 10, 100, w, z + 4, u, zs, None) == B.ERR_ALIGN
    assert f(pk, 256, 2, 10, 100, w, z, u, zs, None) == B.ERR_STRIDE


def test_product_refusals(B):
    f = B.lib().qesgd_mx4_product
    a, b, c = 0x20000, 0x30000, 0x40000
    for args in [(None, b, c), (a, None, c), (a, b, None)]:
        assert f(args[0], args[1], 8, 8, 64, args[2], 0, 8, None, 0, None) == B.ERR_NULL
    for M, N, K in [(0, 8, 64), (8, 0, 64), (8, 8, 0), ((1 << 20) + 1, 8, 64), (8, (1 << 20) + 1, 64), (8, 8, (1 << 20) + 1)]:
        assert f(a, b, M, N, K, c, 0, max(N, 8), None, 0, None) == B.ERR_DIM
        assert B.qesgd_mx4_product_workspace_bytes(M, N, K) == 0
    assert f(a, b, 8, 8, 64, c, 3, 8, None, 0, None) == B.ERR_DTYPE
    assert f(a + 16, b, 8, 8, 64, c, 0, 8, None, 0, None) == B.ERR_ALIGN
    assert f(a, b, 8, 8, 64, c + 4, 0, 8, None, 0, None) == B.ERR_ALIGN
    assert f(a, b, 8, 8, 64, c, 0, 7, None, 0, None) == B.ERR_STRIDE
    assert f(a, b, 8, 8, 64, c, 0, 1 << 39, None, 0, None) == B.ERR_STRIDE


def test_error_strings(B):
    for code in (B.ERR_DTYPE, B.ERR_MODE, B.ERR_STEPS, B.ERR_COEFF):
        assert "unknown" not in B.strerror(code)


def test_types_that_the_binding_refuses(B):
    import torch
    x = torch.zeros(4, 4, dtype=torch.float64)
    with pytest.raises(B.QesgdError) as e:
        B.qesgd_mx4_quantize_pack(x, 4, 0, 4, 4, 1, B.MX4_NEAREST, 0, 0, x, 0, stream=0)
    assert e.value.code == B.ERR_DTYPE


def test_calls_that_would_number_too_many_threads(B):
    assert quantize_rc(B, rows=(1 << 27) + 1, cols=128, ld=128) == B.ERR_DIM
    assert quantize_rc(B, rows=1 << 21, cols=1 << 13, ld=(1 << 13) + 1, packed=None, packed_t=0x20001) == B.ERR_ALIGN     # 2^34: taken
    assert quantize_rc(B, rows=1 << 28, cols=1, ld=1, packed=None, packed_t=0x20001) == B.ERR_DIM
    assert quantize_rc(B, rows=1, cols=1 << 28, ld=1, packed=0x20000, packed_t=0x30000) == B.ERR_DIM          # 2^35 in the transposed form
    f = B.lib().qesgd_mx4_unpack_aggregate_update
    assert f(0x20000, 0, 1, (1 << 27) + 1, 128, None, 0x30000, None, None, None) == B.ERR_DIM
    assert f(0x20000, 0, 1, 1 << 27, 128, None, 0x30004, None, None, None) == B.ERR_ALIGN


def test_tensors_of_the_host_are_refused(B):
    import torch
    x, p = torch.zeros(4, 4), torch.zeros(1024, dtype=torch.uint8)
    for call in (lambda: B.qesgd_mx4_quantize_pack(x, 4, 0, 4, 4, 1, B.MX4_NEAREST, 0, 0, p, 0, stream=0),
                 lambda: B.qesgd_mx4_unpack_aggregate_update(p, 0, 1, 4, 4, None, x, None, None, stream=0),
                 lambda: B.qesgd_mx4_product(p, p, 4, 4, 4, x, 4, stream=0),
                 lambda: B.qesgd_orthogonalize(x, 4, 4, 1, R.USUAL, 1e-7, x, None, stream=0),
                 lambda: B.qesgd_orthogonal_update(x, 4, 4, 1, None, 0.9, True, R.USUAL, 1e-7, 1.0, x, None, None, None, None, None, stream=0)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
