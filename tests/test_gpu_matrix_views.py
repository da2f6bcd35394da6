"""Which tensors the matrix calls take: each refusal on a GPU's tensors, nothing written, and the views that have their strides in the call."""
import numpy as np
import pytest
import torch

import matrix_reference as R

pytestmark = pytest.mark.gpu
USUAL = R.USUAL


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def refused(B, call, *codes):
    with pytest.raises((B.QesgdError, ValueError)) as e:
        call()
    assert (e.value.code if isinstance(e.value, B.QesgdError) else None) in codes


def test_the_quantiser(B):
    rows, cols = 64, 64
    x = torch.randn(rows, cols, device="cuda")
    lay = B.qesgd_mx4_layout_query(rows, cols)
    p, t = (B.alloc_mx4(lay).fill_(0xA5) for _ in range(2))

    def call(v=x, ld=cols, r=rows, c=cols, K=1, xs=0, packed=p, ps=0, packed_t=t, pts=0):
        B.qesgd_mx4_quantize_pack(v, ld, xs, r, c, K, B.MX4_NEAREST, 0, 0, packed, ps, packed_t=packed_t, packed_t_stride=pts)

    for v in (x.t(), torch.randn(64, 128, device="cuda")[:, ::2], torch.randn(64, device="cuda").expand(64, 64), torch.randn(64, 1, device="cuda").expand(64, 64),
              torch.randn(64, 128, device="cuda")[:, :64]):
        refused(B, lambda: call(v), B.ERR_STRIDE)
    refused(B, lambda: call(x[:63]), None)                      # too few rows
    refused(B, lambda: call(ld=65), None)                       # rows further apart than the tensor has room for
    refused(B, lambda: call(K=2, xs=4096, packed=B.alloc_mx4(lay, 2), ps=lay.bytes, packed_t=None), None)
    for bad in (p.view(torch.int8), p.view(torch.float32)):
        refused(B, lambda: call(packed=bad), B.ERR_DTYPE)
        refused(B, lambda: call(packed_t=bad), B.ERR_DTYPE)
    gaps = torch.zeros(2 * lay.bytes, dtype=torch.uint8, device="cuda")[::2]
    refused(B, lambda: call(packed=gaps), B.ERR_STRIDE)
    refused(B, lambda: call(packed_t=gaps), B.ERR_STRIDE)
    short = torch.zeros(lay.bytes - 256, dtype=torch.uint8, device="cuda")
    refused(B, lambda: call(packed=short), None)
    refused(B, lambda: call(packed_t=short), None)
    assert bool((p == 0xA5).all()) and bool((t == 0xA5).all())

    # rows apart, workers apart, in the tensor as in the call
    wide = torch.randn(3, 70, 200, device="cuda")
    v = wide[:, 3:67, 10:74]
    slab = torch.zeros(3, lay.bytes + 256, dtype=torch.uint8, device="cuda")
    call(v, ld=200, K=3, xs=wide.stride(0), packed=slab[:, :lay.bytes], ps=slab.stride(0), packed_t=None)
    for k in range(3):
        call(v[k].contiguous(), packed=p, packed_t=None)
        assert torch.equal(slab[k, :lay.scales_off], p[:lay.scales_off])
    assert not slab[:, lay.bytes:].any()
    column = torch.randn(64, 10, device="cuda")[:, 4]           # a matrix of one column has no steps between columns
    one, two = (B.alloc_mx4(B.qesgd_mx4_layout_query(64, 1)).fill_(0) for _ in range(2))
    call(column[:, None], ld=10, c=1, packed=one, packed_t=None)
    call(column.contiguous(), ld=1, c=1, packed=two, packed_t=None)
    assert torch.equal(one, two)


def test_the_mean(B):
    rows, cols, K = 40, 100, 3
    lay = B.qesgd_mx4_layout_query(rows, cols)
    slab = torch.zeros(K, lay.bytes, dtype=torch.uint8, device="cuda")
    out = {n: torch.full((rows * cols,), 7.0, device="cuda") for n in ("w", "z", "u", "zs")}

    def call(p=slab, ps=lay.bytes, **other):
        o = {**out, **other}
        B.qesgd_mx4_unpack_aggregate_update(p, ps, K, rows, cols, o["w"], o["z"], o["u"], o["zs"])

    refused(B, lambda: call(slab.view(torch.int32)), B.ERR_DTYPE)
    refused(B, lambda: call(slab[:1].expand(K, lay.bytes)), B.ERR_STRIDE)
    refused(B, lambda: call(slab[:2]), None)
    for n in out:
        refused(B, lambda: call(**{n: torch.zeros(2 * rows * cols, device="cuda")[::2]}), B.ERR_STRIDE)
        refused(B, lambda: call(**{n: torch.zeros(rows * cols - 1, device="cuda")}), None)
        refused(B, lambda: call(**{n: torch.zeros(rows * cols, device="cuda", dtype=torch.float64)}), B.ERR_DTYPE)
    assert all(bool((t == 7.0).all()) for t in out.values())
    call()
    assert not out["z"].any() and bool((out["u"] == 7.0).all())


def test_the_product(B):
    M, N, K = 48, 80, 200
    la, lb = B.qesgd_mx4_layout_query(M, K), B.qesgd_mx4_layout_query(N, K)
    a, b = (torch.zeros(lay.bytes, dtype=torch.uint8, device="cuda") for lay in (la, lb))
    c = torch.full((M, N), 3.0, device="cuda")

    def call(a=a, b=b, c=c, ldc=N, ws=None):
        B.qesgd_mx4_product(a, b, M, N, K, c, ldc, workspace=ws)

    guard = torch.full((M, 2 * N), 3.0, device="cuda")
    for bad in (guard[:, ::2], torch.full((N, M), 3.0, device="cuda").t(), torch.full((N,), 3.0, device="cuda").expand(M, N), guard[:, :N]):
        refused(B, lambda: call(c=bad), B.ERR_STRIDE)
        assert bool((bad == 3.0).all())
    refused(B, lambda: call(c=c[:M - 1]), None)
    refused(B, lambda: call(ldc=N + 1), None)
    for n in ("a", "b"):
        lay, own = (la, a) if n == "a" else (lb, b)
        refused(B, lambda: call(**{n: own.view(torch.int8)}), B.ERR_DTYPE)
        refused(B, lambda: call(**{n: torch.zeros(2 * lay.bytes, dtype=torch.uint8, device="cuda")[::2]}), B.ERR_STRIDE)
        refused(B, lambda: call(**{n: own[:lay.scales_off]}), None)
    refused(B, lambda: call(ws=torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 20)), B.ERR_STRIDE)
    assert bool((c == 3.0).all())
    call(c=guard[:, :N], ldc=2 * N)                             # rows apart in the tensor as in the call
    assert not guard[:, :N].any() and bool((guard[:, N:] == 3.0).all())
    call(c=torch.empty(M * 2 * N, device="cuda"), ldc=2 * N)    # a flat buffer with room


def test_the_orthogonalised_update(B):
    n, rows, cols = 2, 40, 60
    shape = (n, rows, cols)

    def tensors():
        return [torch.randn(shape, device="cuda") for _ in range(7)]      # g, momentum, step, z, w, u, zsum

    bad = [lambda: torch.randn(n, cols, rows, device="cuda").mT, lambda: torch.randn(rows, cols, device="cuda").expand(shape),
           lambda: torch.randn(n, rows, 2 * cols, device="cuda")[:, :, :cols], lambda: torch.randn(n, rows, cols + 1, device="cuda")[:, :, 1:]]
    for at in range(7):
        for make, codes in [(m, (B.ERR_STRIDE,)) for m in bad] + [(lambda: torch.randn(1, rows, cols, device="cuda"), (None,)),
                                                                  (lambda: torch.randn(shape, device="cuda", dtype=torch.float64), (B.ERR_DTYPE,))]:
            t = tensors()
            t[at] = make()
            kept = [v.clone() for v in t]
            g, m, step, z, w, u, zsum = t
            refused(B, lambda: B.qesgd_orthogonal_update(g, rows, cols, n, m, 0.9, True, USUAL, 1e-7, 1.0, step, z, w, u, zsum, None), *codes)
            assert all(torch.equal(v, k) for v, k in zip(t, kept))
    x, out = torch.randn(shape, device="cuda"), torch.full(shape, 5.0, device="cuda")
    refused(B, lambda: B.qesgd_orthogonalize(x[:1], rows, cols, n, USUAL, 1e-7, out, None), None)
    refused(B, lambda: B.qesgd_orthogonalize(x, rows, cols, n, USUAL, 1e-7, out[:1], None), None)
    assert bool((out == 5.0).all())
    big = torch.randn(1, 300, 400, device="cuda")
    need = B.qesgd_orthogonalize_workspace_bytes(300, 400, 1)
    refused(B, lambda: B.qesgd_orthogonalize(big, 300, 400, 1, USUAL, 1e-7, torch.empty_like(big), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(need)), B.ERR_STRIDE)
    assert np.isfinite(big.sum().item())
