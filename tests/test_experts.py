"""Layers of experts, what needs no GPU: refusals of every entry point, sizes, and the reference against itself."""
import numpy as np
import pytest
import torch

import expert_reference as X

FAKE = dict(x=0x10000, a=0x20000, b=0x30000, o=0x40000, c=0x50000, d=0x60000, e=0x70000, f=0x80000)


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    binding.lib()
    return binding


def call(B, name, spec, **changed):
    """The C entry point with the arguments of `spec` in order, some of them changed."""
    assert set(changed) <= set(spec)
    return getattr(B.lib(), name)(*{**spec, **changed}.values())


ROUTE = dict(logits=0x10000, dtype=0, ld=8, T=4, E=8, k=2, kind=0, experts=0x20000, gates=0x30000, offsets=0x40000, order=0x50000, slots=0x60000, ws=0x70000,
             ws_bytes=1 << 20, stream=None)
ROUTE_BACK = dict(logits=0x10000, dtype=0, ld=8, T=4, E=8, k=2, kind=0, experts=0x20000, gates=0x30000, dgates=0x40000, dlogits=0x50000, ld_d=8, stream=None)
COMBINE = dict(rows=0x10000, dtype=0, ld=8, R=8, slots=0x20000, gates=0x30000, T=4, k=2, N=8, out=0x40000, ld_out=8, stream=None)
COMBINE_BACK = dict(dy=0x10000, dtype=0, ld_dy=8, rows=0x20000, ld=8, R=8, slots=0x30000, gates=0x40000, T=4, k=2, N=8, drows=0x50000, ld_d=8, dgates=0x60000,
                    stream=None)
QUANTIZE = dict(x=0x10000, dtype=0, ld=8, T=4, order=0x20000, per=2, offsets=0x30000, E=3, R=8, cols=8, mode=0, seed=1, round=0, worker=0, packed=0x40000,
                packed_t=0x50000, stream=None)
PRODUCT = dict(a=0x10000, b=0x20000, stride=1 << 20, offsets=0x30000, E=3, R=8, N=8, K=8, c=0x40000, dtype=0, ldc=8, ws=0x50000, ws_bytes=1 << 30, stream=None)
GRADIENT = dict(a=0x10000, b=0x20000, offsets=0x30000, E=3, R=8, N=8, K=8, d=0x40000, dtype=0, ws=0x50000, ws_bytes=1 << 30, stream=None)
VECTOR = dict(x=0x10000, dtype=0, ld=8, T=4, order=0x20000, per=2, w=0x30000, stride=1 << 20, offsets=0x40000, E=3, R=8, N=8, K=8, y=0x50000, ldy=8, ws=0x60000,
              ws_bytes=1 << 30, stream=None)
BIG = (1 << 20) + 1
REFUSED = [
    ("qesgd_route", ROUTE, [(n, None, "NULL") for n in ("logits", "experts", "gates", "offsets", "order", "slots")] +
     [("E", 0, "EXPERTS"), ("E", 1025, "EXPERTS"), ("k", 0, "EXPERTS"), ("k", 9, "EXPERTS"), ("k", 17, "EXPERTS"), ("T", 0, "DIM"), ("T", 1 << 28, "DIM"),
      ("T", (1 << 64) - 1, "DIM"), ("dtype", 3, "DTYPE"), ("kind", 2, "MODE"), ("ld", 7, "STRIDE"), ("ld", 1 << 40, "STRIDE"), ("logits", 0x10002, "ALIGN"),
      ("experts", 0x20002, "ALIGN"), ("gates", 0x30001, "ALIGN"), ("offsets", 0x40002, "ALIGN"), ("order", 0x50002, "ALIGN"), ("slots", 0x60003, "ALIGN"),
      ("ws", 0x70008, "ALIGN")]),
    ("qesgd_route_backward", ROUTE_BACK, [(n, None, "NULL") for n in ("logits", "experts", "gates", "dgates", "dlogits")] +
     [("E", 0, "EXPERTS"), ("k", 9, "EXPERTS"), ("T", 0, "DIM"), ("dtype", 3, "DTYPE"), ("kind", 7, "MODE"), ("ld", 7, "STRIDE"), ("ld_d", 7, "STRIDE"),
      ("dlogits", 0x50002, "ALIGN"), ("dgates", 0x40002, "ALIGN")]),
    ("qesgd_combine", COMBINE, [("rows", None, "NULL"), ("out", None, "NULL"), ("k", 0, "EXPERTS"), ("k", 17, "EXPERTS"), ("T", 0, "DIM"), ("R", 0, "DIM"),
                                ("N", 0, "DIM"), ("N", (1 << 28) + 1, "DIM"), ("R", (1 << 28) + 1, "DIM"), ("T", 1 << 31, "DIM"), ("dtype", 9, "DTYPE"),
                                ("ld", 7, "STRIDE"), ("ld_out", 7, "STRIDE"), ("rows", 0x10002, "ALIGN"), ("out", 0x40001, "ALIGN"),
                                ("slots", 0x20002, "ALIGN"), ("gates", 0x30002, "ALIGN")]),
    ("qesgd_combine_backward", COMBINE_BACK, [("dy", None, "NULL"), ("rows", None, "NULL"), ("gates", None, "NULL"), ("k", 17, "EXPERTS"), ("T", 0, "DIM"),
                                              ("dtype", 9, "DTYPE"), ("ld_dy", 7, "STRIDE"), ("ld", 7, "STRIDE"), ("ld_d", 7, "STRIDE"),
                                              ("drows", 0x50002, "ALIGN"), ("dgates", 0x60002, "ALIGN")]),
    ("qesgd_mx4_quantize_groups", QUANTIZE, [("x", None, "NULL"), ("offsets", None, "NULL"), ("E", 0, "EXPERTS"), ("E", 1025, "EXPERTS"), ("R", 0, "DIM"),
                                             ("T", 0, "DIM"), ("cols", 0, "DIM"), ("per", 0, "DIM"), ("R", BIG, "DIM"), ("T", BIG, "DIM"), ("cols", BIG, "DIM"),
                                             ("dtype", 3, "DTYPE"), ("mode", 2, "MODE"), ("ld", 7, "STRIDE"), ("x", 0x10002, "ALIGN"),
                                             ("order", 0x20002, "ALIGN"), ("offsets", 0x30002, "ALIGN"), ("packed", 0x40010, "ALIGN"),
                                             ("packed_t", 0x50080, "ALIGN")]),
    ("qesgd_mx4_grouped_product", PRODUCT, [(n, None, "NULL") for n in ("a", "b", "offsets", "c")] +
     [("E", 0, "EXPERTS"), ("E", 1025, "EXPERTS"), ("R", 0, "DIM"), ("N", 0, "DIM"), ("K", 0, "DIM"), ("R", BIG, "DIM"), ("N", BIG, "DIM"), ("K", BIG, "DIM"),
      ("dtype", 3, "DTYPE"), ("ldc", 7, "STRIDE"), ("stride", 256, "STRIDE"), ("stride", (1 << 20) + 16, "STRIDE"), ("stride", 1 << 50, "STRIDE"),
      ("a", 0x10010, "ALIGN"), ("b", 0x20010, "ALIGN"), ("c", 0x40002, "ALIGN"), ("offsets", 0x30001, "ALIGN"), ("ws", 0x50008, "ALIGN")]),
    ("qesgd_mx4_grouped_gradient", GRADIENT, [(n, None, "NULL") for n in ("a", "b", "offsets", "d")] +
     [("E", 0, "EXPERTS"), ("R", 0, "DIM"), ("N", BIG, "DIM"), ("K", BIG, "DIM"), ("dtype", 3, "DTYPE"), ("a", 0x10010, "ALIGN"), ("d", 0x40002, "ALIGN")]),
    ("qesgd_mx4_vector_product", VECTOR, [(n, None, "NULL") for n in ("x", "w", "offsets", "y")] +
     [("E", 0, "EXPERTS"), ("E", 1025, "EXPERTS"), ("R", 0, "DIM"), ("T", BIG, "DIM"), ("per", 0, "DIM"), ("N", BIG, "DIM"), ("K", 0, "DIM"),
      ("dtype", 3, "DTYPE"), ("ld", 7, "STRIDE"), ("ldy", 7, "STRIDE"), ("stride", 0, "STRIDE"), ("x", 0x10002, "ALIGN"), ("w", 0x30010, "ALIGN"),
      ("y", 0x50002, "ALIGN"), ("order", 0x20002, "ALIGN")]),
]


@pytest.mark.parametrize("name,spec,refusals", REFUSED, ids=[r[0] for r in REFUSED])
def test_refusals(B, name, spec, refusals):
    """Fake device addresses: every call has to be rejected before a launch is attempted."""
    for field, value, code in refusals:
        assert call(B, name, spec, **{field: value}) == getattr(B, "ERR_" + code), (field, value)
    assert "unknown" not in B.strerror(B.ERR_EXPERTS)


def test_refusals_of_several_arguments(B):
    assert call(B, "qesgd_combine", COMBINE, slots=None, R=7) == B.ERR_DIM            # T * k rows are wanted
    assert call(B, "qesgd_combine_backward", COMBINE_BACK, drows=None, dgates=None) == B.ERR_NULL
    assert call(B, "qesgd_mx4_quantize_groups", QUANTIZE, packed=None, packed_t=None) == B.ERR_NULL
    assert call(B, "qesgd_mx4_quantize_groups", QUANTIZE, R=1 << 20, cols=1 << 20, T=1 << 20, ld=1 << 20) == B.ERR_DIM
    assert call(B, "qesgd_route", ROUTE, T=1 << 27, E=1024, ld=1024, k=1) == B.ERR_DIM  # 2^37 logits
    need = B.qesgd_route_workspace_bytes(5000, 64, 2)
    if need:
        big = dict(ROUTE, T=5000, E=64, ld=64)
        assert call(B, "qesgd_route", big, ws=None) == B.ERR_WORKSPACE
        assert call(B, "qesgd_route", big, ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_workspaces_that_are_too_small(B):
    for name, spec, rows in (("qesgd_mx4_grouped_product", PRODUCT, 64), ("qesgd_mx4_grouped_gradient", GRADIENT, 4096), ("qesgd_mx4_vector_product", VECTOR, 4)):
        for N, K in ((64, 64), (64, 1 << 15), (1000, 8192)):
            need = getattr(B, name + "_workspace_bytes")(rows, N, K, 3)
            if need:
                sizes = dict(spec, R=rows, N=N, K=K, **{k: 1 << 20 for k in ("ldc", "ldy", "ld") if k in spec}, **({"stride": 1 << 30} if "stride" in spec else {}))
                assert call(B, name, sizes, ws=None) == B.ERR_WORKSPACE
                assert call(B, name, sizes, ws_bytes=need - 1) == B.ERR_WORKSPACE


def test_sizes(B):
    for R_, E in ((1, 1), (1, 1024), (127, 1), (128, 1), (129, 3), (1000, 7), (1 << 20, 1024)):
        columns = B.qesgd_mx4_grouped_columns(R_, E)
        assert columns == X.group_columns(R_, E) and columns % 128 == 0 and columns >= R_
    # the worst that rows can do: one more than a multiple of 128 in as many groups as there are
    for R_, E in ((10, 4), (300, 3), (1000, 500), (129 * 5, 5)):
        used = min(E, R_)
        groups = [1] * used
        groups[0] += R_ - used
        most = sum((g + 127) // 128 * 128 for g in groups)
        assert most <= B.qesgd_mx4_grouped_columns(R_, E)
    assert B.qesgd_mx4_grouped_columns(0, 1) == 0 and B.qesgd_mx4_grouped_columns(5, 0) == 0 and B.qesgd_mx4_grouped_columns(BIG, 1) == 0
    assert B.qesgd_route_workspace_bytes(0, 8, 2) == 0 and B.qesgd_route_workspace_bytes(8, 8, 9) == 0
    for name in ("grouped_product", "grouped_gradient", "vector_product"):
        assert getattr(B, f"qesgd_mx4_{name}_workspace_bytes")(0, 8, 8, 1) == 0


def test_binding_refuses_tensors_of_the_host(B):
    """Before anything is read: the kernels take addresses of the current GPU."""
    if torch.cuda.is_available():
        pytest.skip("a GPU is there")
    x, i = torch.zeros(4, 8), torch.zeros(16, dtype=torch.int32)
    p = torch.zeros(1 << 12, dtype=torch.uint8)
    for f in (lambda: B.qesgd_route(x, 8, 4, 8, 2, 0, i, x, i, i, i), lambda: B.qesgd_combine(x, 8, 4, i, x, 2, 2, 8, x, 8),
              lambda: B.qesgd_mx4_quantize_groups(x, 8, 4, None, 1, i, 2, 4, 8, 0, 0, 0, p),
              lambda: B.qesgd_mx4_grouped_product(p, p, 1024, i, 1, 4, 8, 8, x, 8),
              lambda: B.qesgd_mx4_vector_product(x, 8, 4, None, 1, p, 0, None, 1, 4, 8, 8, x, 8)):
        with pytest.raises((ValueError, AssertionError, RuntimeError, AttributeError, TypeError)):
            f()


def test_reference_route():
    """The reference's sort against one pair at a time."""
    rng = np.random.default_rng(0)
    l = np.round(rng.standard_normal((30, 7)) * 2)
    l[rng.random((30, 7)) < 0.3] = -np.inf
    experts, gates, offsets, order, slots = X.route(l, 3, True)
    places = []
    for e in range(7):
        assert offsets[e] == len(places)
        for t in range(30):
            for j in range(3):
                if experts[t, j] == e:
                    places.append(t * 3 + j)
    assert places == order.tolist() and offsets[7] == len(places)
    for i, s in enumerate(slots):
        assert s == (places.index(i) if i in places else -1)
    for t in range(30):
        ranked = sorted(range(7), key=lambda e: (-l[t, e], e))[:3]
        assert experts[t].tolist() == [e if l[t, e] > -np.inf else -1 for e in ranked]
