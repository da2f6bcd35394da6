"""Which tensors the matrix calls take, no GPU: the binding's checks by themselves."""
import pytest
import torch

import matrix_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 129), (7, 1000), (128, 128), (1, 70_001), (70_001, 1)])
def test_bytes_that_a_packed_matrix_takes(B, rows, cols):
    lay = B.qesgd_mx4_layout_query(rows, cols)
    assert B._mx4_bytes(rows, cols) == lay.scales_off + rows * lay.row_scales <= lay.bytes


def refused(B, code, call):
    with pytest.raises(B.QesgdError) as e:
        call()
    assert e.value.code == code


def test_packed_matrices(B):
    rows, cols, K = 9, 300, 3
    lay = B.qesgd_mx4_layout_query(rows, cols)
    need = B._mx4_bytes(rows, cols)
    slab = torch.zeros(K, lay.bytes, dtype=torch.uint8)
    wide = torch.zeros(K, lay.bytes + 512, dtype=torch.uint8)
    for t, k, stride in ((slab, K, slab.stride(0)), (slab[1], 1, 0), (slab.view(-1), K, lay.bytes), (wide[:, :lay.bytes], K, wide.stride(0)),
                         (wide[:, 256:256 + need], K, wide.stride(0)), (torch.zeros(need, dtype=torch.uint8), 1, 0)):
        assert B._packed("a", -1, t, rows, cols, k, stride) == t.data_ptr()
    for t in (slab.view(torch.int8), slab.float(), slab.view(torch.int32)):
        refused(B, B.ERR_DTYPE, lambda: B._packed("a", -1, t, rows, cols, 1, 0))
    gaps = torch.zeros(2 * lay.bytes, dtype=torch.uint8)[::2]
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, gaps, rows, cols, 1, 0))
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, slab.t(), rows, cols, K, slab.stride(0)))
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, slab[:1].expand(K, lay.bytes), rows, cols, K, lay.bytes))
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, wide[:, :lay.bytes], rows, cols, K, lay.bytes))
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, wide[:2, :lay.bytes], rows, cols, K, wide.stride(0)))
    refused(B, B.ERR_STRIDE, lambda: B._packed("a", -1, wide[:, :need - 1], rows, cols, K, wide.stride(0)))
    for short in (slab[0, :need - 1], slab[:2], slab.view(-1)[:(K - 1) * lay.bytes + need - 1]):
        with pytest.raises(ValueError, match="elements"):
            B._packed("a", -1, short, rows, cols, K if short.numel() > lay.bytes else 1, lay.bytes)


def test_views(B):
    """(count, stride) from the outermost dimension on, against views of every kind."""
    base = torch.zeros(4, 6, 40)
    for t, dims in ((base[:, :, 3:30], ((4, 240), (6, 40), (27, 1))), (base[:, 2:5, :], ((4, 240), (3, 40), (40, 1))), (base[0, :, 5:], ((1, 0), (6, 40), (35, 1))),
                    (base[:, :, :1], ((1, 7), (6, 40), (1, 1))), (base[0, 0, ::2], ((1, 0), (1, 5), (1, 1)))):
        assert not t.is_contiguous() or t.numel() < 3
        B._view("a", t, *dims)
    for t, dims in ((base.transpose(1, 2), ((4, 240), (40, 6), (6, 1))), (base[:, :, ::2], ((4, 240), (6, 40), (20, 1))), (base[:1].expand(4, 6, 40), ((4, 240), (6, 40), (40, 1))),
                    (base[0, :1].expand(6, 40), ((1, 0), (6, 40), (40, 1))), (base[:, :, 3:30], ((4, 240), (6, 27), (27, 1))), (base[:, :, 3:30], ((4, 162), (6, 40), (27, 1))),
                    (base[:, :, 3:30], ((5, 240), (6, 40), (27, 1))), (base[:, :, 3:30], ((4, 240), (7, 40), (27, 1))), (base[:, :, 3:30], ((4, 240), (6, 40), (28, 1))),
                    (base[0, :, 5:], ((2, 240), (6, 40), (35, 1)))):
        refused(B, B.ERR_STRIDE, lambda: B._view("a", t, *dims))


def test_dimensions_that_the_call_does_not_have(B):
    """Any number of the tensor's dimensions may make up one of the call's."""
    conv = torch.zeros(9, 8, 3, 3)
    for t, dims in ((conv[::2], ((1, 0), (5, 144), (72, 1))), (conv[:, ::2], ((9, 72), (4, 18), (9, 1))), (conv[::2, 1:5], ((1, 0), (5, 144), (36, 1))),
                    (conv[::2], ((5, 144), (8, 9), (9, 1))), (conv[::2], ((5, 144), (7, 9), (5, 1))), (conv[:, :, 1:], ((1, 0), (72, 9), (6, 1))),
                    (conv[:, :, 1:], ((9, 72), (8, 9), (6, 1))), (conv[::2][None, :, None], ((1, 0), (5, 144), (72, 1)))):
        assert not t.is_contiguous()
        B._view("a", t, *dims)
    for t, dims in ((conv.to(memory_format=torch.channels_last), ((1, 0), (9, 72), (72, 1))), (conv.permute(0, 2, 3, 1), ((1, 0), (9, 72), (72, 1))),
                    (conv[:, ::2], ((1, 0), (9, 36), (36, 1))), (conv[:, ::2], ((1, 0), (9, 72), (36, 1))), (conv[::2], ((1, 0), (9, 72), (72, 1))),
                    (conv[::2], ((1, 0), (6, 144), (72, 1))), (conv[::2], ((1, 0), (5, 144), (73, 1))), (conv[:, :, :, 1], ((1, 0), (9, 72), (24, 1))),
                    (torch.zeros(4, 0, 3)[:, :, ::2], ((1, 0), (2, 3), (2, 1)))):
        if t.is_contiguous():
            with pytest.raises(ValueError):
                B._view("a", t, *dims)
        else:
            refused(B, B.ERR_STRIDE, lambda: B._view("a", t, *dims))


def reached(dims):
    """Offsets that the call takes, relative to the first, in its order."""
    at = [0]
    for n, step in dims:
        at = [a + i * step for a in at for i in range(n)]
    return at


def test_what_is_taken_lies_in_the_view(B):
    """Random views and calls: one is taken only if every element that it reaches is one of the view's, and always if it goes through the
    view's own dimensions or through a part of them."""
    import random
    rng = random.Random(0)
    taken, base = 0, torch.arange(2 ** 20)
    for _ in range(20_000):
        shape = [rng.randint(1, 5) for _ in range(rng.randint(1, 4))]
        strides, step = [], 1
        for size in reversed(shape):
            step *= rng.choice([1, 1, 1, 2, 3])
            strides.insert(0, 0 if rng.random() < 0.05 else step)
            step *= size
        if rng.random() < 0.2:
            rng.shuffle(strides)
        t = base.as_strided(shape, strides)
        if t.is_contiguous():
            continue
        mine = set(t.reshape(-1).tolist())
        own = rng.random() < 0.5
        dims = [(rng.randint(1, size), stride) for size, stride in zip(shape, strides)] if own else [(rng.randint(1, 6), rng.randint(1, 40)) for _ in range(rng.randint(1, 3))]
        try:
            B._view("a", t, *dims)
            taken += 1
            assert set(reached(dims)) <= mine, (shape, strides, dims)
        except B.QesgdError:
            ordered = all(0 < b <= a for a, b in zip(strides, strides[1:])) and all(s > 0 for s in strides)
            assert not (own and ordered and all(a >= n * b for (a, b, n) in zip(strides, strides[1:], shape[1:]))), (shape, strides, dims)
    assert taken > 1000


def test_vectors_and_workspaces(B):
    v = torch.zeros(100)
    assert B._f32("a", -1, 100, v, None) == [v.data_ptr(), None]
    with pytest.raises(ValueError, match="elements"):
        B._f32("a", -1, 101, v)
    refused(B, B.ERR_STRIDE, lambda: B._f32("a", -1, 50, v[::2]))
    refused(B, B.ERR_DTYPE, lambda: B._f32("a", -1, 50, v.double()))
    assert B._ws("a", -1, v) == (v.data_ptr(), 400)
    for w in (v[::2], torch.zeros(1, dtype=torch.uint8).expand(4096)):
        refused(B, B.ERR_STRIDE, lambda: B._ws("a", -1, w))
