"""What the binding of the calls for layers of experts refuses before it launches anything: tensors of the host, of another type, too short, and
views that are not what the call says; and the views that it takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu
T, E, k, N, K = 6, 4, 2, 40, 72
R = T * k


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


def tensors(B):
    i32 = dict(dtype=torch.int32, device="cuda")
    rows = lambda n, c: torch.randn(n, c, device="cuda")  # noqa: E731
    columns = B.qesgd_mx4_grouped_columns(R, E)
    pack = lambda r, c, *n: B.alloc_mx4(B.qesgd_mx4_layout_query(r, c), *n).fill_(0)  # noqa: E731
    return dict(logits=rows(T, E), experts=torch.zeros(T, k, **i32), gates=torch.rand(T, k, device="cuda"), dgates=torch.rand(T, k, device="cuda"),
                offsets=torch.tensor([0, 3, 3, 9, 12], **i32), order=torch.arange(R, **i32), slots=torch.arange(R, **i32), dlogits=rows(T, E), x=rows(T, K),
                rows=rows(R, N), drows=rows(R, N), y=rows(T, N), dy=rows(T, N), px=pack(R, K), pxt=pack(K, columns), pdt=pack(N, columns), w=pack(N, K, E),
                c=rows(R, N), d=torch.zeros(E, N, K, device="cuda"))


# each call by the names of its tensors, outputs first
CALLS = {
    "qesgd_route": ("experts gates offsets order slots logits", lambda B, t: B.qesgd_route(t["logits"], E, T, E, k, 0, t["experts"], t["gates"], t["offsets"],
                                                                                          t["order"], t["slots"])),
    "qesgd_route_backward": ("dlogits logits experts gates dgates", lambda B, t: B.qesgd_route_backward(t["logits"], E, T, E, k, 0, t["experts"], t["gates"],
                                                                                                       t["dgates"], t["dlogits"], E)),
    "qesgd_combine": ("y rows slots gates", lambda B, t: B.qesgd_combine(t["rows"], N, R, t["slots"], t["gates"], T, k, N, t["y"], N)),
    "qesgd_combine_backward": ("drows dgates dy rows slots gates", lambda B, t: B.qesgd_combine_backward(t["dy"], N, t["rows"], N, R, t["slots"], t["gates"], T, k, N,
                                                                                                        t["drows"], N, t["dgates"])),
    "qesgd_mx4_quantize_groups": ("px pxt x order offsets", lambda B, t: B.qesgd_mx4_quantize_groups(t["x"], K, T, t["order"], k, t["offsets"], E, R, K, 0, 0, 0,
                                                                                                    t["px"], packed_t=t["pxt"])),
    "qesgd_mx4_grouped_product": ("c px w offsets", lambda B, t: B.qesgd_mx4_grouped_product(t["px"], t["w"], t["w"].stride(0), t["offsets"], E, R, N, K, t["c"], N)),
    "qesgd_mx4_grouped_gradient": ("d pdt pxt offsets", lambda B, t: B.qesgd_mx4_grouped_gradient(t["pdt"], t["pxt"], t["offsets"], E, R, N, K, t["d"])),
    "qesgd_mx4_vector_product": ("c x order w offsets", lambda B, t: B.qesgd_mx4_vector_product(t["x"], K, T, t["order"], k, t["w"], t["w"].stride(0), t["offsets"], E,
                                                                                               R, N, K, t["c"], N)),
}


def spoiled(v):
    """Forms of a tensor that no call takes."""
    yield "host", v.cpu()
    # a packed matrix ends with its last scale, up to 255 bytes before the end of its block: that is all that a call reads or writes
    yield "short", v.reshape(-1)[:-256 if v.dtype == torch.uint8 else -1].clone()
    yield "type", v.to(torch.float64) if v.dtype != torch.float64 else v.float()
    apart = torch.zeros(v.numel(), 2, dtype=v.dtype, device="cuda")[:, 0]
    apart.copy_(v.reshape(-1))
    yield "apart", apart
    if v.dim() >= 2 and v.dtype != torch.uint8:
        yield "turned", v.transpose(-1, -2).contiguous().transpose(-1, -2)
        yield "broadcast", v[:1].expand(v.shape)


@pytest.mark.parametrize("name", list(CALLS))
def test_refusals(B, name):
    names, call = CALLS[name]
    call(B, tensors(B))                                         # as it is, it runs
    for arg in names.split():
        for how, bad in spoiled(tensors(B)[arg]):
            t = tensors(B)
            before = {n: v.clone() for n, v in t.items()}
            with pytest.raises((ValueError, B.QesgdError)):
                call(B, {**t, arg: bad})
                raise SystemError(f"{name}: {arg}, {how} was taken")
            torch.cuda.synchronize()
            assert all(torch.equal(t[n], before[n]) for n in t if n != arg), (arg, how)


def test_views_whose_elements_are_the_calls(B):
    """Columns of a wider matrix with the call's stride, and tensors that are longer than the call."""
    t = tensors(B)
    B.qesgd_combine(t["rows"], N, R, t["slots"], t["gates"], T, k, N, t["y"], N)
    wide, out = torch.zeros(R, N + 9, device="cuda"), torch.full((T, N + 5), 3.0, device="cuda")
    wide[:, 4:4 + N] = t["rows"]
    B.qesgd_combine(wide[:, 4:4 + N], N + 9, R, torch.cat((t["slots"], t["slots"])), torch.cat((t["gates"], t["gates"])), T, k, N, out[:, 2:2 + N], N + 5)
    assert torch.equal(out[:, 2:2 + N], t["y"]) and (out[:, :2] == 3.0).all() and (out[:, 2 + N:] == 3.0).all()
    B.qesgd_mx4_vector_product(t["x"], K, T, t["order"], k, t["w"], t["w"].stride(0), t["offsets"], E, R, N, K, t["c"], N)
    wide = torch.zeros(T, K + 3, device="cuda")
    wide[:, 1:1 + K] = t["x"]
    out = torch.full((R, 2 * N), 3.0, device="cuda")
    B.qesgd_mx4_vector_product(wide[:, 1:1 + K], K + 3, T, t["order"], k, t["w"], t["w"].stride(0), t["offsets"], E, R, N, K, out[:, N:], 2 * N)
    assert torch.equal(out[:, N:], t["c"]) and (out[:, :N] == 3.0).all()
