"""What is measured of the operators for matrix parameters: 4-bit microscaled codes and orthogonalised updates.

A case is a dict of plain values.  Its "kind" says which calls make up one pass:

  mean     a round on the wire: qesgd_mx4_quantize_pack of the K workers' matrices, then
           qesgd_mx4_unpack_aggregate_update on the server (rows = 1: a plain vector)
  product  a layer on packed parameters: qesgd_mx4_quantize_pack of the activations, then
           qesgd_mx4_product with the packed weights that the server has sent
  train    a layer's forward pass and both gradients, all three operands quantised in the call, along
           their rows and along their columns
  ortho    the server's step on a batch of equal matrices: momentum, Newton-Schulz iteration, update
           (qesgd_orthogonal_update)
  whiten   qesgd_orthogonalize alone: a matrix in, its orthogonal factor in the same type out

The packed form: a matrix [rows, cols] is padded with zeros to a multiple of 128 columns; two 4-bit elements (E2M1: sign,
0 .5 1 1.5 2 3 4 6) per byte, the even column in the low half; behind the codes, at the next multiple of 256 bytes, one byte
e + 127 for each 32 columns, 255 where one of the 32 is not finite.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFS = ((3.4445, -4.7750, 2.0315),) * 5       # the usual quintic: singular values end within about 0.7 .. 1.2
EPS = 1e-7


def listed():
    return [
        # the least: a small dense layer's gradient from four workers; all latency
        dict(name="mean-16k", kind="mean", rows=128, cols=128, K=4, dtype="f32", mode="stochastic"),
        # odd in everything: five workers, half-width gradients, rows that start nowhere aligned
        dict(name="mean-7m-odd", kind="mean", rows=2737, cols=2681, K=5, dtype="bf16", mode="stochastic"),
        # a mid-sized network's parameters as one vector, many workers
        dict(name="mean-26m", kind="mean", rows=1, cols=25_557_032, K=16, dtype="f32", mode="stochastic"),
        # a single sample through a square layer
        dict(name="product-1x4096", kind="product", M=1, N=4096, K=4096, dtype="bf16"),
        # a few samples through a classifier of 1000 outputs, an odd width
        dict(name="product-37-odd", kind="product", M=37, N=1000, K=2049, dtype="f32"),
        # a large batch through the widest layer of a 138 M parameter network
        dict(name="product-4096x25088", kind="product", M=4096, N=4096, K=25_088, dtype="bf16"),
        # a training step of a small layer
        dict(name="train-512", kind="train", M=256, N=512, K=512, dtype="f32", mode="nearest"),
        # a training step of a large one; gradients rounded without bias
        dict(name="train-4096", kind="train", M=8192, N=4096, K=4096, dtype="bf16", mode="stochastic"),
        # the small matrices that attention-like and narrow layers have, many of one shape at once
        dict(name="ortho-16x64", kind="ortho", rows=64, cols=64, n=16, nesterov=True),
        # two 512-channel 3 x 3 convolutions of an 11 M parameter network as matrices
        dict(name="ortho-512x4608", kind="ortho", rows=512, cols=4608, n=2, nesterov=True),
        # odd, more rows than columns, half width in and out
        dict(name="whiten-2049x1000", kind="whiten", rows=2049, cols=1000, n=1, dtype="bf16"),
        # the largest: the widest layer of a 138 M parameter network
        dict(name="ortho-4096x25088", kind="ortho", rows=4096, cols=25_088, n=1, nesterov=False),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["mean", "mean", "product", "product", "train", "ortho", "ortho", "whiten"])
    dtype = rng.choice(["f32", "f32", "bf16", "bf16", "f16"])
    mode = rng.choice(["stochastic", "nearest"])
    if kind == "mean":
        K = rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 16])
        d = log_int(rng, 256, 408_000_000 // K)
        rows = 1 if rng.random() < 0.3 else min(d, log_int(rng, 1, 8192))
        cols = max(1, d // rows)
        if rng.random() < 0.4 and cols > 128:
            cols = cols // 64 * 64
        return dict(kind=kind, rows=rows, cols=cols, K=K, dtype=dtype, mode=mode)
    if kind == "product":
        M = 1 if rng.random() < 0.25 else log_int(rng, 1, 8192)
        N, K = log_int(rng, 64, 16384), log_int(rng, 32, 25_088)
        if rng.random() < 0.5:
            N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
        N = max(16, min(N, 4096 * 4096 * 25_088 // (M * K)))
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype)
    if kind == "train":
        M, N, K = log_int(rng, 32, 8192), log_int(rng, 32, 8192), log_int(rng, 32, 8192)
        if rng.random() < 0.5:
            M, N, K = (max(64, v // 64 * 64) for v in (M, N, K))
        M = max(16, min(M, 8192 * 4096 * 4096 // (N * K)))
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, mode=mode)
    m, wide = log_int(rng, 8, 4096), math.exp(rng.uniform(0, math.log(8)))
    if rng.random() < 0.4:
        m = max(16, m // 16 * 16)
    rows, cols = m, int(m * wide)
    n = rng.choice([1, 1, 2, 4, 12]) if m <= 1024 else 1
    if rng.random() < 0.4:
        rows, cols = cols, rows
    cols = max(1, min(cols, 4096 * 25_088 // rows))
    if kind == "whiten":
        return dict(kind=kind, rows=rows, cols=cols, n=n, dtype=dtype)
    return dict(kind=kind, rows=rows, cols=cols, n=n, nesterov=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------

def generator(seed, stream):
    return torch.Generator(device=DEV).manual_seed(((int(seed) + 1) << 8) + stream)


def gradients(shape, seed, stream, dtype):
    """Heavy tails and rows of different size, as gradients have them, and some exact zeros."""
    g = generator(seed, stream)
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(torch.randn(shape[:-1] + (1,), generator=g, device=DEV)) * 1e-3
    x *= 1.0 + 4.0 * (torch.rand(shape, generator=g, device=DEV) < 0.02)
    x *= torch.rand(shape, generator=g, device=DEV) > 0.01
    return x.to(dtype)


def activations(shape, seed, stream, dtype):
    """What comes out of a rectifier with a few channels that are much larger."""
    g = generator(seed, stream)
    x = torch.randn(shape, generator=g, device=DEV).clamp_(min=-0.1)
    x *= 1.0 + 7.0 * (torch.rand(shape[-1:], generator=g, device=DEV) < 0.01)
    return x.to(dtype)


def weights(shape, seed, stream, dtype):
    return (torch.randn(shape, generator=generator(seed, stream), device=DEV) / math.sqrt(shape[-1])).to(dtype)


def update_matrices(shape, seed, stream):
    """Updates whose singular values fall off: noise and a few strong directions."""
    g = generator(seed, stream)
    n, rows, cols = shape
    r = max(1, min(rows, cols) // 16)
    left = torch.randn((n, rows, r), generator=g, device=DEV) / (1.0 + torch.arange(r, device=DEV))
    x = torch.randn(shape, generator=g, device=DEV) + 4.0 * torch.matmul(left, torch.randn((n, r, cols), generator=g, device=DEV))
    return x * 1e-3


def up(v, a):
    return (v + a - 1) // a * a


def packed_sizes(rows, cols):
    """(bytes of a row of codes, where the scales begin, bytes of a row of scales, bytes in all)"""
    wide = up(cols, 128)
    at = up(rows * wide // 2, 256)
    return wide // 2, at, wide // 32, at + up(rows * wide // 32, 256)


def packed_buffer(rows, cols, K=None):
    size = packed_sizes(rows, cols)[3]
    return torch.zeros((size,) if K is None else (K, size), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    kind = case["kind"]
    state = dict(case=case, seed=int(seed), kept={})
    if kind == "mean":
        rows, cols, K = case["rows"], case["cols"], case["K"]
        state.update(x=gradients((K, rows, cols), seed, 0, DTYPES[case["dtype"]]),
                     w=torch.randn(rows * cols, generator=generator(seed, 1), device=DEV) * 0.05,
                     packed=packed_buffer(rows, cols, K), z=torch.empty(rows * cols, device=DEV),
                     u=torch.empty(rows * cols, device=DEV), zsum=torch.zeros(rows * cols, device=DEV))
    elif kind == "product":
        M, N, K, t = case["M"], case["N"], case["K"], DTYPES[case["dtype"]]
        # the weights arrive packed, as the server has sent them
        wide, at, per, size = packed_sizes(N, K)
        w = torch.zeros(N, wide * 2, device=DEV)
        w[:, :K] = weights((N, K), seed, 1, torch.float32)
        q, e = nearest_parts(w)
        b = packed_buffer(N, K)
        code = (torch.bucketize(q.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)) + 8 * (q < 0)).to(torch.uint8)
        b[:N * wide] = (code[:, 0::2] | (code[:, 1::2] << 4)).reshape(-1)
        b[at:at + N * per] = (e + 127).to(torch.uint8).reshape(-1)
        state.update(x=activations((M, K), seed, 0, t), a=packed_buffer(M, K), b=b, y=torch.empty((M, N), dtype=t, device=DEV))
    elif kind == "train":
        M, N, K, t = case["M"], case["N"], case["K"], DTYPES[case["dtype"]]
        state.update(x=activations((M, K), seed, 0, t), w=weights((N, K), seed, 1, t), dy=gradients((M, N), seed, 2, t),
                     px=packed_buffer(M, K), pxt=packed_buffer(K, M), pw=packed_buffer(N, K), pwt=packed_buffer(K, N),
                     pdy=packed_buffer(M, N), pdyt=packed_buffer(N, M), y=torch.empty((M, N), dtype=t, device=DEV),
                     dx=torch.empty((M, K), dtype=t, device=DEV), dw=torch.empty((N, K), dtype=t, device=DEV))
    elif kind == "ortho":
        shape = (case["n"], case["rows"], case["cols"])
        state.update(g=update_matrices(shape, seed, 0), m=update_matrices(shape, seed, 1),
                     w=torch.randn(shape, generator=generator(seed, 2), device=DEV) * 0.05,
                     z=torch.zeros(shape, device=DEV), u=torch.empty(shape, device=DEV), zsum=torch.zeros(shape, device=DEV),
                     step=torch.empty(shape, device=DEV), mu=0.95, alpha=-0.02 * math.sqrt(max(1.0, case["rows"] / case["cols"])))
    else:
        shape = (case["n"], case["rows"], case["cols"])
        state.update(x=update_matrices(shape, seed, 0).to(DTYPES[case["dtype"]]), out=torch.empty(shape, dtype=DTYPES[case["dtype"]], device=DEV))
    return state


# ---- plain form -----------------------------------------------------------

def philox(c, key):
    """Philox4x32-10 of counters c (four int64 tensors of 32-bit values); the four output words."""
    low = 0xFFFFFFFF
    k0, k1 = key & low, key >> 32
    c0, c1, c2, c3 = c
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def variates(K, rows, wide, seed, rnd):
    """The 16-bit variates of K workers' padded matrices: coordinate i = row * wide + column takes half i & 1 of word (i & 7) >> 1
    of the call for i >> 3."""
    g = torch.arange(rows * wide // 8, dtype=torch.int64, device=DEV)[None, :]
    worker = torch.arange(K, dtype=torch.int64, device=DEV)[:, None]
    words = torch.stack(philox(torch.broadcast_tensors(g & 0xFFFFFFFF, g >> 32, worker, torch.full_like(g, rnd)), seed), 2)
    return torch.stack((words & 0xFFFF, words >> 16), 3).reshape(K, rows, wide)


def power_of_two(e):
    """2^e in 32 bits for e of -127 .. 126, from its bits."""
    return ((e.int() + 128) << 23).view(torch.float32) * 0.5


def scaled(x, stochastic):
    """Magnitudes over their block's scale, and the exponent of each block: x [..., padded columns] in 32 bits."""
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    amax = blocks.abs().amax(-1)
    frac, e = torch.frexp(amax)                              # amax = frac * 2^e, frac in [1/2, 1)
    e = e - 3                                                # amax / 2^e in [4, 8)
    if stochastic:
        e = e + (frac > 0.75).to(e.dtype)                    # ... in (3, 6]: nothing is cut off
    e = torch.where(amax == 0, -127, e).clamp(-127, 125)
    # exact wherever the result's grid sees it
    return blocks.abs() * power_of_two(-e - 1)[..., None] * 2.0, e, torch.isfinite(amax)


def nearest_parts(x):
    a, e, fine = scaled(x, False)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)        # ties to the even code
    return torch.where(x < 0, -q.reshape(x.shape), q.reshape(x.shape)), torch.where(fine, e, 128)


def mx4_values(x, mode, seed=0, rnd=0):
    """The values that the 4-bit forms of the workers' matrices x [K, rows, cols] stand for, blocks along the rows."""
    K, rows, cols = x.shape
    wide = up(cols, 128)
    v = torch.nn.functional.pad(x.float(), (0, wide - cols))
    if mode == "nearest":
        q, e = nearest_parts(v)
        fine = e != 128
    else:
        a, e, fine = scaled(v, True)
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        low = torch.floor(a / step)
        part = torch.floor((a / step - low) * 65536.0)
        r = variates(K, rows, wide, seed, rnd).reshape(a.shape)
        q = ((low + (r + part >= 65536).float()) * step).clamp(max=6.0).reshape(v.shape)
        q = torch.where(v < 0, -q, q)
    scale = torch.where(fine, power_of_two(torch.where(fine, e, 0)), math.nan)
    return (q.reshape(fine.shape + (32,)) * scale[..., None]).reshape(K, rows, wide)[..., :cols]


def mx4_matrix(x, mode, seed=0, rnd=0):
    return mx4_values(x[None], mode, seed, rnd)[0]


def mx4_decode(packed, rows, cols):
    wide, at, per, _ = packed_sizes(rows, cols)
    codes = packed[:rows * wide].reshape(rows, wide)
    code = torch.stack((codes & 15, codes >> 4), 2).reshape(rows, wide * 2).long()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    e = packed[at:at + rows * per].reshape(rows, per).int()
    scale = torch.where(e == 255, math.nan, power_of_two(torch.where(e == 255, 0, e - 127)))
    return (grid[code].reshape(rows, per, 32) * scale[:, :, None]).reshape(rows, -1)[:, :cols]


def newton_schulz(x):
    """x [n, rows, cols] in 32 bits."""
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()
    x = x * (1.0 / (norm + EPS)).float()
    turn = x.shape[1] > x.shape[2]
    if turn:
        x = x.transpose(1, 2).contiguous()
    for a, b, c in COEFFS:
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(1, 2).contiguous() if turn else x


def plain(state):
    case, seed = state["case"], state["seed"]
    kind = case["kind"]
    if kind == "mean":
        z = mx4_values(state["x"], case["mode"], seed, 3).sum(0).reshape(-1) / case["K"]
        state["zsum"] += z
        return [z, state["w"] + z, state["zsum"]]
    if kind == "product":
        a = mx4_matrix(state["x"], "nearest")
        b = mx4_decode(state["b"], case["N"], case["K"])
        return torch.matmul(a, b.t()).to(state["x"].dtype)
    if kind == "train":
        x, w, dy, t, mode = state["x"], state["w"], state["dy"], state["x"].dtype, case["mode"]
        y = torch.matmul(mx4_matrix(x, "nearest"), mx4_matrix(w, "nearest").t())
        dx = torch.matmul(mx4_matrix(dy, mode, seed, 5), mx4_matrix(w.t(), "nearest").t())
        dw = torch.matmul(mx4_matrix(dy.t(), mode, seed, 5), mx4_matrix(x.t(), "nearest").t())
        return [y.to(t), dx.to(t), dw.to(t)]
    if kind == "ortho":
        g, m = state["g"], state["m"]
        m *= state["mu"]
        m += g
        step = newton_schulz(g + state["mu"] * m if case["nesterov"] else m) * state["alpha"]
        state["z"] += step
        state["zsum"] += state["z"]
        return [m, step, state["z"], state["w"] + state["z"], state["zsum"]]
    return newton_schulz(state["x"].float()).to(state["x"].dtype)


# ---- the library's calls --------------------------------------------------

def run(state):
    if not own:
        return plain(state)
    from paper_1901_03040_amd import binding as B
    case, seed, kept = state["case"], state["seed"], state["kept"]
    kind = case["kind"]
    if kind == "mean":
        rows, cols, K, x, packed = case["rows"], case["cols"], case["K"], state["x"], state["packed"]
        mode = B.MX4_STOCHASTIC if case["mode"] == "stochastic" else B.MX4_NEAREST
        B.qesgd_mx4_quantize_pack(x, x.stride(1), x.stride(0), rows, cols, K, mode, seed, 3, packed, packed.stride(0))
        B.qesgd_mx4_unpack_aggregate_update(packed, packed.stride(0), K, rows, cols, state["w"], state["z"], state["u"], state["zsum"])
        return [state["z"], state["u"], state["zsum"]]
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        if not kept:                                         # a worker keeps its scratch from step to step
            kept["ws"] = B.alloc_workspace(B.qesgd_mx4_product_workspace_bytes(M, N, K), DEV)
        B.qesgd_mx4_quantize_pack(state["x"], K, 0, M, K, 1, B.MX4_NEAREST, 0, 0, state["a"], 0)
        B.qesgd_mx4_product(state["a"], state["b"], M, N, K, state["y"], N, workspace=kept["ws"])
        return state["y"]
    if kind == "train":
        M, N, K = case["M"], case["N"], case["K"]
        mode = B.MX4_STOCHASTIC if case["mode"] == "stochastic" else B.MX4_NEAREST
        if not kept:
            need = max(B.qesgd_mx4_product_workspace_bytes(*s) for s in ((M, N, K), (M, K, N), (N, K, M)))
            kept["ws"] = B.alloc_workspace(need, DEV)
        B.qesgd_mx4_quantize_pack(state["x"], K, 0, M, K, 1, B.MX4_NEAREST, 0, 0, state["px"], 0, packed_t=state["pxt"])
        B.qesgd_mx4_quantize_pack(state["w"], K, 0, N, K, 1, B.MX4_NEAREST, 0, 0, state["pw"], 0, packed_t=state["pwt"])
        B.qesgd_mx4_product(state["px"], state["pw"], M, N, K, state["y"], N, workspace=kept["ws"])
        B.qesgd_mx4_quantize_pack(state["dy"], N, 0, M, N, 1, mode, seed, 5, state["pdy"], 0, packed_t=state["pdyt"])
        B.qesgd_mx4_product(state["pdy"], state["pwt"], M, K, N, state["dx"], K, workspace=kept["ws"])
        B.qesgd_mx4_product(state["pdyt"], state["pxt"], N, K, M, state["dw"], K, workspace=kept["ws"])
        return [state["y"], state["dx"], state["dw"]]
    n, rows, cols = case["n"], case["rows"], case["cols"]
    if not kept:
        kept["ws"] = B.alloc_workspace(B.qesgd_orthogonalize_workspace_bytes(rows, cols, n), DEV)
    if kind == "ortho":
        B.qesgd_orthogonal_update(state["g"], rows, cols, n, state["m"], state["mu"], case["nesterov"], COEFFS, EPS, state["alpha"],
                                  state["step"], state["z"], state["w"], state["u"], state["zsum"], kept["ws"])
        return [state["m"], state["step"], state["z"], state["u"], state["zsum"]]
    B.qesgd_orthogonalize(state["x"], rows, cols, n, COEFFS, EPS, state["out"], kept["ws"])
    return state["out"]


# ---- what it has to do ----------------------------------------------------

def work(case):
    kind = case["kind"]
    size = 4 if case.get("dtype", "f32") == "f32" else 2
    if kind == "mean":
        d, K = case["rows"] * case["cols"], case["K"]
        code = case["rows"] * (-(-case["cols"] // 2) + -(-case["cols"] // 32))
        return {"bytes": K * (size * d + 2 * code) + 20 * d, "flops": 0}
    if kind in ("product", "train"):
        M, N, K = case["M"], case["N"], case["K"]
        code = lambda r, c: r * (-(-c // 2) + -(-c // 32))  # noqa: E731
        if kind == "product":
            return {"bytes": size * M * (K + N) + 2 * code(M, K) + code(N, K), "flops": 2 * M * N * K}
        both = 2 * sum(code(r, c) + code(c, r) for r, c in ((M, K), (N, K), (M, N)))
        return {"bytes": 2 * size * (M * K + N * K + M * N) + both, "flops": 6 * M * N * K}
    # a symmetric product needs half of its operations
    m, k, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"]), case["n"]
    flops = n * len(COEFFS) * (3 * m * m * k + m * m * m)
    d = n * m * k
    return {"bytes": (2 * size if kind == "whiten" else 44) * d, "flops": flops}


# ---- in 64 bits -----------------------------------------------------------

def exact_mx4(x, mode, seed=0, rnd=0, worker=0):
    """From the definition: the scale from the largest magnitude's binary exponent, the element from the list of values."""
    rows, cols = x.shape
    wide = -(-cols // 128) * 128
    v = torch.zeros((rows, wide), dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    out = torch.empty_like(v)
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 8.0], dtype=torch.float64, device=x.device)
    top = v.view(rows, -1, 32).abs().amax(2)
    e = (top.view(torch.int64) >> 52) - 1023 - 2                 # floor(log2(top)) - 2; 0 has the lowest exponent
    power = lambda e: ((e + 1023) << 52).view(torch.float64)  # noqa: E731
    if mode == "stochastic":
        e = torch.where((top > 0) & (top > 6 * power(e.clamp(min=-1000))), e + 1, e)
    s = power(e.clamp(-127, 125)).repeat_interleave(32, 1)
    part = max(1, (1 << 24) // wide)
    for r in range(0, rows, part):
        a = v[r:r + part].abs() / s[r:r + part]
        at = (torch.searchsorted(values, a, right=True) - 1).clamp(0, 7)
        low, high = values[at], values[at + 1]
        f = (a - low) / (high - low)
        if mode == "nearest":
            more = (f > 0.5) | ((f == 0.5) & (at % 2 == 1))
        else:
            n = a.shape[0]
            i = torch.arange(r * wide, (r + n) * wide, device=x.device).view(n, wide)
            g = i[:, ::8].reshape(-1) // 8
            words = philox((g % (1 << 32), g // (1 << 32), torch.full_like(g, worker), torch.full_like(g, rnd)), seed)
            word = torch.stack(words, -1)[:, [0, 0, 1, 1, 2, 2, 3, 3]].view(n, wide)
            u = torch.where(i % 2 == 0, word % 65536, word // 65536)
            more = u.double() + torch.floor(f * 65536) >= 65536
        q = torch.minimum(torch.where(more, high, low), values[7])
        out[r:r + part] = torch.sign(v[r:r + part]) * q * s[r:r + part]
    return out[:, :cols]


def exact_factor(x):
    """Through the singular values where that is quick, by products otherwise."""
    n = torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True)
    if max(x.shape[1:]) <= 256:
        U, s, V = torch.linalg.svd((x / (n + EPS)).cpu(), full_matrices=False)
        for a, b, c in COEFFS:
            s = a * s + b * s ** 3 + c * s ** 5
        return ((U * s[:, None, :]) @ V).to(x.device)
    y = x / (n + EPS)
    wide = y.shape[1] <= y.shape[2]
    for a, b, c in COEFFS:
        if wide:
            g = y @ y.mT
            y = a * y + b * (g @ y) + c * (g @ (g @ y))
        else:
            g = y.mT @ y
            y = a * y + b * (y @ g) + c * ((y @ g) @ g)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "mean":
        z = 0
        for k in range(case["K"]):
            z = z + exact_mx4(s["x"][k], case["mode"], s["seed"], 3, k).flatten()
        z = z / case["K"]
        return [z, s["w"].double() + z, z]
    if kind == "product":
        M, N, K = case["M"], case["N"], case["K"]
        wide, at, per, _ = packed_sizes(N, K)
        byte = s["b"][:N * wide].view(N, wide, 1).int()
        four = torch.cat((byte % 16, byte // 16), 2).view(N, -1)
        size = torch.where(four % 8 < 2, (four % 8) / 2, (2 + four % 2) * (1 << (four % 8) // 2) / 4.0).double()
        b = torch.where(four >= 8, -size, size) * ((s["b"][at:at + N * per].view(N, per).long() + 1023 - 127) << 52).view(torch.float64).repeat_interleave(32, 1)
        return exact_mx4(s["x"], "nearest") @ b[:, :K].mT
    if kind == "train":
        x, w, dy, mode = s["x"], s["w"], s["dy"], case["mode"]
        return [exact_mx4(x, "nearest") @ exact_mx4(w, "nearest").mT,
                exact_mx4(dy, mode, s["seed"], 5) @ exact_mx4(w.mT, "nearest").mT,
                exact_mx4(dy.mT, mode, s["seed"], 5) @ exact_mx4(x.mT, "nearest").mT]
    if kind == "ortho":
        g = s["g"].double()
        m = s["mu"] * s["m"].double() + g
        step = s["alpha"] * exact_factor(g + s["mu"] * m if case["nesterov"] else m)
        return [m, step, step, s["w"].double() + step, step]
    return exact_factor(s["x"].double())
