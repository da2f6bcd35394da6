"""The orthogonalised update, no GPU: the reference's own properties and what the entry points refuse."""
import ctypes as C

import numpy as np
import pytest

import matrix_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_1901_03040_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("rows,cols", [(5, 5), (4, 9), (9, 4), (1, 7)])
def test_reference_acts_on_singular_values_alone(rows, cols):
    rng = np.random.default_rng(rows * 10 + cols)
    x = rng.standard_normal((rows, cols))
    U, s, V = np.linalg.svd(x / (np.linalg.norm(x) + 1e-7), full_matrices=False)
    for a, b, c in R.USUAL:
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(R.newton_schulz(x), (U * s) @ V, atol=1e-12)
    assert (s > 0.6).all() and (s < 1.3).all()
    assert np.allclose(R.newton_schulz(x), R.newton_schulz(x.T).T, atol=1e-12)


def test_reference_converges_with_the_classical_coefficients():
    x = np.random.default_rng(0).standard_normal((6, 11))
    q = R.newton_schulz(x, ((15 / 8, -10 / 8, 3 / 8),) * 14)
    assert np.allclose(q @ q.T, np.eye(6), atol=1e-10)
    assert not R.newton_schulz(np.zeros((3, 4)), eps=0.0).any()


def coeffs(values=(3.4445, -4.7750, 2.0315)):
    return (C.c_float * len(values))(*values)


def test_orthogonalize_refusals(B):
    """Addresses that are none: every call is turned down before a launch."""
    f = B.lib().qesgd_orthogonalize
    need = B.qesgd_orthogonalize_workspace_bytes(300, 400, 2)
    assert need > 0 and B.qesgd_orthogonalize_workspace_bytes(30, 40, 2) == 0
    x, o, ws = 0x10000, 0x20000, 0x30000

    def rc(x=x, dtype=0, rows=300, cols=400, n=2, c=coeffs(), steps=1, eps=1e-7, o=o, ws=ws, size=need):
        return f(x, dtype, rows, cols, n, c, steps, eps, o, ws, size, None)

    assert rc(x=None) == B.ERR_NULL and rc(o=None) == B.ERR_NULL and rc(c=None) == B.ERR_NULL
    assert rc(rows=0) == B.ERR_DIM and rc(cols=0) == B.ERR_DIM and rc(n=0) == B.ERR_DIM
    assert rc(rows=(1 << 20) + 1) == B.ERR_DIM and rc(cols=(1 << 20) + 1) == B.ERR_DIM and rc(n=65536) == B.ERR_DIM
    assert rc(rows=1 << 20, cols=1 << 20) == B.ERR_DIM
    assert rc(dtype=3) == B.ERR_DTYPE
    assert rc(steps=0) == B.ERR_STEPS and rc(steps=33, c=coeffs((0.0,) * 99)) == B.ERR_STEPS
    assert rc(c=coeffs((1.0, float("nan"), 1.0))) == B.ERR_COEFF and rc(c=coeffs((float("inf"), 0.0, 1.0))) == B.ERR_COEFF
    assert rc(eps=-1.0) == B.ERR_COEFF and rc(eps=float("nan")) == B.ERR_COEFF
    assert rc(x=x + 4) == B.ERR_ALIGN and rc(o=o + 8) == B.ERR_ALIGN and rc(ws=ws + 16) == B.ERR_ALIGN
    assert rc(ws=None) == B.ERR_WORKSPACE and rc(size=need - 1) == B.ERR_WORKSPACE
    for r, c, n in [(0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 21, 1, 1), (1, 1, 65536)]:
        assert B.qesgd_orthogonalize_workspace_bytes(r, c, n) == 0


def test_update_refusals(B):
    f = B.lib().qesgd_orthogonal_update
    need = B.qesgd_orthogonalize_workspace_bytes(300, 400, 1)
    g, m, s, z, w, u, zs, ws = (0x10000 * i for i in range(1, 9))

    def rc(g=g, m=m, mu=0.9, alpha=-0.1, s=s, z=z, w=w, u=u, zs=zs, size=need):
        return f(g, 300, 400, 1, m, mu, 1, coeffs(), 1, 1e-7, alpha, s, z, w, u, zs, ws, size, None)

    assert rc(g=None) == B.ERR_NULL
    assert rc(s=None, z=None, w=None, u=None, zs=None) == B.ERR_NULL
    assert rc(w=None) == B.ERR_NULL and rc(u=None) == B.ERR_NULL                     # one needs the other
    assert rc(z=None) == B.ERR_NULL and rc(z=None, w=None, u=None) == B.ERR_NULL     # both, and zsum, need z
    assert rc(mu=float("nan")) == B.ERR_COEFF and rc(alpha=float("inf")) == B.ERR_COEFF
    assert rc(m=m + 4) == B.ERR_ALIGN and rc(zs=zs + 4) == B.ERR_ALIGN and rc(u=u + 4) == B.ERR_ALIGN
    assert rc(size=need - 256) == B.ERR_WORKSPACE


def test_binding_refusals(B):
    import torch
    x = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        B.qesgd_orthogonalize(x, 4, 4, 1, ((1.0, 2.0),), 1e-7, x, None, stream=0)
    with pytest.raises(B.QesgdError) as e:
        B.qesgd_orthogonalize(x, 4, 4, 1, R.USUAL, 1e-7, x.to(torch.bfloat16), None, stream=0)
    assert e.value.code == B.ERR_DTYPE
    with pytest.raises(B.QesgdError) as e:
        B.qesgd_orthogonal_update(x.to(torch.float16), 4, 4, 1, None, 0.9, True, R.USUAL, 1e-7, 1.0, x, None, None, None, None, None, stream=0)
    assert e.value.code == B.ERR_DTYPE
