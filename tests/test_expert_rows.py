"""Rows of fp32 beside results of 16 bits, what needs no GPU: refusals before a launch is attempted (fake device addresses)."""
import pytest

from test_experts import COMBINE, COMBINE_BACK, VECTOR, B, call  # noqa: F401


@pytest.mark.parametrize("dtype", [0x100, 0x101, 0x102])
def test_refusals_of_the_weighted_sum(B, dtype):  # noqa: F811
    for name, spec in (("qesgd_combine", COMBINE), ("qesgd_combine_backward", COMBINE_BACK)):
        assert call(B, name, spec, dtype=dtype + 3) == B.ERR_DTYPE
        assert call(B, name, spec, dtype=dtype | 0x200) == B.ERR_DTYPE
        assert call(B, name, spec, dtype=dtype, rows=spec["rows"] + 2) == B.ERR_ALIGN          # of fp32
        assert call(B, name, spec, dtype=dtype, ld=7) == B.ERR_STRIDE
        assert call(B, name, spec, dtype=dtype, rows=None) == B.ERR_NULL
    assert call(B, "qesgd_combine", COMBINE, dtype=dtype, out=COMBINE["out"] + 1) == B.ERR_ALIGN
    assert call(B, "qesgd_combine_backward", COMBINE_BACK, dtype=dtype, drows=COMBINE_BACK["drows"] + 1) == B.ERR_ALIGN


@pytest.mark.parametrize("dtype", [0x101, 0x102])
def test_gradients_do_not_take_the_place_of_rows_of_another_type(B, dtype):  # noqa: F811
    assert call(B, "qesgd_combine_backward", COMBINE_BACK, dtype=dtype, drows=COMBINE_BACK["rows"]) == B.ERR_DTYPE


@pytest.mark.parametrize("dtype", [0x100, 0x101, 0x102])
def test_refusals_of_single_rows(B, dtype):  # noqa: F811
    name = "qesgd_mx4_vector_product"
    assert call(B, name, VECTOR, dtype=dtype + 3) == B.ERR_DTYPE
    assert call(B, name, VECTOR, dtype=dtype, y=VECTOR["y"] + 2) == B.ERR_ALIGN                # of fp32
    assert call(B, name, VECTOR, dtype=dtype, x=VECTOR["x"] + 1) == B.ERR_ALIGN
    assert call(B, name, VECTOR, dtype=dtype, ldy=7) == B.ERR_STRIDE
