"""What the refusals of the calls for layers of experts say: the argument that is wrong is one of the call's."""
import pytest

from test_experts import ROUTE, ROUTE_BACK, B, call  # noqa: F401


@pytest.mark.parametrize("name,spec", [("qesgd_route", ROUTE), ("qesgd_route_backward", ROUTE_BACK)])
def test_gate_kind(B, name, spec):  # noqa: F811
    code = call(B, name, spec, kind=2)
    assert code == B.ERR_MODE and "gate_kind" in B.strerror(code)


@pytest.mark.parametrize("field,value,word", [("T", 0, "tokens"), ("ld", 7, "row apart"), ("logits", 0x10002, "element")])
def test_sizes_strides_and_alignment(B, field, value, word):  # noqa: F811
    assert word in B.strerror(call(B, "qesgd_route", ROUTE, **{field: value}))
