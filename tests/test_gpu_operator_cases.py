"""perf/operators.py: a case's outputs come laid out alike from the plain form, from the library's calls and from the definition in 64 bits, for each
operator and direction, also where a case has one output."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

SMALL = [dict(kind="layernorm", do="backward", dtype="bf16", N=2, S=9, C=64, add=True, pack=""),
         dict(kind="layernorm", do="both", dtype="f32", N=1, S=5, C=72, add=False, pack="int8"),
         dict(kind="pack", fmt="e4m3", dtype="f32", N=1, S=7, C=40),
         dict(kind="linear", fmt="int8", N=1, S=70, Cin=64, Cout=128),
         dict(kind="embedding", do="forward", dtype="bf16", N=2, S=11, V=30, C=64),
         dict(kind="embedding", do="backward", dtype="bf16", N=2, S=11, V=30, C=64),
         dict(kind="embedding", do="both", dtype="f32", N=1, S=9, V=30, C=64)]


@pytest.fixture(scope="module")
def operators():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("operators_cases", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _layout(v):
    return [_layout(x) for x in v] if isinstance(v, (list, tuple)) else tuple(v.shape)


@pytest.mark.parametrize("case", SMALL, ids=lambda c: "%s %s %s" % (c["kind"], c.get("do", ""), c.get("dtype", "")))
def test_outputs_are_laid_out_alike(operators, case):
    import torch
    operators.own = False
    plain = operators.run(operators.prepare(dict(case), 3))
    exact = operators.exact(dict(case), 3)
    operators.own = True
    try:
        state = operators.prepare(dict(case), 3)
        mine = operators.run(state)
        torch.cuda.synchronize()
    finally:
        operators.own = False
    assert _layout(mine) == _layout(plain) == _layout(exact)
    flat = lambda v: [v] if isinstance(v, torch.Tensor) else list(v)           # noqa: E731
    assert [x.dtype for x in flat(mine)] == [x.dtype for x in flat(plain)]
    state.d.close()
