"""perf/more_operators.py: a case's outputs come laid out alike from the plain form, from the library's calls and from the definition in 64 bits, for each operator and
direction, and the library's are near the definition's."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

SMALL = [dict(kind="attention", do="both", seqs=4, longest=50, even=False, tail=3, heads=4, kv=2, D=64, causal=True),
         dict(kind="attention", do="forward", seqs=1, longest=9, even=True, tail=0, heads=2, kv=1, D=128, causal=False),
         dict(kind="rmsnorm", do="both", dtype="bf16", M=9, C=72, res=True, add=True, pack="int8"),
         dict(kind="rmsnorm", do="forward", dtype="f32", M=5, C=64, res=False, add=False, pack=""),
         dict(kind="rotary", do="both", dtype="f32", M=7, axes=3, heads=3, rest=1, D=32, pairs=False),
         dict(kind="rotary", do="forward", dtype="bf16", M=1, axes=1, heads=1, rest=0, D=80, pairs=True),
         dict(kind="logprob", do="both", dtype="bf16", M=12, V=130, K=5, masked=1),
         dict(kind="logprob", do="forward", dtype="f32", M=2, V=101, K=0, masked=0)]


@pytest.fixture(scope="module")
def operators():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "more_operators.py")
    spec = importlib.util.spec_from_file_location("more_operators_cases", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("case", SMALL, ids=lambda c: "%s %s %s" % (c["kind"], c["do"], c.get("dtype", "")))
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
    assert len(mine) == len(plain) == len(exact)
    for a, b, e in zip(mine, plain, exact):
        assert a.shape == b.shape and a.dtype == b.dtype and (e is None or e.shape == a.shape)
        if e is None:
            assert torch.equal(a, b)
        else:                                                    # roundings to bf16 and E4M3's or int8's steps where one flips: 2 % of the outputs' size; fp32: 2^-15
            assert (a.double() - e).norm() <= (2.0 ** -15 if a.dtype == torch.float32 else 0.02) * e.norm()
    state.d.close()
