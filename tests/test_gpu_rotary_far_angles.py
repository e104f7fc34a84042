"""Rotary positions of up to 2^31 radians: sine and cosine as exact as those near zero.  Pairs of (1, 0) in fp32 come out as (cos, sin) themselves."""
import numpy as np
import pytest

from oracle import decoder as od
from rowops_util import EPS24, Bench

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def places(rng, what, M, half):
    """(positions [M, A], frequencies [A, half]) whose angles reach 2^31 but no further."""
    if what == "near":
        return rng.integers(-3, 4, (M, 2)), rng.uniform(0, 0.5, (2, half))
    if what == "one axis":
        return rng.integers(2 ** 30, 2 ** 31, (M, 1)) * rng.choice([-1, 1], (M, 1)), np.where(np.arange(half) % 2, 1.0, rng.uniform(0.5, 1.0, half))[None]
    if what == "three axes":
        return rng.integers(-2 ** 29, 2 ** 29, (M, 3)), rng.uniform(0.5, 1.0, (3, half))
    if what == "eight axes":
        return rng.integers(2 ** 27, 2 ** 28, (M, 8)), rng.uniform(0.5, 1.0, (8, half))
    # positions beyond 2^53, which 64 bits of floating point do not hold
    return rng.integers(2 ** 60, 2 ** 62, (M, 2)) * np.array([[1, -1]]), rng.uniform(0.5, 1.0, (2, half)) * 2.0 ** -32


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("what", ["near", "one axis", "three axes", "eight axes", "far positions"])
def test_sine_and_cosine(torch_mod, what, pairs):
    """With an exact angle: the fraction of a turn to fp32, times 2 pi and 2 pi's own rounding, 2.5 e of an eighth of a turn (0.79); the polynomials' last two
    operations, 2 e, and 0.2 e for what is in them: at most 3.5 e, absolute, of sine and cosine."""
    import paper_2203_15980_amd as dl
    print("angles", what, pairs, flush=True)
    rng = np.random.default_rng(len(what))
    M, D = 500, 128
    pos, freq = places(rng, what, M, D // 2)
    freq = freq.astype(np.float32)
    theta = od.angles(pos, freq)
    assert np.abs(theta).max() < 2.0 ** 31 and (what == "near" or np.abs(theta).max() > 2.0 ** 28)
    one = np.zeros((M, D), np.float32)
    if pairs:
        one[:, ::2] = 1
    else:
        one[:, :D // 2] = 1
    b = Bench(torch_mod, [M * D * 4, pos.size * 8, M * D * 4, M * D * 4, M * D * 4])
    b.put(0, one)
    b.put(1, pos.astype(np.int64))
    b.put(3, one)
    f = b.dev(freq)
    L = b.layer(dl.OP_ROTARY, M, D, D, 0, 2, "f32", res=1, y2=dl.NO_TENSOR, y3=dl.NO_TENSOR, R=1, S=0, scale=f.data_ptr(), flags=dl.ROTARY_PAIRS if pairs else 0)
    b.d.recompute_segment([L])
    b.d.backward_segment([b.bwd(L, 3, gx=4)])
    for t, sign in ((2, 1), (4, -1)):
        got = b.get(t, np.float32, (M, D)).astype(np.float64)
        c, s = (got[:, ::2], got[:, 1::2]) if pairs else (got[:, :D // 2], got[:, D // 2:])
        off = max(np.abs(c - np.cos(theta).astype(np.float64)).max(), np.abs(s - sign * np.sin(theta).astype(np.float64)).max())
        assert off <= 3.5 * EPS24, off / EPS24
    b.close()
