"""Root-mean-square normalisation's gradients where a row and its gradient are both large, or both small: what they are made of, r, s r and g, is far inside fp32, their products
g s are not.  eps = 0, which is allowed; rows up to 2^63 / sqrt(C)."""
import numpy as np
import pytest

from oracle import decoder as od
from decoder_util import TINY, rmsnorm_noise, run_rmsnorm
from rowops_util import EPS24, half_step, storage, values

pytestmark = pytest.mark.gpu

SIZES = [(0, 0), (55, 80), (-60, -95), (55, -60), (-60, 50), (30, 100), (-62, 0), (55, 71)]        # of a row's values and its gradients', powers of two


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


# a launch for both gradients (up to 128 rows of 16384 values together, channels by 32), and others: a wavefront to a row, a workgroup to a row
@pytest.mark.parametrize("M,C", [(8, 32), (8, 64), (8, 2048), (16, 1024), (128, 128), (2, 8192), (8, 40), (129, 64), (9, 2048), (9, 4096)])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_large_and_small_rows(torch_mod, dtype, add, M, C):
    """Tolerance: half a step of the storage type and decoder_util.rmsnorm_noise, relative to r G of each row; numbers below 2^-126 may be held as zero.  dgamma: the rows' terms,
    sums from 2^-95 to 2^100, by the sum of their magnitudes."""
    print("far sizes", dtype, add, M, C, flush=True)
    rng = np.random.default_rng(M * 31 + C)
    by = np.exp2(np.array([SIZES[m % len(SIZES)] for m in range(M)], float))
    x, gy = rng.normal(size=(M, C)) * by[:, :1], rng.normal(size=(M, C)) * by[:, 1:]
    gamma, w = rng.uniform(0.5, 1.5, C).astype(np.float32), rng.normal(size=(M, C))
    b, o = run_rmsnorm(torch_mod, x, None, gamma, 0.0, dtype, 0, gy, w if add else None)
    v = lambda a: values(storage(a, dtype), dtype)                                   # noqa: E731
    s, g = v(x), v(gy)
    fwd, ngx, ndg = rmsnorm_noise(s, g, gamma, 0.0)
    want = od.rmsnorm(s, gamma, 0.0)
    assert (np.abs(values(o["y"], dtype) - want) <= (half_step(dtype) + fwd) * np.abs(want) + TINY).all()
    gx, dg = od.rmsnorm_bwd(s, g, gamma, 0.0, v(w) if add else None)
    got = values(o["gx"], dtype)
    tol = (half_step(dtype) + EPS24) * np.abs(gx) + ngx + (2 * EPS24 * np.abs(v(w)) if add else 0) + TINY
    bad = ~(np.abs(got - gx) <= tol)
    assert not bad.any(), ("rows of sizes", sorted({SIZES[m % len(SIZES)] for m in np.flatnonzero(bad.any(axis=1))}))
    assert (np.abs(o["gw"] - dg) <= ndg + TINY).all()
    b.close()
