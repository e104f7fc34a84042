"""The gradient of log probabilities where the logits lie far from zero: what moves all logits of a row alike moves no probability, so the error must not grow with it."""
import numpy as np
import pytest

from oracle import decoder as od
from decoder_util import logprob_noise, run_logprob
from rowops_util import EPS24, half_step, storage, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.mark.parametrize("offset", [0.0, 500.0, -3000.0, 4096.0, 16384.0, -2.0 ** 20])
@pytest.mark.parametrize("V", [300, 5001, 50001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_does_not_lose_what_the_row_is_moved_by(torch_mod, dtype, V, offset):
    """Tolerance, relative to p: an argument d = (z - z_id) + lp is off by e (|z - z_id| + |d|), by what lp as stored is off (logprob_noise and e |lp|), a weight further by
    (4 + 3 |d|) e; where the log-sum-exp is the smaller number, at most 4 |lp|, it may take lp's place: e (|lse| + |d|) and its own noise.  The bracket by 6 e of its terms, the
    errors of d and of the entropy; one rounding to the storage type."""
    print("far", dtype, V, offset, flush=True)
    rng = np.random.default_rng(V)
    M = 12
    z = rng.normal(size=(M, V)) * 2
    z[np.arange(M), rng.integers(0, V, M)] += 7
    z = storage(np.round(z * 8) / 8 + offset, dtype)
    zf = values(z, dtype)
    ids = rng.integers(0, V, M)
    ids[:6] = zf[:6].argmax(axis=1)
    gy = (rng.normal(size=(3, M)) / 3).astype(np.float32)
    gy[1:, :3] = 0                                               # the loss alone
    b, o = run_logprob(torch_mod, z, ids, dtype, 0, gy)
    g = np.abs(gy.astype(np.float64))
    want, (y, _, _) = od.logprob_bwd(zf, ids, gy.astype(np.float64)), od.logprob(zf, ids)
    mine = zf[np.arange(M), ids][:, None]
    lpn, nH, nl = logprob_noise(zf, y)
    lp, lse = np.abs(y[0])[:, None], np.abs(y[2])[:, None]
    l = zf - y[2][:, None]
    p, la = np.exp(l), np.abs(l)
    by_lp = EPS24 * (np.abs(zf - mine) + la + lp) + lpn(zf.max(axis=1) - mine[:, 0])[:, None]
    by_lse = EPS24 * (lse + la) + nl[:, None]
    d = np.where(lse <= 4.01 * lp, np.maximum(by_lp, by_lse), by_lp)
    bracket = (g[2] + g[0])[:, None] + g[1][:, None] * (la + np.abs(y[1])[:, None])
    tol = half_step(dtype) * np.abs(want) + p * (bracket * (d + EPS24 * (10 + 3 * la)) + g[1][:, None] * (d + nH[:, None])) + 2 * EPS24 * g[0][:, None] * (np.arange(V) == ids[:, None])
    assert lse.min() >= abs(offset) - 40 and d.max() <= 1e-4
    bad = np.abs(o["gz"] - want) > tol + 2.0 ** -126
    assert not bad.any(), (int(bad.sum()), float((np.abs(o["gz"] - want) / (tol + 2.0 ** -126)).max()))
    if dtype == "f32":                                           # the loss moves with no offset: its gradient's sum over a row is what the roundings leave
        assert (np.abs(o["gz"][:3].sum(axis=1)) <= tol[:3].sum(axis=1)).all()
    b.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_without_weight_and_far_below_the_rest(torch_mod, dtype):
    """A given token of no weight, of the type's lowest value, of one that is 2^15 below the others: its own log probability says nothing of the others' place, the
    log-sum-exp does, to its rounding.  And a row of nothing but the lowest value, whose log-sum-exp holds no log V."""
    rng = np.random.default_rng(4)
    V, M = 700, 6
    z = storage(2048.0 + rng.integers(-8, 9, size=(M, V)) * (16 if dtype == "bf16" else 1), dtype)
    zf = values(z, dtype)
    low = storage(np.full(1, -3.3895313892515355e38 if dtype == "bf16" else -3.4028234663852886e38), dtype)[0]
    z[0, 5], z[1, 5], z[2, 5] = storage(np.array([-np.inf, 0, -2.0 ** 15]), dtype)
    z[1, 5], z[3, :] = low, low                                  # row 3: uniform
    z[4, 7] = storage(np.array([np.inf]), dtype)[0]
    zf = values(z, dtype)
    ids = np.full(M, 5)
    gy = np.tile(np.array([[0.5], [0.25], [0.125]], np.float32), (1, M))
    gy[0, 0] = 0                                                 # of a log probability of -infinity
    b, o = run_logprob(torch_mod, z, ids, dtype, 0, gy)
    fine = [0, 1, 2, 3, 5]
    want, (y, _, _) = od.logprob_bwd(zf[fine], ids[fine], gy[:, fine].astype(np.float64)), od.logprob(zf[fine], ids[fine])
    p = np.exp(np.where(np.isfinite(zf[fine]), zf[fine], -1e300) - y[2][:, None])
    # the log-sum-exp of rows 0, 1, 2, 5 is rounded at 2^11, by 2^-13, the forward's error is no larger; the bracket's terms are below 4 together
    tol = half_step(dtype) * np.abs(want) + p * 4 * (2.0 ** -12) + 4 * EPS24
    want[3] = 0.5 * ((np.arange(V) == 5) - 1 / V) + 0.125 / V    # uniform, its entropy -log p: 64 bits too lose log V beside 3e38
    tol[3] = half_step(dtype) * np.abs(want[3]) + 4 * (40 + 4 * np.log(V)) * EPS24 / V + EPS24
    got = o["gz"][fine]
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    assert np.isnan(o["gz"][4]).any()
    b.close()
