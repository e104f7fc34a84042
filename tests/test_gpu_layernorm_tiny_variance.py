"""Layer normalisation's gradients where var + eps lies near and below the smallest normal fp32 number (eps = 0, which is allowed): 1 / sqrt(var + eps) is
some 2^60 to 2^66 and finite, its square is not.  Rows of pairs (a, -a), a = 2^-k or 2^-k / 2: their mean is exactly zero in any order, their squares'
sum exact, and every one exact in both checkpoint formats.

Tolerance: half a step of the storage type and rowops_util.layernorm_noise, and what the rounding of a subnormal variance to a multiple of 2^-149
adds: var off by 2^-150 is d = 2^-151 / var of 1 / sqrt(var) and of xh, which with G = max|g|, H = max|xh| is at most d r G (1 + 3 H^2 + 1) of gx
(its three terms, the last with xh twice and r) and d |gy| |xh| of dgamma."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, half_step, layernorm_noise, storage, values

pytestmark = pytest.mark.gpu

K = [0, 30, 58, 59, 60, 61, 62, 63, 64, 65]


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


# a wavefront to a row (one, two and four pieces of 512 channels) and a workgroup to a row; few rows and more than a round of the workers
@pytest.mark.parametrize("rows,C", [(10, 64), (10, 768), (10, 1536), (10, 4096), (4200, 64), (1100, 2048)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["", "int8", "e4m3"])
def test_gradients_are_finite_and_right(torch_mod, rows, C, dtype, fmt):
    print("rows", rows, "C", C, dtype, fmt, flush=True)
    rng = np.random.default_rng(rows + C)
    a = rng.choice([0.5, 1.0], (rows, C // 2)) * np.exp2(-np.array(K, float))[np.arange(rows) % len(K)][:, None]
    x = storage(np.stack([a, -a], axis=2).reshape(rows, C), dtype)
    gy, add = storage(rng.normal(size=(rows, C)), dtype), storage(rng.normal(size=(rows, C)), dtype)
    gamma = rng.uniform(0.5, 1.5, C).astype(np.float32)
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C)] + [x.nbytes] * 4)
    b.put(0, x); b.put(2, gy); b.put(4, add)
    g = b.dev(gamma)
    pack = {"": 0, "int8": b.dl.PACK_INT8, "e4m3": b.dl.PACK_E4M3}[fmt]
    if fmt:
        b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, C, C, 0, 1, dtype, pack=pack)])
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 1 if fmt else 0, 5, dtype, scale=g.data_ptr(), shift=g.data_ptr(), eps=0.0, pack=pack)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    X, GY, ADD = values(x, dtype), values(gy, dtype), values(add, dtype)
    var = (X * X).mean(axis=1, keepdims=True)
    r = 1 / np.sqrt(var)
    d = np.where(var < 2.0 ** -126, 2.0 ** -151 / var, 0)
    G, H = np.abs(GY * gamma).max(axis=1, keepdims=True), np.abs(X * r).max(axis=1, keepdims=True)
    ngx, ndg, ndb = layernorm_noise(X, GY, gamma, 0.0)
    ngx = 2 * ngx + d * r * G * (2 + 3 * H * H)
    ndg = ndg + (d * np.abs(GY) * np.abs(X * r)).sum(axis=0)
    for with_add in (False, True):
        gw, _ = b.guarded(2 * C)
        b.d.backward_segment([b.bwd(fwd, 2, gx=3, add=4 if with_add else None, gw=gw, ws=ws)])
        gx = values(b.get(3, x.dtype, x.shape), dtype)
        want, rdg, rdb = ro.layernorm_bwd(X, GY, gamma, 0.0, ADD if with_add else None)
        bad = ~np.isfinite(gx).all(axis=1)
        assert not bad.any(), ("rows that are not finite: exponents", sorted({K[i % len(K)] for i in np.flatnonzero(bad)}))
        assert (np.abs(gx - want) <= half_step(dtype) * np.abs(want) + ngx + EPS24 * np.abs(ADD)).all()
        got = gw.cpu().numpy().astype(np.float64)
        assert (np.abs(got[:C] - rdg) <= ndg).all() and (np.abs(got[C:] - rdb) <= ndb + 1e-30).all()
    b.close()
