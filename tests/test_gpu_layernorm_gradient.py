"""Layer normalisation in fp32 and over wide rows, and its gradients, against float64 (oracle/rowops.py).

Tolerances: half a step of the storage type (bf16 2^-8, fp32 2^-24 of the value) plus the bounds of fp32 arithmetic that
rowops_util.layernorm_noise derives from the inputs."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, half_step, layernorm_noise, storage, values

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def _case(rows, C, dtype, seed=0, shift=1.5):
    rng = np.random.default_rng(1000 * rows + C + seed)
    x = storage(rng.normal(size=(rows, C)) * rng.uniform(0.5, 2.0, C) + shift, dtype)
    gy, add = storage(rng.normal(size=(rows, C)), dtype), storage(rng.normal(size=(rows, C)), dtype)
    gamma, beta = rng.uniform(0.5, 1.5, C).astype(np.float32), rng.normal(0, 0.1, C).astype(np.float32)
    return x, gy, add, gamma, beta


# rows: one, fewer than a workgroup has wavefronts, ragged, more than one round of the persistent workers
SHAPES = [(1, 8), (1, 768), (3, 64), (7, 512), (9, 520), (77, 768), (8, 1024), (65, 1032), (130, 2048), (5, 2112), (33, 4096), (3, 8192),
          (4500, 64), (4099, 768), (600, 2560), (1100, 1536),
          (1023, 1544), (1024, 1544), (1025, 2048), (2050, 1032), (1030, 2112)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_gradients_match_float64(torch_mod, rows, C, dtype):
    print("rows", rows, "C", C, dtype, flush=True)
    x, gy, add, gamma, beta = _case(rows, C, dtype)
    b = Bench(torch_mod, [x.nbytes] * 5)
    b.put(0, x); b.put(2, gy); b.put(4, add)
    g, sh = b.dev(gamma), b.dev(beta)
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 0, 1, dtype, scale=g.data_ptr(), shift=sh.data_ptr(), eps=EPS)
    need = b.d.backward_workspace(fwd)
    ws, whole = b.workspace(need)
    X, GY = values(x, dtype), values(gy, dtype)
    ngx, ndg, ndb = layernorm_noise(X, GY, gamma, EPS)
    runs = []
    for with_add in (False, True):
        gw, guard = b.guarded(2 * C)
        desc = b.bwd(fwd, 2, gx=3, add=4 if with_add else None, gw=gw, ws=ws)
        assert b.d.backward_kernel(desc) == "gx, gw: layernorm"
        b.d.backward_segment([desc])
        gx = values(b.get(3, x.dtype, x.shape), dtype)
        rgx, rdg, rdb = ro.layernorm_bwd(X, GY, gamma, EPS, values(add, dtype) if with_add else None)
        tol = half_step(dtype) * np.abs(rgx) + 2 * ngx + EPS24 * np.abs(values(add, dtype))
        assert (np.abs(gx - rgx) <= tol).all(), float((np.abs(gx - rgx) / tol).max())
        got = gw.cpu().numpy().astype(np.float64)
        assert (np.abs(got[:C] - rdg) <= ndg).all(), float((np.abs(got[:C] - rdg) / ndg).max())
        assert (np.abs(got[C:] - rdb) <= ndb + 1e-30).all(), float((np.abs(got[C:] - rdb) / ndb).max())
        assert (guard[:64] == 12345.0).all() and (guard[64 + 2 * C:] == 12345.0).all()
        runs.append(got)
        # the same bits again, gx and gw each alone too
        first = b.get(3, x.dtype, x.shape).copy()
        b.d.backward_segment([b.bwd(fwd, 2, gx=3, add=4 if with_add else None)])
        assert np.array_equal(b.get(3, x.dtype, x.shape), first)
    alone, _ = b.guarded(2 * C)
    b.d.backward_segment([b.bwd(fwd, 2, gw=alone, ws=ws)])
    b.d.sync()
    assert np.array_equal(alone.cpu().numpy().astype(np.float64), runs[0]) and np.array_equal(runs[0], runs[1])
    assert (whole[max(need, 256):] == 0x7F).all()
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("rows,C,dtype", [(37, 768, "f32"), (1, 8, "f32"), (5, 2048, "f32"), (13, 1000, "f32"), (2, 8192, "f32"), (1030, 2112, "bf16"),
                                          (3, 8192, "bf16"), (1, 4096, "bf16"), (17000, 64, "f32"), (9, 1032, "f32"),
                                          (1100, 1544, "f32"), (1, 2040, "f32")])
def test_forward_in_fp32_and_over_wide_rows(torch_mod, rows, C, dtype):
    print("rows", rows, "C", C, dtype, flush=True)
    x, _, _, gamma, beta = _case(rows, C, dtype)
    b = Bench(torch_mod, [x.nbytes] * 2)
    b.put(0, x)
    g, sh = b.dev(gamma), b.dev(beta)
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 0, 1, dtype, scale=g.data_ptr(), shift=sh.data_ptr(), eps=EPS)
    assert b.d.layer_kernel(fwd) == "layernorm " + dtype
    b.d.recompute_segment([fwd])
    got = values(b.get(1, x.dtype, x.shape), dtype)
    X = values(x, dtype)
    ref = ro.layernorm(X, gamma, beta, EPS)
    c = X - X.mean(axis=1, keepdims=True)
    r = 1 / np.sqrt((c * c).mean(axis=1, keepdims=True) + EPS)
    noise = 40 * EPS24 * (np.abs(X).max(axis=1, keepdims=True) * r + np.abs(c * r)) * gamma + 2 * EPS24 * np.abs(beta)
    assert (np.abs(got - ref) <= half_step(dtype) * np.abs(ref) + noise).all()
    assert b.untouched()
    b.close()


def test_a_row_of_equal_values_has_no_gradient_beyond_eps_and_a_bad_row_stays_alone(torch_mod):
    rows, C = 40, 256
    x, gy, _, gamma, beta = _case(rows, C, "f32")
    x[3] = 2.5                                               # variance 0: xh = 0, gx = (g - mean g) / sqrt(eps)
    x[7, 11] = np.inf
    gy[9, 5] = np.nan
    b = Bench(torch_mod, [x.nbytes] * 4)
    b.put(0, x); b.put(2, gy)
    g, sh = b.dev(gamma), b.dev(beta)
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 0, 1, "f32", scale=g.data_ptr(), shift=sh.data_ptr(), eps=EPS)
    b.d.backward_segment([b.bwd(fwd, 2, gx=3)])
    gx = b.get(3, np.float32, x.shape).astype(np.float64)
    G = gy[3].astype(np.float64) * gamma
    assert np.allclose(gx[3], (G - G.mean()) / np.sqrt(EPS), rtol=1e-5, atol=40 * EPS24 * np.abs(G).max() / np.sqrt(EPS))
    assert np.isnan(gx[7]).all() and np.isnan(gx[9]).all()
    good = [r for r in range(rows) if r not in (7, 9)]
    assert np.isfinite(gx[good]).all()
    b.close()


def test_gradients_agree_with_differences_of_the_forward_kernel(torch_mod):
    """fp32: L = sum(y * gy); the forward kernel at x +- h against the gradient kernel.  The difference is off by h^2 terms and
    by the forward's rounding over h: 1e-2 of the largest gradient at h = 2^-6."""
    rows, C, h = 2, 64, 2.0 ** -6
    x, gy, _, gamma, beta = _case(rows, C, "f32", shift=0.25)
    b = Bench(torch_mod, [x.nbytes] * 4)
    b.put(2, gy)
    g, sh = b.dev(gamma), b.dev(beta)
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 0, 1, "f32", scale=g.data_ptr(), shift=sh.data_ptr(), eps=EPS)

    def loss(a):
        b.put(0, a)
        b.d.recompute_segment([fwd])
        return float((b.get(1, np.float32, x.shape).astype(np.float64) * gy).sum())
    at = [(0, 0), (0, 31), (1, 8), (1, 63)]
    diff = []
    for (i, j) in at:
        hi, lo = x.copy(), x.copy()
        hi[i, j] += h
        lo[i, j] -= h
        diff.append((loss(hi) - loss(lo)) / (float(hi[i, j]) - float(lo[i, j])))
    b.put(0, x)
    b.d.backward_segment([b.bwd(fwd, 2, gx=3)])
    gx = b.get(3, np.float32, x.shape)
    assert np.abs(np.array(diff) - [gx[i, j] for (i, j) in at]).max() <= 1e-2 * np.abs(gx).max()
    b.close()


def test_refusals(torch_mod):
    rows, C = 16, 64
    nb = rows * C * 2
    b = Bench(torch_mod, [nb, nb, nb, nb, nb, nb // 2, rows * 2112 * 2, rows * 2112 * 2, rows * 2056 * 2, rows * 2056 * 2, rows * 8256 * 2, rows * 8256 * 2])
    dl = b.dl
    one = torch_mod.ones(9000, device="cuda:0")
    kw = dict(scale=one.data_ptr(), shift=one.data_ptr(), eps=EPS)
    fwd = b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 1, **kw)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, _ = b.guarded(2 * C)
    ok = dict(gx=3, gw=gw, ws=ws)

    def refused(desc, status=dl.ERR_INVALID):
        with pytest.raises(dl.DeltaError) as e:
            b.d.backward_segment([desc])
        assert e.value.status == status
        with pytest.raises(dl.DeltaError):
            b.d.backward_kernel(desc) if status == dl.ERR_INVALID else b.d.backward_segment([desc])
    refused(b.bwd(fwd, 2))                                                       # nothing to compute
    refused(b.bwd(fwd, 2, gw=gw, ws=ws, add=4))                                  # gx_add without gx
    refused(b.bwd(fwd, 2, **{**ok, "gx": 0}))                                    # gx over x, gy, a tensor of another size
    refused(b.bwd(fwd, 2, **{**ok, "gx": 2}))
    refused(b.bwd(fwd, 2, **{**ok, "gx": 5}))
    refused(b.bwd(fwd, 2, add=3, **ok))                                          # gx_add over gx
    refused(b.bwd(fwd, 2, add=99, **ok))
    refused(b.bwd(fwd, 2, gpre=4, **ok))
    refused(b.bwd(fwd, 2, mask_gx=1, **ok))
    refused(b.bwd(fwd, 2, gy_masked=1, **ok))
    refused(b.bwd(fwd, 2, gx=3, gw=gw))                                          # no workspace
    refused(b.bwd(fwd, 2, **ok, workspace_bytes=ws.numel() - 256))
    refused(b.bwd(fwd, 2, gx=3, gw=gw, ws=ws[16:]))                              # misaligned
    refused(b.bwd(fwd, 2, gx=3, gw=gw[1:], ws=ws))
    refused(b.bwd(b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 1, scale=one.data_ptr() + 4, shift=one.data_ptr(), eps=EPS), 2, **ok))
    refused(b.bwd(b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 1, scale=one.data_ptr(), shift=one.data_ptr(), eps=-1.0), 2, **ok))
    refused(b.bwd(b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 1, pack=3, **kw), 2, **ok))
    refused(b.bwd(b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 1, pack=dl.PACK_INT8, **kw), 2, **ok))     # x is no checkpoint
    for c, x, y in ((2056, 8, 9), (8256, 10, 11)):                               # channels
        with pytest.raises(dl.DeltaError):
            b.d.recompute_segment([b.layer(dl.OP_LAYERNORM, rows, c, c, x, y, **kw)])
    b.d.recompute_segment([b.layer(dl.OP_LAYERNORM, rows, 2112, 2112, 6, 7, **kw)])
    b.d.release(2, dl.EV_FREE)
    refused(b.bwd(fwd, 2, **ok), dl.ERR_STATE)                                   # gy is gone
    b.close()
