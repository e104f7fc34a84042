"""The decoder operators against float64 on the operands that the GPU reads, each at sizes and masks where it can go wrong.  Tolerances: decoder_util."""
import numpy as np
import pytest

from oracle import decoder as od, rowops as ro
from decoder_util import check_attention, logprob_noise, rmsnorm_noise, run_attention, run_logprob, run_rmsnorm
from rowops_util import EPS24, Bench, half_step, storage, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def near(got, ref, tol):
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:3].tolist(), float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max()))


# ------------------------------------------------------------------ root-mean-square normalisation

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,C,res,add,pack", [(1, 8, False, False, 0), (3, 40, True, True, 1), (77, 768, True, True, 2), (5, 1000, False, True, 1), (130, 512, True, False, 0),
                                              (9, 2048, True, True, 1), (9, 2056, True, True, 2), (4, 8192, True, True, 1), (2100, 64, False, False, 2), (7, 4104, False, False, 0),
                                              (3, 1544, True, False, 2),
                                              (128, 96, True, True, 1), (16, 1024, False, True, 0), (129, 64, True, True, 0), (2, 8192, False, False, 1)])
def test_rmsnorm(torch_mod, dtype, M, C, res, add, pack):
    print("rmsnorm", dtype, M, C, res, add, pack, flush=True)
    import paper_2203_15980_amd as dl
    rng = np.random.default_rng(M * 10007 + C)
    eps = 1e-6
    x, r = rng.normal(size=(M, C)) * 2, rng.normal(size=(M, C)) * 3
    x[0] *= 1e-4
    gamma, gy, w = rng.uniform(0.5, 1.5, C).astype(np.float32), rng.normal(size=(M, C)), rng.normal(size=(M, C))
    b, o = run_rmsnorm(torch_mod, x, r if res else None, gamma, eps, dtype, pack, gy, w if add else None)
    h = half_step(dtype)
    v = lambda a: values(storage(a, dtype), dtype)                                   # noqa: E731
    s = values(o["sum"], dtype)
    if res:
        want = v(x) + v(r)
        near(s, want, (h + EPS24) * np.abs(want))
    fwd, ngx, ndg = rmsnorm_noise(s, v(gy), gamma, eps)
    want = od.rmsnorm(s, gamma, eps)
    y = values(o["y"], dtype)
    near(y, want, (h + fwd) * np.abs(want))
    if pack:                                                     # the bits that the checkpoint operator makes of the stored y
        fmt = "int8" if pack == dl.PACK_INT8 else "e4m3"
        pay, sc = ro.pack(y, fmt)
        got_pay, got_sc = ro.split_packed(o["held"], M, C)
        assert np.array_equal(sc, got_sc)
        assert np.array_equal(ro.unpack(got_pay, got_sc, fmt), ro.unpack(pay, sc, fmt))
    gx, dg = od.rmsnorm_bwd(s, v(gy), gamma, eps, v(w) if add else None)
    near(values(o["gx"], dtype), gx, (h + EPS24) * np.abs(gx) + ngx + (2 * EPS24 * np.abs(v(w)) if add else 0))
    near(o["gw"], dg, ndg)
    assert b.untouched()
    # each gradient by itself has the same bits
    b1, o1 = run_rmsnorm(torch_mod, x, r if res else None, gamma, eps, dtype, pack, gy, w if add else None, gw=False)
    assert np.array_equal(o1["gx"], o["gx"])
    b2, o2 = run_rmsnorm(torch_mod, x, r if res else None, gamma, eps, dtype, pack, gy, None, gx=False)
    assert np.array_equal(o2["gw"], o["gw"])
    for k in (b, b1, b2):
        k.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rmsnorm_of_tiny_zero_and_bad_rows(torch_mod, dtype):
    import paper_2203_15980_amd as dl
    rng = np.random.default_rng(5)
    M, C = 9, 264
    x = rng.normal(size=(M, C))
    x[1] *= 1e-25                                                # the squares are lost, eps is what is left: y = s / sqrt(eps)
    x[2] = 0
    x[3, 7], x[4, 100] = np.inf, np.nan
    x[5] *= 1e15
    gamma, gy = np.ones(C, np.float32), rng.normal(size=(M, C))
    b, o = run_rmsnorm(torch_mod, x, None, gamma, 1e-30, dtype, dl.PACK_INT8, gy)
    s, g, y, gx = values(o["sum"], dtype), values(storage(gy, dtype), dtype), values(o["y"], dtype), values(o["gx"], dtype)
    fine = [0, 1, 2, 5, 6, 7, 8]
    want, _ = od.rmsnorm_bwd(s[fine], g[fine], gamma, 1e-30)
    fwd, ngx, _ = rmsnorm_noise(s[fine], g[fine], gamma, 1e-30)
    near(y[fine], od.rmsnorm(s[fine], gamma, 1e-30), (half_step(dtype) + fwd) * np.abs(od.rmsnorm(s[fine], gamma, 1e-30)) + 1e-37)
    near(gx[fine], want, (half_step(dtype) + EPS24) * np.abs(want) + ngx + 1e-37)
    assert np.isnan(y[3, 7]) and (y[3, :7] == 0).all() and np.isnan(y[4]).all() and np.isnan(gx[4]).all()
    _, sc = ro.split_packed(o["held"], M, C)
    assert (sc[4] == 255).all() and sc[3, 0] == 255 and (sc[3, 1:] != 255).all() and (sc[fine] != 255).all()
    b.close()


# ------------------------------------------------------------------ rotary positions

def run_rotary(torch, x, pos, freq, heads, rest, D, pairs, dtype, gy=None):
    import paper_2203_15980_amd as dl
    M, W = x.shape
    es = 4 if dtype == "f32" else 2
    t = np.float32 if dtype == "f32" else np.uint16
    b = Bench(torch, [M * W * es, pos.size * 8, M * W * es, M * W * es, M * W * es])
    b.put(0, storage(x, dtype))
    b.put(1, np.asarray(pos, np.int64))
    f = b.dev(np.asarray(freq, np.float32))
    L = b.layer(dl.OP_ROTARY, M, W, W, 0, 2, dtype, res=1, y2=dl.NO_TENSOR, y3=dl.NO_TENSOR, R=heads, S=rest, scale=f.data_ptr(), flags=dl.ROTARY_PAIRS if pairs else 0)
    b.d.recompute_segment([L])
    y = values(b.get(2, t, (M, W)), dtype)
    gx = None
    if gy is not None:
        b.put(3, storage(gy, dtype))
        b.d.release(0, dl.EV_EVICT)                              # the gradient does not read x
        b.d.backward_segment([b.bwd(L, 3, gx=4)])
        gx = values(b.get(4, t, (M, W)), dtype)
    return b, y, gx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("M,heads,rest,D,axes,far", [(1, 1, 0, 16, 1, 0), (5, 3, 2, 64, 1, 100000), (77, 24, 12, 64, 1, 0), (33, 5, 1, 80, 3, 700), (9, 2, 0, 256, 2, 2 ** 24),
                                                     (130, 10, 2, 128, 8, 50), (4, 3, 3, 96, 1, 2 ** 31 - 9)])
def test_rotary(torch_mod, dtype, pairs, M, heads, rest, D, axes, far):
    print("rotary", dtype, pairs, M, heads, rest, D, axes, far, flush=True)
    rng = np.random.default_rng(M + D)
    W = (heads + rest) * D
    x, gy = rng.normal(size=(M, W)), rng.normal(size=(M, W))
    pos = far + rng.integers(-50, 50, size=(M, axes))
    freq = np.zeros((axes, D // 2), np.float32)
    i = np.arange(D // 2)
    freq[i % axes, i] = 10000.0 ** (-2.0 * i / D)
    if axes == 8:
        freq += rng.normal(size=freq.shape).astype(np.float32) * 0.01              # angles of all axes in each pair
    theta = od.angles(pos, freq)
    b, y, gx = run_rotary(torch_mod, x, pos, freq, heads, rest, D, pairs, dtype, gy)
    v = lambda a: values(storage(a, dtype), dtype)                                   # noqa: E731
    # an angle is off by 2^-51 of it (products and sums in 64 bits, 8 axes at most) and 3 roundings of an eighth of a turn; sine and cosine by 3 more
    off = 2.0 ** -50 * float(np.abs(theta).max()) + 8 * EPS24
    for got, src, sign in ((y, v(x), 1), (gx, v(gy), -1)):
        want = od.rotary(src, sign * theta, heads, D, pairs)
        size = np.abs(src).max(axis=1, keepdims=True) * 2
        near(got[:, :heads * D], want[:, :heads * D], (half_step(dtype) * np.abs(want) + off * size)[:, :heads * D])
        assert np.array_equal(got[:, heads * D:], src[:, heads * D:])
    assert b.untouched()
    b.close()


# ------------------------------------------------------------------ attention

def offsets(lens, before=0):
    return np.concatenate([[before], before + np.cumsum(lens)]).astype(np.int64)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,before,behind,heads,kv,D", [
    ([1], 0, 0, 1, 1, 64), ([77], 0, 0, 12, 12, 64), ([64], 0, 0, 2, 1, 128), ([65, 0, 1, 127, 128, 129], 0, 0, 4, 2, 64), ([31, 33, 63, 2], 5, 40, 3, 3, 128),
    ([300], 0, 130, 8, 1, 128), ([0, 0, 200, 0], 0, 0, 6, 2, 64), ([257, 255], 1, 1, 4, 4, 128), ([700], 0, 0, 2, 2, 64), ([513, 40], 0, 3, 16, 2, 64), ([0], 9, 8, 2, 1, 64), ([20], 0, 0, 256, 64, 64), ([9, 8], 0, 2, 64, 8, 128)])
def test_attention(torch_mod, causal, lens, before, behind, heads, kv, D):
    print("attention", causal, lens, before, behind, heads, kv, D, flush=True)
    rng = np.random.default_rng(sum(lens) + D + heads)
    off = offsets(lens, before)
    M, W = int(off[-1]) + behind, (heads + 2 * kv) * D
    x = storage(rng.normal(size=(M, W)) * np.where(np.arange(W) < (heads + kv) * D, 1.3, 1.0), "bf16")
    gy = storage(rng.normal(size=(M, heads * D)), "bf16")
    x[:before], gy[:before], x[off[-1]:], gy[off[-1]:] = 0x7FC0, 0x7FC0, 0x7FC0, 0x7FC0          # NaN in rows of no sequence
    b, o = run_attention(torch_mod, x, off, heads, kv, D, causal, gy)
    alone = np.r_[0:before, off[-1]:M].astype(int)
    assert not o["y"][alone].any() and not o["lse"][:, alone].any() and not o["gx"][alone].any()
    xf, gf = values(x, "bf16"), values(gy, "bf16")
    xf[alone], gf[alone] = 0, 0
    ref = od.attention(xf, off, heads, kv, D, causal, gf)
    check_attention(o, ref, heads, D, max(lens))
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("n,most", [(200, 9), (5000, 2)])
def test_attention_of_many_sequences(torch_mod, n, most):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, most + 1, n)
    off = offsets(lens)
    M, heads, kv, D = int(off[-1]) + 3, 2, 1, 64
    x, gy = storage(rng.normal(size=(M, 4 * D)), "bf16"), storage(rng.normal(size=(M, 2 * D)), "bf16")
    b, o = run_attention(torch_mod, x, off, heads, kv, D, True, gy)
    check_attention(o, od.attention(values(x, "bf16"), off, heads, kv, D, True, values(gy, "bf16")), heads, D, most)
    b.close()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("seqs,most,heads,kv,D", [(60, 300, 8, 2, 64), (62, 150, 8, 8, 128), (63, 150, 8, 8, 128), (3, 600, 12, 4, 64), (2, 500, 12, 12, 128), (100, 60, 16, 2, 64), (1, 1100, 12, 3, 64), (1, 2200, 16, 4, 128)])
def test_attention_where_the_chip_is_full(torch_mod, causal, seqs, most, heads, kv, D):
    """Launches of one and two groups of wavefronts to a tile, of both gradients apart, and of more sequences than a wavefront has lanes."""
    print("attention", causal, seqs, most, heads, kv, D, flush=True)
    rng = np.random.default_rng(seqs + most)
    lens = rng.integers(0, most + 1, seqs)
    lens[-1] = most
    off = offsets(lens, 3)
    M = int(off[-1]) + 70
    x, gy = storage(rng.normal(size=(M, (heads + 2 * kv) * D)), "bf16"), storage(rng.normal(size=(M, heads * D)), "bf16")
    b, o = run_attention(torch_mod, x, off, heads, kv, D, causal, gy)
    alone = np.r_[0:3, off[-1]:M]
    assert not o["y"][alone].any() and not o["lse"][:, alone].any() and not o["gx"][alone].any()
    check_attention(o, od.attention(values(x, "bf16"), off, heads, kv, D, causal, values(gy, "bf16")), heads, D, most)
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("size", [1e-3, 8.0, 40.0])
def test_attention_with_flat_and_sharp_scores(torch_mod, size):
    """Scores of almost no spread, and of some thousand units: a single key has all the weight."""
    rng = np.random.default_rng(7)
    heads, kv, D, off = 2, 1, 64, offsets([150, 90])
    M = int(off[-1])
    x = rng.normal(size=(M, 4 * D))
    x[:, :3 * D] *= size
    x, gy = storage(x, "bf16"), storage(rng.normal(size=(M, 2 * D)), "bf16")
    b, o = run_attention(torch_mod, x, off, heads, kv, D, True, gy)
    check_attention(o, od.attention(values(x, "bf16"), off, heads, kv, D, True, values(gy, "bf16")), heads, D, 150)
    b.close()


def test_attention_without_its_log_sum_exp(torch_mod):
    import paper_2203_15980_amd as dl
    rng = np.random.default_rng(18)
    off = offsets([70, 33])
    x = storage(rng.normal(size=(103, 4 * 64)), "bf16")
    b, o = run_attention(torch_mod, x, off, 2, 1, 64, True)
    b.d.release(3, dl.EV_EVICT)
    o["L"].y2 = dl.NO_TENSOR
    b.d.recompute_segment([o["L"]])
    assert np.array_equal(values(b.get(2, np.uint16, (103, 128)), "bf16"), o["y"])
    with pytest.raises(dl.DeltaError):
        b.d.tensor_ptr(3)
    b.close()


def test_attention_keeps_a_bad_row_in_its_sequence(torch_mod):
    rng = np.random.default_rng(8)
    heads, kv, D, off = 4, 2, 64, offsets([100, 61, 130])
    M, W = int(off[-1]), 8 * 64
    x, gy = storage(rng.normal(size=(M, W)), "bf16"), storage(rng.normal(size=(M, heads * D)), "bf16")
    b, o = run_attention(torch_mod, x, off, heads, kv, D, True, gy)
    bad = x.copy()
    bad[130] = 0x7FC0                                            # NaN in the second sequence
    bad[140, ::3] = 0x7F80
    b1, o1 = run_attention(torch_mod, bad, off, heads, kv, D, True, gy)
    others = np.r_[0:100, 161:M]
    for n in ("y", "gx"):
        assert np.array_equal(o1[n][others], o[n][others])
    assert np.array_equal(o1["lse"][:, others], o["lse"][:, others]) and np.isnan(o1["y"][130]).all()
    b.close()
    b1.close()


@pytest.mark.parametrize("off", [[0, 50, 20, 200], [-5, 300, 10 ** 12, 7], [200, 150, 100, 0], [2 ** 62, -2 ** 62, 3, 3]])
def test_attention_with_bad_offsets_stays_inside_its_tensors(torch_mod, off):
    """Offsets that do not ascend or leave the rows: every boundary is held in [0, rows] where it is read (packed_attention.hpp, boundary), so what is
    computed is some rows of the tensors."""
    rng = np.random.default_rng(9)
    x, gy = storage(rng.normal(size=(200, 4 * 64)), "bf16"), storage(rng.normal(size=(200, 128)), "bf16")
    b, o = run_attention(torch_mod, x, off, 2, 1, 64, True, gy)
    assert b.untouched()
    b.close()


def test_attention_of_one_sequence_is_the_padded_operators(torch_mod):
    """A batch of equal sequences, not causal, equal heads of 64: the operator over padded sequences computes the same."""
    import paper_2203_15980_amd as dl
    rng = np.random.default_rng(10)
    N, S, heads = 3, 130, 4
    x = storage(rng.normal(size=(N * S, 3 * heads * 64)), "bf16")
    b, o = run_attention(torch_mod, x, offsets([S] * N), heads, heads, 64, False)
    b.d.recompute_segment([b.layer(dl.OP_ATTENTION, S, 3 * heads * 64, heads * 64, 0, 2, N=N, R=heads)])
    y = values(b.get(2, np.uint16, (N * S, heads * 64)), "bf16")
    ref = od.attention(values(x, "bf16"), offsets([S] * N), heads, heads, 64, False)
    # both are within 2^-8 |y| + (2^-8 + scores' and sums' errors) sum p |v| of the definition
    tol = 2 * (2.0 ** -8 * np.abs(ref["y"]) + (2.0 ** -8 + 2.0 ** -12) * ref["pv"])
    near(y, o["y"], tol)
    b.close()


# ------------------------------------------------------------------ log probabilities

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,K", [(1, 1, 1), (3, 7, 7), (5, 64, 64), (2, 511, 20), (4, 4096, 5), (9, 4099, 64), (3, 16383, 1), (2, 16385, 33), (1, 30522, 20), (3, 50001, 0), (70, 100, 0),
                                   (300, 17, 3)])
def test_logprob(torch_mod, dtype, M, V, K):
    print("logprob", dtype, M, V, K, flush=True)
    rng = np.random.default_rng(V + K)
    z = rng.normal(size=(M, V)) * 3
    z[:, rng.integers(0, V)] += 8
    if V > 10:
        z[:, V // 2:V // 2 + 3] = -np.inf
    z = storage(np.round(z * 4) / 4 if V == 4099 else z, dtype)                    # many equal ones
    ids = rng.integers(0, V, M)
    if M > 4:
        ids[1], ids[3] = -1, V
    if V > 10 and M > 2:
        ids[2] = V // 2                                          # a token without weight
    gy = (rng.normal(size=(3, M)) / 3).astype(np.float32)
    gy[0, 2:3] = 0
    b, o = run_logprob(torch_mod, z, ids, dtype, K, gy)
    zf = values(z, dtype)
    y, best, which = od.logprob(zf, ids, K)
    lp, nH, nl = logprob_noise(zf, y)
    m = zf.max(axis=1)
    mine = zf[np.arange(M), np.clip(ids, 0, V - 1)]
    for k, tol in ((0, lp(np.where(np.isfinite(mine), m - mine, 0))), (1, nH), (2, nl)):
        fine = np.isfinite(y[k])
        near(o["y"][k][fine], y[k][fine], tol[fine])
        assert np.array_equal(o["y"][k][~fine], y[k][~fine])
    if K:
        assert np.array_equal(o["which"], which)
        fine = np.isfinite(best)
        theirs = np.take_along_axis(zf, np.clip(which, 0, V - 1), axis=1)
        near(np.where(fine, o["best"], 0), np.where(fine, best, 0), lp(np.where(np.isfinite(theirs), m[:, None] - theirs, 0)))
        assert np.array_equal(o["best"][~fine], best[~fine])
    want = od.logprob_bwd(zf, ids, gy.astype(np.float64))
    # p by the stored log-sum-exp (its error and rounding) and 4 + 3 |log p| roundings; the bracket by 4 roundings of its terms and the errors of H and of the log-sum-exp
    with np.errstate(invalid="ignore", over="ignore"):
        l = zf - np.where(np.isfinite(y[2]), y[2], 0)[:, None]
        p = np.exp(l)
        la = np.where(p > 0, np.abs(l), 0)
    rel = (nl + EPS24 * np.abs(np.where(np.isfinite(y[2]), y[2], 0)))[:, None] + EPS24 * (4 + 3 * la)
    g = np.abs(gy.astype(np.float64))
    bracket = (g[2] + g[0])[:, None] + g[1][:, None] * (la + np.abs(y[1])[:, None])
    tol = half_step(dtype) * np.abs(want) + p * (bracket * (rel + 6 * EPS24) + g[1][:, None] * (nl + nH)[:, None]) + 2 * EPS24 * g[0][:, None]
    near(o["gz"], want, tol)
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprob_of_special_rows(torch_mod, dtype):
    low = -3.3895313892515355e38 if dtype == "bf16" else -3.4028234663852886e38    # the type's lowest
    V, K = 70, 9
    z = np.zeros((9, V))
    z[0] = low                                                   # uniform
    z[1, :], z[1, 5] = low, 3.0                                  # all but one masked with it
    z[2] = -np.inf
    z[3, 11], z[4, 12], z[5, ::2] = np.nan, np.inf, -np.inf
    z[6, ::2] = -0.0
    z[7] = 3e38
    z[8] = np.linspace(-1e30, 1e30, V)
    z = storage(z, dtype)
    ids = np.array([3, 5, 1, 2, 2, 3, 4, 69, 69])
    gy = np.full((3, 9), 0.5, np.float32)
    b, o = run_logprob(torch_mod, z, ids, dtype, K, gy)
    zf = values(z, dtype)
    y, best, which = od.logprob(zf, ids, K)
    which[3] = [11] + [j for j in range(K)][:K - 1]              # of a row with a NaN: the NaN, then the zeros in order
    assert np.array_equal(o["which"], which)
    for r in (3, 4):
        assert np.isnan(o["y"][0, r]) and np.isnan(o["y"][1, r]) and not np.isfinite(o["y"][2, r])
    for r in (0, 1, 2, 5, 6, 7, 8):
        inf = ~np.isfinite(y[:, r])
        assert np.array_equal(o["y"][inf, r], y[inf, r])
        assert (np.abs(o["y"][~inf, r] - y[~inf, r]) <= 200 * EPS24 * (1 + np.abs(y[:, r][~inf]))).all(), (r, o["y"][:, r], y[:, r])
        f = np.isfinite(best[r])
        assert (np.abs(o["best"][r][f] - best[r][f]) <= 200 * EPS24 * (1 + np.abs(best[r][f]))).all()
    assert not o["gz"][2].any() and np.isnan(o["gz"][3]).any()
    want = od.logprob_bwd(zf[[5, 6]], ids[[5, 6]], gy[:, [5, 6]].astype(np.float64))
    near(o["gz"][[5, 6]], want, (half_step(dtype) + 300 * EPS24) * np.abs(want) + 300 * EPS24 / V)
    b.close()


def test_logprob_gradient_of_a_row_far_from_zero(torch_mod):
    """Logits around 10000: the log-sum-exp is rounded to 2^-11 there, which bounds the error of p."""
    rng = np.random.default_rng(11)
    z = storage(10000 + rng.normal(size=(4, 300)), "f32")
    ids, gy = np.arange(4), np.ones((3, 4), np.float32)
    b, o = run_logprob(torch_mod, z, ids, "f32", 0, gy)
    want = od.logprob_bwd(z.astype(np.float64), ids, gy)
    near(o["gz"], want, (2.0 ** -10) * 8 * (np.exp(z.astype(np.float64) - 10005) + 0.02) + 2.0 ** -9)
    b.close()
