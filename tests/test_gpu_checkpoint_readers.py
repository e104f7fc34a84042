"""What the checkpoint format treats specially, in the gradients that read it: blocks that hold an infinity or a NaN (scale byte 255), the smallest scale (byte
7, whose E4M3 values are subnormal in bf16), the largest ones, in the last valid row and in the middle.  The readers work on the values that unpacking gives:
the weight gradient is compared with the exact one (whole numbers) and with the unpacked tensor's, layer normalisation's gradients bit for bit with the
unpacked tensor's."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import Bench, storage, values

pytestmark = pytest.mark.gpu

FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


class Linear:
    """x [rows, C] and g [rows, K] in bf16, x's checkpoint and what it unpacks to; the weight gradient from either."""

    def __init__(self, torch, x, g, fmt):
        rows, C = x.shape
        K = g.shape[1]
        self.shape = (K, C)
        self.b = b = Bench(torch, [x.nbytes, ro.packed_bytes(rows, C), x.nbytes, g.nbytes, g.nbytes])
        b.put(0, x); b.put(3, g)
        self.k = {"int8": b.dl.PACK_INT8, "e4m3": b.dl.PACK_E4M3}[fmt]
        b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, C, C, 0, 1, pack=self.k), b.layer(b.dl.OP_UNPACK8, rows, C, C, 1, 2, pack=self.k)])
        one, zero, w = b.dev(np.ones(K, np.float32)), b.dev(np.zeros(K, np.float32)), b.dev(np.zeros((K, C), np.int16))
        self.kw = dict(w=w.data_ptr(), scale=one.data_ptr(), shift=zero.data_ptr())
        self.rows = rows

    def gw(self, packed):
        b, (K, C) = self.b, self.shape
        fwd = b.layer(b.dl.OP_CONV, self.rows, C, K, 1 if packed else 2, 4, pack=self.k if packed else 0, **self.kw)
        ws, _ = b.workspace(b.d.backward_workspace(fwd))
        gw, guard = b.guarded(K * C)
        desc = b.bwd(fwd, 3, gw=gw, ws=ws)
        assert ("from" in b.d.backward_kernel(desc)) == packed
        b.d.backward_segment([desc])
        b.d.backward_join()
        b.d.sync()
        assert (guard[:64] == 12345.0).all() and (guard[64 + K * C:] == 12345.0).all()
        return gw.cpu().numpy().reshape(K, C)


def _whole(rows, C, K):
    """Whole numbers that both formats hold exactly, and so do all sums."""
    rng = np.random.default_rng(rows + C + K)
    return rng.integers(-8, 9, (rows, C)).astype(np.float64), rng.integers(-4, 5, (rows, K)).astype(np.float64)


# every shape of tile: (64, 128, 256 of k) x (64, 128, 256 of c); rows that end inside a slice, a step and a group of eight
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,C,K", [(333, 64, 64), (200, 64, 128), (333, 64, 256), (129, 128, 64), (333, 128, 128), (200, 256, 64), (1001, 256, 128), (1, 64, 64),
                                      (7, 128, 256), (65, 64, 256), (4097, 320, 192)])
def test_a_bad_block_spoils_its_columns_alone(torch_mod, rows, C, K, fmt):
    print("rows", rows, "C", C, "K", K, fmt, flush=True)
    x, g = _whole(rows, C, K)
    spoilt = np.zeros(C, bool)
    for row, col, what in ((rows - 1, C - 1, np.inf), (rows // 2, 0, np.nan)):
        x[row, col] = what
        spoilt[col // 32 * 32:col // 32 * 32 + 32] = True
    t = Linear(torch_mod, storage(x, "bf16"), storage(g, "bf16"), fmt)
    want = g.T @ np.where(spoilt, 0.0, np.nan_to_num(x, posinf=0.0))
    got = t.gw(True)
    assert np.isnan(got[:, spoilt]).all()
    assert np.array_equal(got[:, ~spoilt], want[:, ~spoilt])
    assert np.array_equal(got, t.gw(False), equal_nan=True)
    t.b.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,C,K", [(333, 64, 64), (129, 128, 128), (200, 256, 64), (65, 64, 256)])
def test_the_smallest_and_largest_scales(torch_mod, rows, C, K, fmt):
    """Columns 0 .. 31: multiples of 2^-129 (E4M3 holds them at scale byte 7; int8 rounds them to zero).  Columns 32 .. 63: one value near the top of bf16 in
    each, in one row whose g is small, beside zeros; one of them rounds up to 2^128, an infinity, as in the unpacked tensor."""
    rng = np.random.default_rng(rows + C)
    x, g = _whole(rows, C, K)
    g[g == 0] = 1.0                                          # an infinity times zero is another matter
    x[:, :32] = rng.integers(-7, 8, (rows, 32)) * 2.0 ** -129
    x[0, 0] = 7 * 2.0 ** -129
    x[:, 32:64] = 0.0
    at = rows - 1
    x[at, 32:64] = 1.5 * 2.0 ** 127 * np.where(np.arange(32) % 2, 1, -0.5)
    x[at, 40] = 255 * 2.0 ** 120                             # bf16's largest: 64 * 2^122 in int8, 256 * 2^120 in E4M3
    t = Linear(torch_mod, storage(x, "bf16"), storage(g, "bf16"), fmt)
    pay, sc = ro.pack(values(storage(x, "bf16"), "bf16"), fmt)
    # 255 * 2^120 is more than 127 * 2^121 = 254 * 2^120, and more than 448 * 2^119 = 224 * 2^120: e = 122 and 120
    assert (sc[:, 0] == 7).all() and sc[at, 1] == 127 + {"int8": 122, "e4m3": 120}[fmt]
    u = values(storage(ro.unpack(pay, sc, fmt), "bf16"), "bf16")
    assert np.isinf(u[at, 40]) and np.isfinite(np.delete(u[at], 40)).all()
    assert np.array_equal(values(t.b.get(2, np.uint16, x.shape), "bf16"), u)
    g[at] = np.sign(g[at]) * 2.0 ** -4
    t.b.put(3, storage(g, "bf16"))
    with np.errstate(invalid="ignore"):
        want = g.T @ np.where(np.isinf(u), 0.0, u)
    got, plain = t.gw(True), t.gw(False)
    assert np.array_equal(got, plain)
    assert np.isposinf(got[:, 40] * np.sign(g[at])).all()
    rest = np.ones(C, bool)
    rest[40] = False
    rest[:32] = False                                        # of subnormal factors: as from the unpacked tensor, above
    assert np.array_equal(got[:, rest], want[:, rest].astype(np.float32))
    t.b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,C", [(77, 72), (40, 768), (1030, 1544), (9, 2112), (1100, 2048)])
def test_normalisation_reads_bad_blocks_and_extreme_scales_as_unpacked(torch_mod, rows, C, fmt, dtype):
    print("rows", rows, "C", C, fmt, dtype, flush=True)
    rng = np.random.default_rng(rows + C)
    x = rng.normal(size=(rows, C))
    bad = [2, rows // 2, rows - 1]
    x[bad[0], C - 1], x[bad[1], 0], x[bad[2], C // 2] = np.inf, np.nan, -np.inf
    x[5] = rng.integers(-7, 8, C) * 2.0 ** -129              # the smallest scale
    x[6] *= 2.0 ** 60                                        # large ones: squares leave fp32 from 2^64 on
    gy = storage(rng.normal(size=(rows, C)), dtype)
    x = storage(x, dtype)
    gamma = rng.uniform(0.5, 1.5, C).astype(np.float32)
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C)] + [x.nbytes] * 4)
    b.put(0, x); b.put(3, gy)
    g = b.dev(gamma)
    k = {"int8": b.dl.PACK_INT8, "e4m3": b.dl.PACK_E4M3}[fmt]
    kw = dict(scale=g.data_ptr(), shift=g.data_ptr(), eps=1e-5)
    b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, C, C, 0, 1, dtype, pack=k), b.layer(b.dl.OP_UNPACK8, rows, C, C, 1, 2, dtype, pack=k)])
    runs = []
    for source, pack in ((1, k), (2, 0)):
        fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, source, 5, dtype, pack=pack, **kw)
        ws, _ = b.workspace(b.d.backward_workspace(fwd))
        gw, _ = b.guarded(2 * C)
        b.d.backward_segment([b.bwd(fwd, 3, gx=4, gw=gw, ws=ws)])
        gx = values(b.get(4, x.dtype, x.shape), dtype)
        runs.append((gx, gw.cpu().numpy()))
    for gx, gw in runs:
        assert np.isnan(gx[bad]).all() and np.isfinite(np.delete(gx, bad, axis=0)).all()
        assert np.isnan(gw[:C]).all() and np.isfinite(gw[C:]).all()
    assert np.array_equal(runs[0][0], runs[1][0], equal_nan=True) and np.array_equal(runs[0][1], runs[1][1], equal_nan=True)
    b.close()
