"""Pins of the row operators' oracle (oracle/rowops.py) to things other than itself: differences of the forward
functions, closed forms, and blocks worked by hand; and the checks of the entry point that needs no GPU."""
import numpy as np
import pytest

import paper_2203_15980_amd as dl
from oracle import rowops as ro


def test_layernorm_gradients_are_those_of_the_forward_function_by_differences():
    rng = np.random.default_rng(5)
    M, C, eps = 3, 16, 1e-5
    x, gy, add = rng.normal(1.0, 2.0, (M, C)), rng.normal(size=(M, C)), rng.normal(size=(M, C))
    gamma, beta = rng.uniform(0.5, 1.5, C), rng.normal(size=C)
    loss = lambda x_, g_, b_: (ro.layernorm(x_, g_, b_, eps) * gy).sum() + (x_ * add).sum()      # noqa: E731
    gx, dg, db = ro.layernorm_bwd(x, gy, gamma, eps, add)
    h = 1e-6
    for (i, j) in [(0, 0), (1, 7), (2, 15)]:
        d = np.zeros((M, C))
        d[i, j] = h
        assert abs((loss(x + d, gamma, beta) - loss(x - d, gamma, beta)) / (2 * h) - gx[i, j]) < 1e-7
    for j in (0, 9):
        d = np.zeros(C)
        d[j] = h
        assert abs((loss(x, gamma + d, beta) - loss(x, gamma - d, beta)) / (2 * h) - dg[j]) < 1e-7
        assert abs((loss(x, gamma, beta + d) - loss(x, gamma, beta - d)) / (2 * h) - db[j]) < 1e-7


def test_layernorm_gradient_vanishes_along_shift_and_scale_of_a_row():
    rng = np.random.default_rng(6)
    x, gy = rng.normal(size=(4, 24)), rng.normal(size=(4, 24))
    gx = ro.layernorm_bwd(x, gy, np.ones(24), 0.0)[0]
    assert np.abs(gx.sum(axis=1)).max() < 1e-12 and np.abs((gx * x).sum(axis=1)).max() < 1e-12


def test_e4m3_numbers():
    v = ro.E4M3
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[126] == 448.0
    assert (np.diff(v) > 0).all()
    assert ro._nearest_e4m3(np.array([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10])).tolist() == [0x38, 0x3A, 0, 2]     # ties go to the even code


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_checkpoint_scales_are_the_smallest_that_fit(fmt):
    most = ro.MOST[fmt]
    x = np.zeros((6, 40))
    x[0, 3] = most                          # exactly at the limit: e = 0
    x[1, 3] = np.nextafter(most, 1e9)       # just beyond: e = 1
    x[2, 35] = -most * 2.0 ** -7            # in the short last block
    x[3, 0] = 2.0 ** -149                   # far below the smallest scale
    x[4, 0] = np.inf
    pay, sc = ro.pack(x, fmt)
    assert sc[:, 0].tolist() == [127, 128, 7, 7, 255, 7]
    assert sc[2, 1] == 120 and sc[0, 1] == 7
    back = ro.unpack(pay, sc, fmt)
    assert back[0, 3] == most and back[1, 3] == {"int8": 128.0, "e4m3": 448.0}[fmt] and back[2, 35] == x[2, 35] and back[3, 0] == 0
    assert np.isnan(back[4, :32]).all() and (back[4, 32:] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_checkpoint_error_is_half_a_step_and_values_are_exact_in_bf16(fmt):
    rng = np.random.default_rng(7)
    x = rng.normal(size=(50, 72)) * np.exp(3 * rng.normal(size=(50, 1)))
    pay, sc = ro.pack(x, fmt)
    back = ro.unpack(pay, sc, fmt)
    step = np.repeat(np.exp2(sc.astype(float) - 127), 32, axis=1)[:, :72]
    bound = step / 2 if fmt == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, step * 2.0 ** -10)
    assert (np.abs(back - x) <= bound).all()
    assert ((back.astype(np.float32).view(np.uint32) & 0xFFFF) == 0).all()
    assert np.array_equal(ro.unpack(*ro.pack(back, fmt), fmt), back)      # packing again changes nothing


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    rng = np.random.default_rng(8)
    V, C = 9, 8
    ids = np.array([3, 0, -1, 3, 8, 9, 2 ** 40, 3])
    scale = rng.uniform(0.5, 2, C)
    w, gy = rng.normal(size=(V, C)), rng.normal(size=(len(ids), C))
    y, gw = ro.embedding(ids, w, scale), ro.embedding_bwd(ids, gy, scale, V)
    assert (y[[2, 5, 6]] == 0).all()
    assert abs((y * gy).sum() - (w * gw).sum()) < 1e-12
    assert (gw[[1, 2, 4, 5, 6, 7]] == 0).all()


def test_packed_bytes_on_a_planner_only_context():
    d = dl.Delta()
    for rows, C in [(1, 8), (1, 32), (3, 40), (77, 768), (16384, 768), (5, 1016), (2 ** 31 - 1, 8192)]:
        assert d.packed_bytes(rows, C) == ro.packed_bytes(rows, C)
    for rows, C in [(0, 8), (1, 0), (1, 12), (2 ** 31, 8)]:
        with pytest.raises(dl.DeltaError) as e:
            d.packed_bytes(rows, C)
        assert e.value.status == dl.ERR_INVALID
    d.close()
