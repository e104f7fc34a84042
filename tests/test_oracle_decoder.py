"""Pins of the decoder operators' oracle: gradients against differences, closed forms, hand-made cases."""
import numpy as np
import pytest

from oracle import decoder as od


def differences(f, x, h=1e-6):
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_rmsnorm_and_its_gradient():
    rng = np.random.default_rng(0)
    s, g, w, gamma = rng.normal(size=(3, 8)), rng.normal(size=(3, 8)), rng.normal(size=(3, 8)), rng.uniform(0.5, 1.5, 8)
    y = od.rmsnorm(s, gamma, 0.0) / gamma
    assert np.allclose((y * y).mean(axis=1), 1)
    assert np.allclose(od.rmsnorm(7 * s, gamma, 0.0), od.rmsnorm(s, gamma, 0.0))
    gx, dg = od.rmsnorm_bwd(s, g, gamma, 1e-3, w)
    assert np.allclose(gx - w, differences(lambda a: (od.rmsnorm(a, gamma, 1e-3) * g).sum(), s), atol=1e-7)
    assert np.allclose(dg, differences(lambda a: (od.rmsnorm(s, a, 1e-3) * g).sum(), gamma), atol=1e-7)


@pytest.mark.parametrize("pairs", [False, True])
def test_rotary_keeps_lengths_and_turns_by_differences_of_positions(pairs):
    rng = np.random.default_rng(1)
    D, heads = 16, 2
    freq = np.zeros((2, D // 2), np.float32)
    freq[0, ::2] = 0.3
    freq[1, 1::2] = 0.7
    q, k = rng.normal(size=(1, heads * D + 8)), rng.normal(size=(1, heads * D + 8))
    dot = lambda p, t: float((od.rotary(q, od.angles([p], freq), heads, D, pairs)[:, :D] * od.rotary(k, od.angles([t], freq), heads, D, pairs)[:, :D]).sum())   # noqa: E731
    assert np.isclose(dot((5, 9), (3, 2)), dot((105, 40), (103, 33)))
    y = od.rotary(q, od.angles([(3, 4)], freq), heads, D, pairs)
    assert np.isclose((y * y).sum(), (q * q).sum()) and np.array_equal(y[:, heads * D:], q[:, heads * D:])
    assert np.allclose(od.rotary(y, -od.angles([(3, 4)], freq), heads, D, pairs), q)
    x = np.zeros((1, D))
    x[0, 0] = 1.0
    y = od.rotary(x, od.angles([(1, 0)], freq), 1, D, pairs)
    assert np.isclose(y[0, 0], np.cos(np.float32(0.3))) and np.isclose(y[0, 1 if pairs else D // 2], np.sin(np.float32(0.3)))


def test_attention_of_hand_made_sequences_and_its_gradient():
    rng = np.random.default_rng(2)
    H, G, D = 4, 2, 4
    x = rng.normal(size=(7, (H + 2 * G) * D))
    off = [1, 4, 4, 6]
    o = od.attention(x, off, H, G, D, True)
    v = x[:, (H + G) * D:].reshape(7, G, D)
    for first in (1, 4):                                         # a sequence's first row sees itself alone
        for h in range(H):
            assert np.allclose(o["y"][first, h * D:(h + 1) * D], v[first, h // 2])
    assert not o["y"][[0, 6]].any() and not o["lse"][:, [0, 6]].any()
    full = od.attention(x, off, H, G, D, False)
    assert np.allclose(full["y"][3], o["y"][3]) and not np.allclose(full["y"][1], o["y"][1])
    y = x.copy()
    y[:, H * D:(H + G) * D] = 0                                  # equal scores: means
    m = od.attention(y, off, H, G, D, False)
    assert np.allclose(m["y"][2, :D], v[1:4, 0].mean(axis=0)) and np.allclose(m["lse"][:, 2], np.log(3))
    for causal in (False, True):
        g = rng.normal(size=(7, H * D))
        got = od.attention(x, off, H, G, D, causal, g)["gx"]
        assert np.allclose(got, differences(lambda a: (od.attention(a, off, H, G, D, causal)["y"] * g).sum(), x), atol=1e-7)


def test_logprob_closed_forms_and_gradient():
    z = np.array([[0.0, 0.0, 0.0, 0.0], [1.0, -np.inf, 1.0, -np.inf], [-np.inf] * 4, [3.0, 1.0, np.nan, 1.0], [2.0, 2.0, -0.0, 0.0]])
    y, best, which = od.logprob(z, [1, 0, 2, 0, 4], 3)
    assert np.allclose(y[:, 0], [-np.log(4), np.log(4), np.log(4)])
    assert np.allclose(y[:, 1], [-np.log(2), np.log(2), 1 + np.log(2)])
    assert y[0, 2] == y[2, 2] == -np.inf and y[1, 2] == 0 and np.isnan(y[:, 3]).all()
    assert (y[:, 4] == 0).all() and (which[4] == -1).all() and (best[4] == 0).all()
    assert which[:4].tolist() == [[0, 1, 2], [0, 2, 1], [0, 1, 2], [2, 0, 1]]
    rng = np.random.default_rng(3)
    z, ids, g = rng.normal(size=(4, 9)) * 3, [0, 8, 3, -1], rng.normal(size=(3, 4))
    gz = od.logprob_bwd(z, ids, g)
    assert np.allclose(gz, differences(lambda a: (od.logprob(a, ids)[0] * g).sum(), z), atol=1e-7)
    assert not gz[3].any()
    z[0, 4] = -np.inf
    assert od.logprob_bwd(z, ids, g)[0, 4] == 0 and np.isfinite(od.logprob_bwd(z, ids, g)).all()
