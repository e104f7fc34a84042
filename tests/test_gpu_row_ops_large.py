"""Layer normalisation, checkpoints and the embedding on tensors of more than 4 GiB: rows behind 32-bit offsets, on both sides of them and the last."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, half_step, layernorm_noise, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    return torch


def _fill(torch, b, i, dtype, seed):
    t = b.arena[b.at[i]:b.at[i] + b.sizes[i]].view(dtype)
    t.normal_(generator=torch.Generator("cuda:0").manual_seed(seed))
    torch.cuda.synchronize()
    return t


def test_normalisation_and_checkpoint(torch_mod):
    torch, rows, C = torch_mod, 270000, 8192                 # 4.4 GB in bf16, 2.2 GB of bytes; row 262144 begins at 2^32 and at 2^31
    nb, pb = rows * C * 2, ro.packed_bytes(rows, C)
    b = Bench(torch, [nb, pb, nb, nb, nb])
    dl = b.dl
    x, gy = _fill(torch, b, 0, torch.bfloat16, 1).view(rows, C), _fill(torch, b, 2, torch.bfloat16, 2).view(rows, C)
    at = [0, 1, 131071, 131072, 262143, 262144, 262145, rows - 2, rows - 1]
    pick = lambda t: values(t[at].view(torch.int16).cpu().numpy().view(np.uint16), "bf16")
    X, GY = pick(x), pick(gy)
    gamma = np.random.default_rng(3).uniform(0.5, 1.5, C).astype(np.float32)
    g = b.dev(gamma)
    kw = dict(scale=g.data_ptr(), shift=g.data_ptr(), eps=1e-5)
    view = lambda i: b.arena[b.at[i]:b.at[i] + nb].view(torch.bfloat16).view(rows, C)
    b.d.recompute_segment([b.layer(dl.OP_PACK8, rows, C, C, 0, 1, pack=dl.PACK_INT8), b.layer(dl.OP_UNPACK8, rows, C, C, 1, 3, pack=dl.PACK_INT8)])
    b.d.sync()
    U = ro.unpack(*ro.pack(X, "int8"), "int8")
    assert np.array_equal(pick(view(3)), U)
    fwd = b.layer(dl.OP_LAYERNORM, rows, C, C, 0, 4, **kw)
    b.d.recompute_segment([fwd])
    b.d.sync()
    c = X - X.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + 1e-5)
    y = c * r * gamma + gamma
    noise = 40 * EPS24 * (np.abs(X).max(axis=1, keepdims=True) * r + np.abs(c * r).max(axis=1, keepdims=True)) * gamma      # as rowops_util derives it for xh
    assert (np.abs(pick(view(4)) - y) <= half_step("bf16") * np.abs(y) + 2 * noise + EPS24 * np.abs(y)).all()
    for source, pack, have in ((0, 0, X), (1, dl.PACK_INT8, U)):
        b.d.backward_segment([b.bwd(b.layer(dl.OP_LAYERNORM, rows, C, C, source, 4, pack=pack, **kw), 2, gx=3)])
        b.d.sync()
        want = ro.layernorm_bwd(have, GY, gamma, 1e-5, None)[0]
        tol = half_step("bf16") * np.abs(want) + 2 * layernorm_noise(have, GY, gamma, 1e-5)[0]
        assert (np.abs(pick(view(3)) - want) <= tol).all()
    b.close()


def test_embedding(torch_mod):
    torch, V, C, n = torch_mod, 270000, 4096, 300            # table and gradient 4.4 GB in fp32
    w = torch.empty(V, C, device="cuda:0").normal_(generator=torch.Generator("cuda:0").manual_seed(5))
    rng = np.random.default_rng(6)
    ids = rng.integers(0, V, n)
    ids[:8] = [V - 1, 0, 262143, 262144, V - 1, 131072, -1, V]
    scale = np.full(C, 2.0, np.float32)
    b = Bench(torch, [n * 8, n * C * 4, n * C * 4])
    gi = rng.integers(-64, 65, (n, C)).astype(np.float32)
    b.put(0, ids); b.put(2, gi)
    s = b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, "f32", w=w.data_ptr(), scale=s.data_ptr())
    b.d.recompute_segment([fwd])
    got = b.get(1, np.float32, (n, C))
    there = (ids >= 0) & (ids < V)
    want = w[torch.from_numpy(np.where(there, ids, 0)).to("cuda:0")].cpu().numpy() * 2 * there[:, None]
    assert np.array_equal(got, want)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    w.fill_(float("nan"))                                    # its memory takes the gradient
    torch.cuda.synchronize()
    b.d.backward_segment([b.bwd(fwd, 2, gw=w, ws=ws)])
    b.d.sync()
    some, place = np.unique(ids[there], return_inverse=True)
    sums = np.zeros((len(some), C), np.float32)
    np.add.at(sums, place, gi[there])
    at = torch.from_numpy(some).to("cuda:0")
    assert np.array_equal(w[at].cpu().numpy(), 2 * sums)
    w[at] = 0
    assert int(torch.count_nonzero(w)) == 0
    b.close()
