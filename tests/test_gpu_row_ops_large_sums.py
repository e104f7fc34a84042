"""The row operators' sums over tensors of more than 4 GiB, and the table gradient of wide rows where the sort goes over all workgroups.  References are made
on the device, in float64 or in whole numbers (exact in fp32, whatever the order)."""
import numpy as np
import pytest

from rowops_util import EPS24, Bench

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    return torch


def _ids(torch, n, V, seed):
    """Ids over the whole table, the table's ends, one frequent id, some of no token."""
    g = torch.Generator("cuda:0").manual_seed(seed)
    ids = torch.randint(0, V, (n,), device="cuda:0", generator=g)
    ids[torch.rand(n, device="cuda:0", generator=g) < 0.05] = V // 3
    ids[torch.rand(n, device="cuda:0", generator=g) < 0.1] = -1
    ids[0], ids[1], ids[2], ids[n - 1] = V - 1, 0, V, V - 1
    return ids


# sort: 512 tokens a workgroup with rows of 2048 channels; then over a table of 4.4 GB, whose zeros four launches write, 256 and 512 tokens a workgroup
@pytest.mark.parametrize("n,V,C,dtype", [(32768, 131072, 2048, "bf16"), (65536, 30522, 768, "f32"), (8193, 270000, 4096, "f32"), (20001, 270000, 4096, "bf16"),
                                         (16385, 1000, 8192, "f32")])
def test_table_gradient(torch_mod, n, V, C, dtype):
    torch = torch_mod
    print("tokens", n, "V", V, "C", C, dtype, flush=True)
    es, t = (2, torch.bfloat16) if dtype == "bf16" else (4, torch.float32)
    b = Bench(torch, [n * 8, n * C * es, n * C * es])
    view = lambda i, t: b.arena[b.at[i]:b.at[i] + b.sizes[i]].view(t)          # noqa: E731
    ids = _ids(torch, n, V, n)
    view(0, torch.int64).copy_(ids)
    gy = view(2, t).view(n, C)
    gy.copy_(torch.randint(-8, 9, (n, C), device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(n + 1)))
    s = b.dev(np.full(C, 2.0, np.float32))
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, dtype, w=s.data_ptr(), scale=s.data_ptr())
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw = torch.full((V, C), float("nan"), device="cuda:0")
    torch.cuda.synchronize()
    b.d.backward_segment([b.bwd(fwd, 2, gw=gw, ws=ws)])
    b.d.sync()
    there = (ids >= 0) & (ids < V)
    want = torch.zeros(V, C, device="cuda:0")
    want.index_add_(0, ids[there], gy[there].float() * 2)
    assert torch.equal(gw, want)
    b.close()


def test_embedding_of_more_than_4_gib(torch_mod):
    """y and gy of 4.4 GB: rows behind 2^32 bytes are stored and read."""
    torch, n, V, C = torch_mod, 270000, 300, 8192
    b = Bench(torch, [n * 8, n * C * 2, n * C * 2])
    view = lambda i, t: b.arena[b.at[i]:b.at[i] + b.sizes[i]].view(t)          # noqa: E731
    ids = _ids(torch, n, V, 9)
    view(0, torch.int64).copy_(ids)
    w = torch.randint(-8, 9, (V, C), device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(1)).to(torch.bfloat16)
    gy = view(2, torch.bfloat16).view(n, C)
    gy.copy_(torch.randint(-8, 9, (n, C), device="cuda:0", dtype=torch.int8, generator=torch.Generator("cuda:0").manual_seed(2)))
    s = b.dev(np.full(C, 2.0, np.float32))
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, w=w.data_ptr(), scale=s.data_ptr())
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw = torch.full((V, C), float("nan"), device="cuda:0")
    torch.cuda.synchronize()
    b.d.recompute_segment([fwd])
    b.d.backward_segment([b.bwd(fwd, 2, gw=gw, ws=ws)])
    b.d.sync()
    y, there = view(1, torch.bfloat16).view(n, C), (ids >= 0) & (ids < V)
    want = torch.zeros(V, C, device="cuda:0")
    for at in range(0, n, 16384):
        rows = slice(at, min(n, at + 16384))
        i, ok = ids[rows], there[rows]
        assert torch.equal(y[rows], (2 * w[torch.where(ok, i, 0)]) * ok[:, None]), at
        want.index_add_(0, i[ok], gy[rows][ok].float() * 2)
    assert torch.equal(gw, want)
    b.close()


def test_normalisation_sums_over_more_than_4_gib(torch_mod):
    """dgamma and dbeta of 270000 rows of 8192 channels: 256 workers add up 1055 rows each one after the other, 64 threads four of their sums each, then two
    times eight: each addition is off by half a step of the sum of magnitudes at most; xh as rowops_util derives it."""
    torch, rows, C = torch_mod, 270000, 8192
    nb = rows * C * 2
    b = Bench(torch, [nb, nb, nb, nb])
    view = lambda i: b.arena[b.at[i]:b.at[i] + nb].view(torch.bfloat16).view(rows, C)          # noqa: E731
    for i in (0, 2):
        view(i).normal_(generator=torch.Generator("cuda:0").manual_seed(i + 1))
    gamma = b.dev(np.random.default_rng(3).uniform(0.5, 1.5, C).astype(np.float32))
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 0, 1, scale=gamma.data_ptr(), shift=gamma.data_ptr(), eps=1e-5)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, _ = b.guarded(2 * C)
    torch.cuda.synchronize()
    b.d.backward_segment([b.bwd(fwd, 2, gx=3, gw=gw, ws=ws)])
    b.d.sync()
    dg, db, mag, noise = (torch.zeros(C, dtype=torch.float64, device="cuda:0") for _ in range(4))
    absolute = torch.zeros(C, dtype=torch.float64, device="cuda:0")
    for at in range(0, rows, 8192):
        x, gy = (view(i)[at:at + 8192].double() for i in (0, 2))
        c = x - x.mean(1, keepdim=True)
        r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5)
        xh = c * r
        dg += (gy * xh).sum(0)
        db += gy.sum(0)
        mag += (gy * xh).abs().sum(0)
        absolute += gy.abs().sum(0)
        noise += (gy.abs() * (40 * EPS24 * (x.abs().amax(1, keepdim=True) * r + xh.abs().amax(1, keepdim=True)))).sum(0)
    depth = (1055 + 4 + 8 + 8) * EPS24
    got = gw.double()
    assert bool(((got[:C] - dg).abs() <= noise + depth * mag).all())
    assert bool(((got[C:] - db).abs() <= depth * absolute).all())
    b.close()
