"""The embedding at its edges: factors that are infinities or NaN, ids that very many tokens hold."""
import numpy as np
import pytest

from rowops_util import EPS24, Bench, storage, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [16, 768, 2056])
def test_no_token_is_zero_whatever_the_factors_are(torch_mod, C, dtype):
    """Lookup: the row of an id outside the table is zero.  Gradient: so is the row of an id that does not occur; others follow the factor."""
    n, V = 70, 9
    rng = np.random.default_rng(C)
    ids = rng.integers(0, V - 2, n)                          # V - 2 and V - 1 do not occur
    ids[::3] = np.array([-1, V, 2 ** 40])[np.arange(len(ids[::3])) % 3]
    w, gy = storage(rng.integers(1, 9, (V, C)), dtype), storage(rng.integers(1, 9, (n, C)), dtype)
    scale = np.full(C, 2.0, np.float32)
    scale[1], scale[7], scale[C - 3] = np.inf, np.nan, -np.inf
    b = Bench(torch_mod, [ids.nbytes, gy.nbytes, gy.nbytes])
    b.put(0, ids); b.put(2, gy)
    wd, s = b.dev(w.view(np.int16) if dtype == "bf16" else w), b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, dtype, w=wd.data_ptr(), scale=s.data_ptr())
    b.d.recompute_segment([fwd])
    there = (ids >= 0) & (ids < V)
    want = np.where(there[:, None], values(w, dtype)[np.where(there, ids, 0)] * scale, 0.0)
    assert np.array_equal(values(b.get(1, w.dtype, (n, C)), dtype), want, equal_nan=True)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, _ = b.guarded(V * C)
    b.d.backward_segment([b.bwd(fwd, 2, gw=gw, ws=ws)])
    b.d.sync()
    sums = np.zeros((V, C))
    np.add.at(sums, ids[there], values(gy, dtype)[there])
    occurs = np.isin(np.arange(V), ids[there])
    assert not occurs[V - 2:].any()
    assert np.array_equal(gw.cpu().numpy().reshape(V, C), np.where(occurs[:, None], sums * scale, 0.0), equal_nan=True)
    b.close()


EVERYWHERE = [(16384, 768, "all"), (8192, 2048, "half"), (30000, 2056, "runs"), (1 << 17, 2048, "all"), (1 << 22, 8, "all"), (1 << 22, 16, "half"), ((1 << 20) + 77, 264, "runs"), (40000, 1032, "runs"), (1 << 16, 8192, "half")]


@pytest.mark.parametrize("n,C,kind", EVERYWHERE)
def test_the_row_of_a_frequent_id_is_as_exact_as_others(torch_mod, n, C, kind):
    """An id that very many tokens hold: fp32 values of one sign, against float64.  A chunk's chain is 8, 16 or 32 additions; `side` groups (8 up to 512 channels,
    one from 2048 on) join up to 256 chunks each at once.  Of more, s being the power of two next above the square root of the chunks, spans of s are joined ahead
    in chains of s / side + side, then at most 3 s of chunks, spans, chunks; one more rounding for the factor, each half a step of the sum of magnitudes."""
    torch = torch_mod
    print("tokens", n, "C", C, kind, flush=True)
    V = 11
    g = torch.Generator("cuda:0").manual_seed(n + C)
    ids = torch.full((n,), 5, device="cuda:0", dtype=torch.int64)
    if kind == "half":
        some = torch.rand(n, device="cuda:0", generator=g) < 0.5
        ids[some] = torch.randint(0, V, (int(some.sum()),), device="cuda:0", generator=g)
    if kind == "runs":                                       # long runs whose ends lie anywhere, some short, an id of no token among them
        ids = torch.tensor([1, 4, 4, 4, 9, 9, -1, 0], device="cuda:0")[torch.randint(0, 8, (n,), device="cuda:0", generator=g)]
        ids[:40] = 10
    b = Bench(torch, [n * 8, n * C * 4, n * C * 4])
    view = lambda i, t: b.arena[b.at[i]:b.at[i] + b.sizes[i]].view(t)          # noqa: E731
    view(0, torch.int64).copy_(ids)
    gy = view(2, torch.float32).view(n, C)
    value = 0.05 + torch.rand(C, device="cuda:0", generator=g)                 # one value to a channel: every addition of a chain rounds the same way
    gy.copy_(value[None])
    scale = np.full(C, 1.5, np.float32)
    s = b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, "f32", w=s.data_ptr(), scale=s.data_ptr())
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    runs = []
    for fill in (0x7F, 0x00):
        ws.fill_(fill)
        gw, guard = b.guarded(V * C)
        torch.cuda.synchronize()
        b.d.backward_segment([b.bwd(fwd, 2, gw=gw, ws=ws)])
        b.d.sync()
        runs.append(gw.clone())
    assert torch.equal(runs[0], runs[1])
    count = torch.bincount(ids[ids >= 0], minlength=V).double()
    want = count[:, None] * value.double()[None] * 1.5
    chunk, side = 8 if n <= 8192 else 16 if n <= 16384 else 32, 1 if C >= 2048 else min(8, 512 // (C // 8))
    chunks, span = -(-n // chunk), 2
    while span * span < chunks:
        span *= 2
    chain = chunk + (chunks / side if chunks <= 256 * side else 4 * span / side + side) + side + 1
    off = (runs[0].view(V, C).double() - want).abs() / want.clamp(min=1e-30)
    assert float(off.max()) <= chain * EPS24, (float(off.max()) / EPS24, chain)
    b.close()


def test_long_runs_captured_into_a_graph_and_replayed_with_other_ids(torch_mod):
    """The gradient whose spans are joined ahead, captured; each replay finds other ids in place: runs elsewhere, none, one over all tokens.  Whole numbers:
    equality with sums made on the device."""
    torch, n, V, C = torch_mod, 40000, 50, 1032
    stream = torch.cuda.Stream()
    b = Bench(torch, [n * 8, n * C * 2, n * C * 2], stream=stream)
    view = lambda i, t: b.arena[b.at[i]:b.at[i] + b.sizes[i]].view(t)          # noqa: E731
    g = torch.Generator("cuda:0").manual_seed(3)
    gy = view(2, torch.bfloat16).view(n, C)
    gy.copy_(torch.randint(-8, 9, (n, C), device="cuda:0", generator=g))
    s = b.dev(np.full(C, 2.0, np.float32))
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, w=s.data_ptr(), scale=s.data_ptr())
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, guard = b.guarded(V * C)
    desc = b.bwd(fwd, 2, gw=gw, ws=ws)
    ids = view(0, torch.int64)
    ids.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        b.d.backward_segment([desc])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.d.backward_segment([desc])
    for k in range(5):
        now = torch.randint(0, V, (n,), device="cuda:0", generator=g)
        if k in (1, 4):
            now[torch.rand(n, device="cuda:0", generator=g) < 0.7] = 7 * k
        if k == 2:
            now[:] = V - 1
        if k == 3:
            now = torch.sort(torch.randint(-1, 4, (n,), device="cuda:0", generator=g)).values
        ids.copy_(now)
        gw.fill_(float("nan"))
        ws.fill_(0x7F if k % 2 else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros(V, C, device="cuda:0")
        there = now >= 0
        want.index_add_(0, now[there], gy[there].float() * 2)
        assert torch.equal(gw.view(V, C), want), k
        assert bool((guard[:64] == 12345.0).all()) and bool((guard[64 + V * C:] == 12345.0).all())
    del graph
    b.close()
