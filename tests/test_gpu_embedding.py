"""Embedding lookup and its gradient through the C ABI.  Lookup: one fp32 product, rounded once: equality.  Gradient:
on whole numbers every sum is exact in fp32: equality; on others a chain's rounding."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, storage, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def _ids(kind, n, V, rng):
    if kind == "same":
        return np.full(n, V // 2, np.int64)
    if kind == "none":
        return np.where(rng.random(n) < 0.5, -1, V).astype(np.int64)
    if kind == "bad":                                        # ids outside the table, also by more than 32 bits, among good ones
        ids = rng.integers(0, V, n)
        bad = np.array([-1, V, V + 1, 2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 32, 2 ** 63 - 1, -2 ** 63], np.int64)
        return np.where(rng.random(n) < 0.4, bad[rng.integers(0, len(bad), n)], ids)
    if kind == "runs":                                       # a few ids, their runs' ends on both sides of windows
        return rng.integers(0, min(V, 5), n)
    if kind == "falling":
        return np.minimum(V - 1, np.floor((V + 3.0) ** rng.random(n) - 1)).astype(np.int64)
    return rng.integers(0, V, n)


# tokens on both sides of: one wavefront, the sort in one workgroup, a sort block, several; ids of 1 to 22 bits
GRADIENT = [(1, 1, 8, "any"), (1, 100, 768, "any"), (63, 7, 64, "any"), (64, 2, 8, "any"), (65, 30522, 768, "any"), (77, 300, 1000, "bad"),
            (31, 5, 16, "same"), (32, 5, 16, "same"), (95, 5, 2056, "same"), (2047, 1000, 64, "falling"), (2048, 3, 72, "runs"),
            (2048, 1000, 64, "same"), (2049, 1000, 64, "falling"), (2049, 1, 8, "any"), (2050, 70000, 8, "any"), (3070, 2, 64, "runs"),
            (4096, 257, 64, "bad"), (5000, 4, 520, "runs"), (5000, 30522, 768, "falling"), (9000, 50, 64, "none"), (16384, 30522, 96, "falling"),
            (16384, 100, 64, "same"), (20000, 2 ** 17, 8, "any"), (40001, 1000, 16, "falling"), (70000, 2 ** 22 - 1, 8, "bad"), (300, 2 ** 22 - 1, 8, "any"),
            (2100, 33, 8192, "runs"), (1024, 300, 64, "falling"), (1025, 300, 64, "falling"), (4096, 2 ** 18, 8, "any"), (4097, 2 ** 18 - 1, 8, "falling"),
            (16384, 2 ** 20, 8, "bad"), (16385, 3, 64, "same"), (16401, 7, 64, "runs"), (33, 7, 64, "same"), (48, 3, 64, "runs"), (65537, 3, 8, "same"),
            (16383, 300, 16, "falling"), (65536, 100, 8, "falling"), (65537, 2 ** 17, 16, "bad"), (200001, 3000, 8, "falling"),
            (4096, 2 ** 20 - 1, 8, "any"), (4096, 2 ** 20, 8, "bad"), (8192, 2 ** 19 - 1, 8, "bad"), (8191, 2 ** 19, 8, "any"), (8192, 2 ** 19, 8, "falling"),
            (8193, 300, 64, "falling"), (8192, 3, 64, "runs"), (8192, 100, 64, "same"), (6001, 1, 8, "any"), (4095, 30, 64, "none"),
            (2 ** 20, 5000, 8, "falling"), (2 ** 20 + 1, 2 ** 22 - 1, 8, "bad"), (2 ** 20 + 8191, 5000, 8, "falling")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,C,kind", GRADIENT)
def test_gradient_is_exact_on_whole_numbers(torch_mod, n, V, C, kind, dtype):
    print("tokens", n, "V", V, "C", C, kind, dtype, flush=True)
    rng = np.random.default_rng(n + V + C)
    ids = _ids(kind, n, V, rng)
    gi = rng.integers(-64, 65, (n, C)).astype(np.float32)
    gy = storage(gi, dtype)
    scale = np.exp2(rng.integers(-2, 3, C)).astype(np.float32)
    b = Bench(torch_mod, [ids.nbytes, gy.nbytes, gy.nbytes])
    b.put(0, ids); b.put(2, gy)
    s = b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, dtype, w=s.data_ptr(), scale=s.data_ptr())     # the gradient does not read the table
    need = b.d.backward_workspace(fwd)
    ws, whole = b.workspace(need)
    gw, guard = b.guarded(V * C)
    desc = b.bwd(fwd, 2, gw=gw, ws=ws)
    assert b.d.backward_kernel(desc) == "gw: embedding"
    there = (ids >= 0) & (ids < V)
    want = np.zeros((V, C), np.float32)
    np.add.at(want, ids[there], gi[there])
    want *= scale
    for fill in (0x7F, 0x00):                                # whatever the workspace holds
        ws.fill_(fill)
        gw.fill_(float("nan"))
        torch_mod.cuda.synchronize()
        b.d.backward_segment([desc])
        b.d.sync()
        got = gw.cpu().numpy().reshape(V, C)
        assert np.array_equal(got, want), (int((got != want).sum()), got.size)
    assert (guard[:64] == 12345.0).all() and (guard[64 + V * C:] == 12345.0).all() and (whole[max(need, 256):] == 0x7F).all()
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("n,V,C,kind", [(77, 50, 768, "falling"), (5000, 300, 256, "falling"), (16384, 7, 64, "runs")])
def test_gradient_matches_float64_and_repeats_its_bits(torch_mod, n, V, C, kind):
    rng = np.random.default_rng(n)
    ids = _ids(kind, n, V, rng)
    gy = storage(rng.normal(size=(n, C)), "f32")
    scale = rng.uniform(0.5, 30, C).astype(np.float32)
    b = Bench(torch_mod, [ids.nbytes, gy.nbytes, gy.nbytes])
    b.put(0, ids); b.put(2, gy)
    s = b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, "f32", w=s.data_ptr(), scale=s.data_ptr())
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    runs = []
    for _ in range(3):
        gw, _ = b.guarded(V * C)
        b.d.backward_segment([b.bwd(fwd, 2, gw=gw, ws=ws)])
        b.d.sync()
        runs.append(gw.cpu().numpy().reshape(V, C))
    assert np.array_equal(runs[0], runs[1]) and np.array_equal(runs[0], runs[2])
    want, size = ro.embedding_bwd(ids, gy, scale, V), ro.embedding_bwd(ids, np.abs(gy), scale, V)
    longest = np.bincount(ids, minlength=V).max()            # no chain is longer than an id's tokens
    assert (np.abs(runs[0] - want) <= (min(longest, 600) + 4) * EPS24 * size).all()
    b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,C,kind", [(1, 1, 8, "any"), (77, 30522, 768, "any"), (300, 11, 1000, "bad"), (9, 5, 8192, "any"), (5, 4, 2056, "bad"),
                                        (20000, 300, 64, "falling"), (4097, 2 ** 22 - 1, 8, "any")])
def test_lookup_is_exact(torch_mod, n, V, C, kind, dtype):
    print("tokens", n, "V", V, "C", C, kind, dtype, flush=True)
    rng = np.random.default_rng(n + C)
    ids = _ids(kind, n, V, rng)
    w = storage(rng.normal(size=(V, C)), dtype)
    scale = rng.uniform(0.1, 30, C).astype(np.float32)
    y = w[:1].nbytes * n
    b = Bench(torch_mod, [ids.nbytes, y])
    b.put(0, ids)
    wd, s = b.dev(w.view(np.int16) if dtype == "bf16" else w), b.dev(scale)
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, dtype, w=wd.data_ptr(), scale=s.data_ptr())
    assert b.d.layer_kernel(fwd) == "embedding " + dtype
    b.d.recompute_segment([fwd])
    got = b.get(1, w.dtype, (n, C))
    there = (ids >= 0) & (ids < V)
    f = values(w[np.where(there, ids, 0)], dtype).astype(np.float32) * scale
    want = storage(np.where(there[:, None], f, np.float32(0)), dtype)
    assert np.array_equal(got, want)
    assert b.untouched()
    b.close()


def test_evicted_embedding_is_looked_up_again(torch_mod):
    n, V, C = 200, 64, 128
    rng = np.random.default_rng(2)
    ids, w = rng.integers(0, V, n), storage(rng.normal(size=(V, C)), "bf16")
    b = Bench(torch_mod, [ids.nbytes, n * C * 2])
    b.put(0, ids)
    wd, s = b.dev(w.view(np.int16)), b.dev(np.full(C, 2.0, np.float32))
    fwd = b.layer(b.dl.OP_EMBEDDING, n, V, C, 0, 1, w=wd.data_ptr(), scale=s.data_ptr())
    b.d.recompute_segment([fwd])
    first = b.get(1, np.uint16, (n, C)).copy()
    b.d.release(1, b.dl.EV_EVICT)
    b.d.recompute_segment([fwd])
    b.at[1] = b.d.tensor_ptr(1) - b.arena.data_ptr()
    assert np.array_equal(b.get(1, np.uint16, (n, C)), first)
    b.close()


def test_refusals(torch_mod):
    n, V, C = 16, 10, 64
    b = Bench(torch_mod, [n * 8, n * C * 2, n * C * 2, n * C * 2, n * 12 * 2])
    dl = b.dl
    b.put(0, np.zeros(n, np.int64))
    one = torch_mod.ones(4096, device="cuda:0")
    p = one.data_ptr()

    def refused(call, desc, status=dl.ERR_INVALID):
        with pytest.raises(dl.DeltaError) as e:
            call([desc])
        assert e.value.status == status, e.value.message
    fw, bw = b.d.recompute_segment, b.d.backward_segment
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, scale=p))                # no table, no factors, misaligned ones
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p + 8, scale=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p, scale=p + 4))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, 12, 0, 4, w=p, scale=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, 0, 0, 1, w=p, scale=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, 0, C, 0, 1, w=p, scale=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, 2 ** 22, C, 0, 1, w=p, scale=p))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 1, 2, w=p, scale=p))           # ids of the wrong size
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p, scale=p, res=2))
    refused(fw, b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p, scale=p, pack=1))
    fwd = b.layer(dl.OP_EMBEDDING, n, V, C, 0, 1, w=p, scale=p)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, _ = b.guarded(V * C)
    refused(bw, b.bwd(fwd, 2, ws=ws))
    refused(bw, b.bwd(fwd, 2, gw=gw))
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws, gx=3))
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws, add=3))
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws, gpre=3))
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws, gy_masked=1))
    refused(bw, b.bwd(fwd, 0, gw=gw, ws=ws))
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws, workspace_bytes=ws.numel() - 256))
    refused(bw, b.bwd(fwd, 2, gw=gw[2:], ws=ws))
    b.d.release(2, dl.EV_FREE)
    refused(bw, b.bwd(fwd, 2, gw=gw, ws=ws), dl.ERR_STATE)
    b.close()
