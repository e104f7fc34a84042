"""The embedding at its edges: factors that are infinities or NaN."""
import numpy as np
import pytest

from rowops_util import Bench, storage, values

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
