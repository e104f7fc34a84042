"""Layer normalisation in bf16 over more rows than one launch holds threads for (2^26 wavefronts), and over more than 2^31."""
import numpy as np
import pytest

from rowops_util import EPS24, Bench, half_step

pytestmark = pytest.mark.gpu

EPS, C = 1e-5, 8


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def _context(torch, N, H, c, es=2):
    """A context whose tensors (0 .. 3, the shape's size) are never made resident, and the layer's fields."""
    import paper_2203_15980_amd as dl
    arena = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    d = dl.Delta(arena, torch.cuda.current_stream().cuda_stream)
    d.bind([N * H * c * es] * 4)
    one = torch.ones(2048, device="cuda:0")
    layer = dl.LayerDesc(x=0, res=dl.NO_TENSOR, y=1, dtype=dl.DTYPE_BF16 if es == 2 else dl.DTYPE_F32, N=N, H=H, W=1, Cin=c, Cout=c, R=1, S=1, stride=1, pad=0,
                         relu=0, op=dl.OP_LAYERNORM, scale=one.data_ptr(), shift=one.data_ptr(), eps=EPS)
    return dl, d, layer, (arena, one)


def test_what_is_taken_and_refused(torch_mod):
    for N, H, c, es, forward, backward in ((32767, 65536, 8, 2, True, True), (32769, 65536, 8, 2, True, False), (131071, 65536, 8, 2, True, False),
                                           (131073, 65536, 8, 2, False, False), (32769, 65536, 8, 4, False, False), (32769, 65536, 2112, 2, False, False)):
        dl, d, layer, keep = _context(torch_mod, N, H, c, es)
        if forward:
            assert d.layer_kernel(layer) == "layernorm bf16"
        else:
            with pytest.raises(dl.DeltaError) as e:
                d.layer_kernel(layer)
            assert e.value.status == dl.ERR_INVALID
        desc = dl.BwdDesc(fwd=layer, gy=2, gpre=2, gx=3, gx_add=dl.NO_TENSOR, gw=None, workspace=None, workspace_bytes=0)
        if backward:
            assert d.backward_kernel(desc) == "gx: layernorm" and d.backward_workspace(layer) > 0
        else:
            for call in (lambda: d.backward_kernel(desc), lambda: d.backward_workspace(layer), lambda: d.backward_segment([desc])):
                with pytest.raises(dl.DeltaError) as e:
                    call()
                assert e.value.status == dl.ERR_INVALID
        d.close()


@pytest.mark.parametrize("rows", [(1 << 25) + 3, (1 << 26) + 5, (1 << 31) + (1 << 25) + 3])
def test_every_row_is_normalised(torch_mod, rows):
    """x[m] is one of 4096 rows, by m modulo 4096 (and so by its place in any launch, which holds a multiple of them): y against those rows' results."""
    torch, nb = torch_mod, rows * C * 2
    if torch.cuda.mem_get_info()[0] < 3 * nb:
        pytest.skip("needs %d GB of device memory" % (3 * nb >> 30))
    print("rows", rows, flush=True)
    b = Bench(torch, [nb, nb])
    view = lambda i: b.arena[b.at[i]:b.at[i] + nb].view(torch.bfloat16).view(rows, C)          # noqa: E731
    some = torch.randn(4096, C, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(7)).to(torch.bfloat16)
    last = torch.randn(3, C, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(8)).to(torch.bfloat16)
    x, whole = view(0), rows // 4096 * 4096
    assert rows - whole >= 3
    x[:whole].view(-1, 4096, C).copy_(some[None])
    x[whole:] = some[:rows - whole]
    x[-3:] = last                                            # the last rows are others
    g = b.dev(np.linspace(0.5, 1.5, C).astype(np.float32))
    h = b.dev(np.linspace(-1, 1, C).astype(np.float32))
    torch.cuda.synchronize()
    n = 1 if rows < 1 << 31 else next(k for k in range(3, 1 << 16, 2) if rows % k == 0)        # N * H: each dimension has 31 bits
    fwd = b.layer(b.dl.OP_LAYERNORM, rows // n, C, C, 0, 1, N=n, scale=g.data_ptr(), shift=h.data_ptr(), eps=EPS)
    b.d.recompute_segment([fwd])
    b.d.sync()

    def want(v):
        v = v.double()
        c = v - v.mean(1, keepdim=True)
        r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
        y = c * r * g.double() + h.double()
        return y, half_step("bf16") * y.abs() + 40 * EPS24 * ((v.abs().amax(1, keepdim=True) * r + (c * r).abs()) * g.double() + h.double().abs())
    y = view(1)
    first = y[:4096].clone()                                 # the repeats are equal bits; the first ones and the last rows are right
    ref, tol = want(x[:4096])
    assert bool(((first.double() - ref).abs() <= tol).all())
    ref, tol = want(x[-3:])
    assert bool(((y[-3:].double() - ref).abs() <= tol).all())
    bits, step = first.view(torch.int64), 1 << 12
    for at in range(0, whole // 4096, step):
        got = y[at * 4096:min(whole, (at + step) * 4096)].view(torch.int64).view(-1, *bits.shape)
        assert bool((got == bits[None]).all()), at
    if whole < rows - 3:
        assert bool((y[whole:-3].view(torch.int64) == bits[:rows - 3 - whole]).all())
    b.close()
