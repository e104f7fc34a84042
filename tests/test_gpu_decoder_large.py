"""The decoder operators on tensors of more than 4 GiB: what lies beyond is read and written where it belongs."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


class Table:
    """A context over tensors of the given shapes and types, all resident, as views of its arena."""

    def __init__(self, torch, **shapes):
        import paper_2203_15980_amd as dl
        self.i = {n: k for k, n in enumerate(shapes)}
        size = [int(np.prod(s)) * torch.empty((), dtype=t).element_size() for s, t in shapes.values()]
        self.arena = torch.empty(sum((n + 255) // 256 * 256 for n in size) + (1 << 20), dtype=torch.uint8, device="cuda:0")
        self.d = dl.Delta(self.arena, torch.cuda.current_stream().cuda_stream)
        self.d.bind(size)
        self.v = {}
        for (n, (s, t)), nb in zip(shapes.items(), size):
            at = self.d.alloc(self.i[n]) - self.arena.data_ptr()
            self.v[n] = self.arena[at:at + nb].view(t).reshape(s)

    def layer(self, op, rows, cin, cout, **kw):
        import paper_2203_15980_amd as dl
        base = dict(res=dl.NO_TENSOR, y2=dl.NO_TENSOR, y3=dl.NO_TENSOR, dtype=dl.DTYPE_BF16, N=1, H=rows, W=1, Cin=cin, Cout=cout, R=1, S=1, stride=1, op=op)
        return dl.LayerDesc(**{**base, **kw})

    def bwd(self, fwd, gy, gx, ws=None, gw=None):
        import paper_2203_15980_amd as dl
        return dl.BwdDesc(fwd=fwd, gy=gy, gpre=gy, gx=gx, gx_add=dl.NO_TENSOR, gw=gw.data_ptr() if gw is not None else None,
                          workspace=ws.data_ptr() if ws is not None else None, workspace_bytes=ws.numel() if ws is not None else 0)


def test_logprob_beyond_4_gib(torch_mod):
    import paper_2203_15980_amd as dl
    torch = torch_mod
    M, V, K = 70001, 32771, 3
    t = Table(torch, z=((M, V), torch.bfloat16), ids=((M,), torch.int64), y=((3, M), torch.float32), best=((M, K), torch.float32), which=((M, K), torch.int64),
              gy=((3, M), torch.float32), gz=((M, V), torch.bfloat16))
    z, ids = t.v["z"], t.v["ids"]
    for lo in range(0, M, 10000):
        z[lo:lo + 10000] = torch.randn(min(10000, M - lo), V, device="cuda:0", generator=None).mul_(2).to(torch.bfloat16)
    ids.copy_(torch.randint(0, V, (M,), device="cuda:0"))
    t.v["gy"].fill_(0.5)
    i = t.i
    L = t.layer(dl.OP_LOGPROB, M, V, K, x=i["z"], res=i["ids"], y=i["y"], y2=i["best"], y3=i["which"])
    t.d.recompute_segment([L])
    t.d.backward_segment([t.bwd(L, i["gy"], i["gz"])])
    t.d.sync()
    assert M * V * 2 > 4 << 30
    for r in (0, 35000, 65535, 65536, M - 2, M - 1):
        v = z[r].double()
        lp = torch.log_softmax(v, 0)
        p = lp.exp()
        H, lse = -(p * lp).sum(), torch.logsumexp(v, 0)
        got = t.v["y"][:, r].double()
        # sums of 32771 weights in fp32, depth 32 and the tree's: off by less than 150 e, the entropy by a few times that
        assert (got - torch.stack([lp[ids[r]], H, lse])).abs().max().item() <= 1e-4
        order = torch.sort(v, descending=True, stable=True).indices[:K]
        assert torch.equal(t.v["which"][r], order)
        hot = torch.zeros_like(p)
        hot[ids[r]] = 1
        want = 0.5 * (hot - p) - 0.5 * p * (lp + H) + 0.5 * p
        assert ((t.v["gz"][r].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5 * p + 1e-12).all()
    t.d.close()


def test_rmsnorm_and_rotary_beyond_4_gib(torch_mod):
    import paper_2203_15980_amd as dl
    torch = torch_mod
    M, C, D = 280001, 8192, 128
    d = dl.Delta()
    held = d.packed_bytes(M, C)
    d.close()
    big = ((M, C), torch.bfloat16)
    t = Table(torch, x=big, res=big, s=big, y=big, held=((held,), torch.uint8), gy=big, gx=big, pos=((M, 2), torch.int64), rot=big)
    g = torch.randn(997, C, device="cuda:0")
    for n, by in (("x", 1.0), ("res", 2.0), ("gy", 0.5)):       # rows repeat after 997, each tensor's from another one on
        for lo in range(0, M, 997):
            m = min(997, M - lo)
            t.v[n][lo:lo + m] = (torch.roll(g, int(by * 10), 0)[:m] * by).to(torch.bfloat16)
    t.v["pos"].copy_(torch.stack([torch.arange(M, device="cuda:0"), torch.arange(M, device="cuda:0") % 7], 1))
    gamma = torch.rand(C, device="cuda:0") + 0.5
    freq = torch.zeros(2, D // 2, device="cuda:0")
    freq[0, ::2], freq[1, 1::2] = 0.01, 0.3
    i = t.i
    N = t.layer(dl.OP_RMSNORM, M, C, C, x=i["x"], res=i["res"], y=i["y"], y2=i["s"], y3=i["held"], pack=dl.PACK_INT8, scale=gamma.data_ptr(), eps=1e-6)
    R = t.layer(dl.OP_ROTARY, M, C, C, x=i["y"], res=i["pos"], y=i["rot"], R=48, S=16, scale=freq.data_ptr())
    t.d.recompute_segment([N, R])
    ws, gw = torch.empty(max(t.d.backward_workspace(N), 256), dtype=torch.uint8, device="cuda:0"), torch.empty(C, device="cuda:0")
    t.d.backward_segment([t.bwd(N, i["gy"], i["gx"], ws, gw)])
    t.d.sync()
    assert M * C * 2 > 4 << 30
    at = (M * C + 15) // 16 * 16
    dg = torch.zeros(C, dtype=torch.float64, device="cuda:0")
    for lo in range(0, M, 20000):
        s, gy = t.v["s"][lo:lo + 20000].double(), t.v["gy"][lo:lo + 20000].double()
        dg += (gy * s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt()).sum(0)
        del s, gy
    # 547 rows to a workgroup's sum, and a tree over the workgroups: 700 e of the sum of magnitudes (at most M * 0.5 * max)
    assert (gw.double() - dg).abs().max().item() <= 700 * 2.0 ** -24 * M * 2.0
    for r in (0, 131071, 131072, 262143, 262144, M - 1):
        s = (t.v["x"][r].float() + t.v["res"][r].float()).to(torch.bfloat16)
        assert torch.equal(t.v["s"][r], s)
        s = s.double()
        inv = (s.square().mean() + 1e-6).rsqrt()
        y = s * inv * gamma.double()
        assert ((t.v["y"][r].double() - y).abs() <= 2.0 ** -8 * 1.01 * y.abs()).all()
        scale = torch.exp2(t.v["held"][at + r * (C // 32):at + (r + 1) * (C // 32)].double() - 127).repeat_interleave(32)
        q = t.v["held"][r * C:(r + 1) * C].view(torch.int8).double() * scale
        assert ((q - t.v["y"][r].double()).abs() <= scale / 2).all()
        gy, sh = t.v["gy"][r].double(), s * inv
        gg = gy * gamma.double()
        want = inv * (gg - sh * (gg * sh).mean())
        assert ((t.v["gx"][r].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 1e-5 * inv * gg.abs().max()).all()
        theta = (t.v["pos"][r].double()[:, None] * freq.double()).sum(0)
        h = t.v["y"][r].double().reshape(64, 2, D // 2)
        turned = torch.stack([h[:, 0] * theta.cos() - h[:, 1] * theta.sin(), h[:, 0] * theta.sin() + h[:, 1] * theta.cos()], 1)
        turned[48:] = h[48:]
        turned = turned.reshape(-1)
        assert ((t.v["rot"][r].double() - turned).abs() <= 2.0 ** -8 * turned.abs() + 1e-5).all()
    t.d.close()


def test_attention_beyond_4_gib(torch_mod):
    """90000 rows of 24576 channels in sequences of 60 and one of 1000 at the end: its rows lie beyond 4 GiB in x, gy and gx, in each of which the sequence's own
    definition in 64 bits is compared (tolerances: 1.5 % of a row's largest value, some times what two roundings to bf16 of p and of ds and one of the result leave)."""
    import paper_2203_15980_amd as dl
    torch = torch_mod
    H, D, n = 64, 128, 1000
    off = list(range(0, 89001, 60)) + [90000]
    off[-2] = 90000 - n
    M, W = 90000 + 3, 3 * H * D
    t = Table(torch, x=((M, W), torch.bfloat16), off=((len(off),), torch.int64), y=((M, H * D), torch.bfloat16), lse=((H, M), torch.float32), gy=((M, H * D), torch.bfloat16),
              gx=((M, W), torch.bfloat16))
    for lo in range(0, M, 10000):
        t.v["x"][lo:lo + 10000] = torch.randn(min(10000, M - lo), W, device="cuda:0").to(torch.bfloat16)
        t.v["gy"][lo:lo + 10000] = torch.randn(min(10000, M - lo), H * D, device="cuda:0").to(torch.bfloat16)
    t.v["off"].copy_(torch.tensor(off))
    i = t.i
    L = t.layer(dl.OP_ATTENTION_PACKED, M, W, H * D, x=i["x"], res=i["off"], y=i["y"], y2=i["lse"], R=H, S=H, flags=dl.ATTENTION_CAUSAL)
    t.d.recompute_segment([L])
    ws = torch.empty(t.d.backward_workspace(L), dtype=torch.uint8, device="cuda:0")
    t.d.backward_segment([t.bwd(L, i["gy"], i["gx"], ws)])
    t.d.sync()
    assert M * W * 2 > 4 << 30
    assert not t.v["gx"][90000:].any() and not t.v["y"][90000:].any() and not t.v["lse"][:, 90000:].any()
    for a, b in ((off[-2], off[-1]), (off[700], off[701])):
        x, gy = t.v["x"][a:b].double(), t.v["gy"][a:b].double()
        keep = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda:0").tril()
        for h in (0, 37, 63):
            c = [slice((k * H + h) * D, (k * H + h + 1) * D) for k in range(3)]
            q, k, v, g = x[:, c[0]].contiguous(), x[:, c[1]].contiguous(), x[:, c[2]].contiguous(), gy[:, c[0]].contiguous()
            s = (q @ k.t().contiguous() * D ** -0.5).masked_fill(~keep, -float("inf"))
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            y = p @ v
            ds = p * (g @ v.t().contiguous() - (g * y).sum(1, keepdim=True)) * D ** -0.5
            assert (t.v["lse"][h, a:b].double() - lse).abs().max().item() <= 1e-4
            for got, want in ((t.v["y"][a:b, c[0]], y), (t.v["gx"][a:b, c[0]], ds @ k), (t.v["gx"][a:b, c[1]], ds.t().contiguous() @ q), (t.v["gx"][a:b, c[2]], p.t().contiguous() @ g)):
                assert ((got.double() - want).abs() <= 0.015 * want.abs().amax()).all()
    t.d.close()


def attention_of_some_heads(torch, off, M, H, D, heads, causal, seed):
    """Both ways with as many key heads as query heads; `heads` of them against 64 bits, the rows of no sequence against zero."""
    import paper_2203_15980_amd as dl
    from decoder_util import check_attention
    from oracle import decoder as od
    W = 3 * H * D
    t = Table(torch, x=((M, W), torch.bfloat16), off=((len(off),), torch.int64), y=((M, H * D), torch.bfloat16), lse=((H, M), torch.float32), gy=((M, H * D), torch.bfloat16),
              gx=((M, W), torch.bfloat16))
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    for n in ("x", "gy"):
        for lo in range(0, M, 16):
            part = t.v[n][lo:lo + 16]
            part.copy_(torch.randn(part.shape, device="cuda:0", generator=g))
    t.v["off"].copy_(torch.tensor(off))
    for n in ("y", "lse", "gx"):
        t.v[n].fill_(float("nan"))
    i = t.i
    L = t.layer(dl.OP_ATTENTION_PACKED, M, W, H * D, x=i["x"], res=i["off"], y=i["y"], y2=i["lse"], R=H, S=H, flags=dl.ATTENTION_CAUSAL if causal else 0)
    t.d.recompute_segment([L])
    ws = torch.empty(t.d.backward_workspace(L), dtype=torch.uint8, device="cuda:0")
    t.d.backward_segment([t.bwd(L, i["gy"], i["gx"], ws)])
    t.d.sync()
    assert not t.v["gx"][off[-1]:].any() and not t.v["y"][off[-1]:].any() and not t.v["lse"][:, off[-1]:].any()
    some = lambda n, k: np.concatenate([t.v[n][:, (j * H + h) * D:(j * H + h + 1) * D].double().cpu().numpy() for j in range(k) for h in heads], axis=1)      # noqa: E731
    x, gy = some("x", 3), some("gy", 1)
    x[off[-1]:], gy[off[-1]:] = 0, 0
    o = dict(y=some("y", 1), gx=some("gx", 3), lse=t.v["lse"][list(heads)].double().cpu().numpy())
    check_attention(o, od.attention(x, np.asarray(off), len(heads), len(heads), D, causal, gy), len(heads), D, int(np.diff(off).max()))
    t.d.close()


@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_rows_of_17_megabytes(torch_mod, causal):
    """A workgroup's 256 rows of values lie further apart than 32 bits reach: 255 rows of 17.66 MB are 4.5e9 bytes."""
    H, D = 23000, 128
    assert 255 * 3 * H * D * 2 > 2 ** 32
    attention_of_some_heads(torch_mod, [0, 255], 256, H, D, (0, 11111, 22999), causal, 40)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("M,seqs,D", [(32, 32765, 64), (2048, 32700, 128)])
def test_attention_of_as_many_sequences_as_a_launch_takes(torch_mod, causal, M, seqs, D):
    """256 heads: both gradients in one launch would be 32768 x 512 workgroups of 256 threads, 2^32, with 32 rows; with 2048 the gradient of keys and values takes 32710 x 256 of
    512 threads, 2^32 - 7602176."""
    H = 256
    lens = np.zeros(seqs, np.int64)
    lens[[0, 1, 63, 64, 4095, 4096, seqs // 2, seqs - 2, seqs - 1]] = np.array([5, 1, 0, 2, 3, 1, 4, 6, 7]) if M == 32 else np.array([300, 1, 65, 129, 31, 32, 700, 257, 500])
    off = np.concatenate([[0], np.cumsum(lens)])
    assert off[-1] <= M
    attention_of_some_heads(torch_mod, off.tolist(), M, H, D, (0, 100, 255), causal, 41)
