"""The decoder operators together, as a training step uses them: embedding, normalisation, projections, rotary positions, attention over packed sequences, a
feed-forward whose input is kept in 8 bits, log probabilities of the next tokens; the backward pass through all of it; released and recomputed, captured into a graph and
replayed, two contexts side by side.  And what the calls refuse, and leave as it was.

Each tensor is compared with float64 on the operands that the GPU itself stored (decoder_util, rowops_util)."""
import numpy as np
import pytest

from oracle import decoder as od, rowops as ro
from decoder_util import check_attention, logprob_noise, rmsnorm_noise, run_attention, run_logprob
from rowops_util import EPS24, Bench, storage, values

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def near(got, ref, tol, what=""):
    assert (np.abs(got - ref) <= tol).all(), (what, float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max()))


class Decoder:
    """x0 = embedding(ids); n1 = norm(x0); qkv = n1 wq; rot; ctx; ao = ctx wo; (s2, n2, c.n2) = norm(ao + x0); h = relu(n2 w1); f = h w2; (s3, n3) = norm(f + s2);
    z = n3 wv; lp = log probabilities of the next ids."""
    H, G, D, K = 4, 2, 64, 3

    def __init__(self, torch, lens=(70, 1, 129), behind=5, V=192, FF=128, seed=1, stream=None, causal=True):
        import paper_2203_15980_amd as dl
        self.dl, self.torch = dl, torch
        rng = np.random.default_rng(seed)
        H, G, D, K = self.H, self.G, self.D, self.K
        C, Q = H * D, (H + 2 * G) * D
        self.C, self.Q, self.V, self.FF, self.causal = C, Q, V, FF, causal
        self.off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        T = self.T = int(self.off[-1]) + behind
        self.longest = max(lens)
        wide = dict(x0=C, n1=C, qkv=Q, rot=Q, ctx=C, ao=C, s2=C, n2=C, h=FF, f=C, s3=C, n3=C, z=V)
        self.wide = {**wide, **{"g." + n: w for n, w in wide.items()}, "gp.h": FF}
        names = ["ids", "next", "off", "pos"] + list(self.wide) + ["lse", "lp", "best", "which", "g.lp", "c.n2"]
        size = dict(ids=T * 8, next=T * 8, off=self.off.size * 8, pos=T * 16, lse=H * T * 4, lp=T * 12, best=T * K * 4, which=T * K * 8, **{"g.lp": T * 12, "c.n2": ro.packed_bytes(T, C)})
        size.update({n: T * w * 2 for n, w in self.wide.items()})
        self.i = i = {n: k for k, n in enumerate(names)}
        b = self.b = Bench(torch, [size[n] for n in names], stream=stream)
        self.ids, self.next = rng.integers(0, V, T), rng.integers(0, V, T)
        self.ids[T - behind:] = self.next[T - behind:] = -1
        self.pos = np.stack([np.concatenate([np.arange(n) for n in lens] + [np.zeros(behind, int)]), rng.integers(0, 9, T)], axis=1)
        self.glp = (rng.normal(size=(3, T)) / 4).astype(np.float32)
        b.put(i["ids"], self.ids.astype(np.int64))
        b.put(i["next"], self.next.astype(np.int64))
        b.put(i["off"], self.off)
        b.put(i["pos"], self.pos.astype(np.int64))
        b.put(i["g.lp"], self.glp)
        P = self.P = {"table": storage(rng.normal(size=(V, C)), "bf16")}
        lin = dict(q=(C, Q), o=(C, C), u=(C, FF), d=(FF, C), v=(C, V))
        for k, (a, c) in lin.items():
            P["w" + k] = storage(rng.normal(size=(c, a)) / np.sqrt(a), "bf16")
            P["one" + k], P["b" + k] = np.ones(c, np.float32), (rng.normal(size=c) * 0.02).astype(np.float32)
        for k in "123":
            P["g" + k] = rng.uniform(0.5, 1.5, C).astype(np.float32)
        P["scale"] = np.ones(C, np.float32)
        P["freq"] = np.zeros((2, D // 2), np.float32)
        P["freq"][0, ::2], P["freq"][1, 1::2] = 100.0 ** (-np.arange(D // 4) / (D // 4)), 0.25
        self.dev = {k: b.dev(v.view(np.int16) if v.dtype == np.uint16 else v) for k, v in P.items()}
        self.wt = {k: b.dev(np.zeros(c, np.int16)) for k, c in lin.items()}
        p, none = (lambda n: self.dev[n].data_ptr()), dl.NO_TENSOR
        L = lambda op, x, y, cin, cout, **kw: b.layer(op, T, cin, cout, i[x], i[y], **kw)      # noqa: E731
        line = lambda k, x, y, **kw: L(dl.OP_CONV, x, y, *lin[k], w=p("w" + k), scale=p("one" + k), shift=p("b" + k), **kw)    # noqa: E731
        norm = lambda k, x, y, **kw: L(dl.OP_RMSNORM, x, y, C, C, scale=p("g" + k), eps=EPS, **{**dict(y2=none, y3=none), **kw})   # noqa: E731
        F = self.F = dict(
            emb=L(dl.OP_EMBEDDING, "ids", "x0", V, C, w=p("table"), scale=p("scale")), n1=norm("1", "x0", "n1"), q=line("q", "n1", "qkv"),
            rot=L(dl.OP_ROTARY, "qkv", "rot", Q, Q, res=i["pos"], y2=none, y3=none, R=H + G, S=G, scale=p("freq")),
            att=L(dl.OP_ATTENTION_PACKED, "rot", "ctx", Q, C, res=i["off"], y2=i["lse"], y3=none, R=H, S=G, flags=dl.ATTENTION_CAUSAL if causal else 0),
            o=line("o", "ctx", "ao"), n2=norm("2", "ao", "n2", res=i["x0"], y2=i["s2"], y3=i["c.n2"], pack=dl.PACK_INT8), u=line("u", "n2", "h", relu=1),
            d=line("d", "h", "f"), n3=norm("3", "f", "n3", res=i["s2"], y2=i["s3"]), v=line("v", "n3", "z"),
            lp=L(dl.OP_LOGPROB, "z", "lp", V, K, res=i["next"], y2=i["best"], y3=i["which"]))
        self.forward = list(F.values())
        held = dl.LayerDesc.from_buffer_copy(F["u"])
        held.x, held.pack = i["c.n2"], dl.PACK_INT8
        need = [b.d.backward_workspace(d) for d in self.forward if d.op != dl.OP_ROTARY] + [b.d.backward_workspace(held)]
        self.ws, self.whole = b.workspace(2 * max(need) + 256)
        self.gw = {n: b.guarded(int(np.prod(s)))[0] for n, s in dict(emb=(V, C), n1=C, n2=C, n3=C, q=(Q, C), o=(C, C), u=(FF, C), d=(C, FF), v=(V, C)).items()}
        for k in lin:
            b.d.bwd_weights(F[k], self.wt[k].data_ptr())
        B = lambda f, gy, gx, w=None, k=None, add=None, **kw: b.bwd(f, i[gy], gx=i[gx] if gx else None, add=i[add] if add else None,      # noqa: E731
                                                                    gw=self.gw[w] if w else None, ws=self.ws, **({"wt": self.wt[k].data_ptr()} if k else {}), **kw)
        self.backward = [
            B(F["lp"], "g.lp", "g.z"), B(F["v"], "g.z", "g.n3", "v", "v"), B(F["n3"], "g.n3", "g.s3", "n3"), B(F["d"], "g.s3", "g.h", "d", "d"),
            B(held, "g.h", "g.n2", "u", "u", gpre=i["gp.h"]), B(F["n2"], "g.n2", "g.s2", "n2", add="g.s3"), B(F["o"], "g.s2", "g.ctx", "o", "o"), B(F["att"], "g.ctx", "g.rot"),
            B(F["rot"], "g.rot", "g.qkv"), B(F["q"], "g.qkv", "g.n1", "q", "q"), B(F["n1"], "g.n1", "g.x0", "n1", add="g.s2"), B(F["emb"], "g.x0", None, "emb")]

    def run(self):
        self.b.d.recompute_segment(self.forward)
        self.b.d.backward_segment(self.backward)
        self.b.d.backward_join()

    USED = ["g." + n for n in ("z", "n3", "s3", "h", "n2", "s2", "ctx", "rot", "qkv", "n1", "x0")] + ["gp.h"]
    MADE = ["x0", "n1", "qkv", "rot", "ctx", "ao", "s2", "n2", "h", "f", "s3", "n3", "z"]

    def everything(self):
        self.b.d.sync()
        o = {n: values(self.b.get(self.i[n], np.uint16, (self.T, self.wide[n])), "bf16").copy() for n in self.MADE + self.USED}
        o["lse"] = self.b.get(self.i["lse"], np.float32, (self.H, self.T)).astype(np.float64)
        o["lp"], o["best"] = (self.b.get(self.i[n], np.float32, s).astype(np.float64) for n, s in (("lp", (3, self.T)), ("best", (self.T, self.K))))
        o["which"], o["held"] = self.b.get(self.i["which"], np.int64, (self.T, self.K)).copy(), self.b.get(self.i["c.n2"], np.uint8, (-1,)).copy()
        o.update({"gw." + n: t.cpu().numpy().astype(np.float64) for n, t in self.gw.items()})
        return o

    def check(self, o):
        P = {k: (values(v, "bf16") if v.dtype == np.uint16 else v.astype(np.float64)) for k, v in self.P.items()}
        T, half = self.T, 2.0 ** -8
        near(o["x0"], ro.embedding(self.ids, P["table"], P["scale"]), half * np.abs(ro.embedding(self.ids, P["table"], P["scale"])))
        line = dict(q=("n1", "qkv"), o=("ctx", "ao"), u=("n2", "h"), d=("h", "f"), v=("n3", "z"))
        for k, (x, y) in line.items():
            want = o[x] @ P["w" + k].T + P["b" + k]
            noise = o[x].shape[1] * EPS24 * (np.abs(o[x]) @ np.abs(P["w" + k]).T + np.abs(P["b" + k]))
            want = np.maximum(want, 0) if k == "u" else want
            near(o[y], want, half * np.abs(want) + noise, y)
        for k, s, y, gy, gx, add in (("1", "x0", "n1", "g.n1", "g.x0", "g.s2"), ("2", "s2", "n2", "g.n2", "g.s2", "g.s3"), ("3", "s3", "n3", "g.n3", "g.s3", None)):
            fwd, ngx, ndg = rmsnorm_noise(o[s], o[gy], P["g" + k], EPS)
            want = od.rmsnorm(o[s], P["g" + k], EPS)
            near(o[y], want, (half + fwd) * np.abs(want), y)
            a = o[add] if add else np.zeros((T, self.C))
            want, dg = od.rmsnorm_bwd(o[s], o[gy], P["g" + k], EPS, a)
            near(o[gx], want, (half + EPS24) * np.abs(want) + ngx + 2 * EPS24 * np.abs(a), gx)
            near(o["gw.n" + k], dg, ndg, "dgamma")
        for s, a, r in (("s2", "ao", "x0"), ("s3", "f", "s2")):
            near(o[s], o[a] + o[r], (half + EPS24) * np.abs(o[a] + o[r]), s)
        pay, sc = ro.pack(o["n2"], "int8")
        got = ro.split_packed(o["held"], T, self.C)
        assert np.array_equal(ro.unpack(*got, "int8"), ro.unpack(pay, sc, "int8"))
        theta = od.angles(self.pos, self.P["freq"])
        for x, y, sign in (("qkv", "rot", 1), ("g.rot", "g.qkv", -1)):
            want = od.rotary(o[x], sign * theta, self.H + self.G, self.D, False)
            near(o[y], want, half * np.abs(want) + 10 * EPS24 * 2 * np.abs(o[x]).max(axis=1, keepdims=True), y)
        ref = od.attention(o["rot"], self.off, self.H, self.G, self.D, self.causal, o["g.ctx"])
        check_attention(dict(y=o["ctx"], lse=o["lse"], gx=o["g.rot"]), ref, self.H, self.D, self.longest)
        y, best, which = od.logprob(o["z"], self.next, self.K)
        lp, nH, nl = logprob_noise(o["z"], y)
        d = o["z"].max(axis=1) - o["z"].min(axis=1)
        for k, tol in enumerate((lp(d), nH, nl)):
            near(o["lp"][k], y[k], tol, "lp")
        assert np.array_equal(o["which"], which)
        near(o["best"], best, lp(d)[:, None] + 0 * best, "best")
        g = self.glp.astype(np.float64)
        want = od.logprob_bwd(o["z"], self.next, g)
        near(o["g.z"], want, half * np.abs(want) + 1e-5 * np.abs(g).sum(axis=0)[:, None] * 0.1, "g.z")      # p is off by less than 2^-20: what half a step does not cover
        back = dict(v=("g.z", "g.n3", "n3"), d=("g.s3", "g.h", "h"), u=("gp.h", "g.n2", None), o=("g.s2", "g.ctx", "ctx"), q=("g.qkv", "g.n1", "n1"))
        for k, (gy, gx, x) in back.items():
            want = o[gy] @ P["w" + k]
            near(o[gx], want, half * np.abs(want) + o[gy].shape[1] * EPS24 * (np.abs(o[gy]) @ np.abs(P["w" + k])), gx)
            X = o[x] if x else ro.unpack(pay, sc, "int8")
            near(o["gw." + k].reshape(-1, X.shape[1]), o[gy].T @ X, T * EPS24 * (np.abs(o[gy]).T @ np.abs(X)) + 1e-30, "gw." + k)
        assert np.array_equal(o["gp.h"], np.where(o["h"] > 0, o["g.h"], 0))
        size = ro.embedding_bwd(self.ids, np.abs(o["g.x0"]), P["scale"], self.V)
        near(o["gw.emb"].reshape(self.V, self.C), ro.embedding_bwd(self.ids, o["g.x0"], P["scale"], self.V), T * EPS24 * size)


@pytest.mark.parametrize("lens,behind,V,FF,causal", [((70, 1, 129), 5, 192, 128, True), ((1,), 0, 64, 64, True), ((33, 0, 400), 0, 320, 256, False)])
def test_step_released_and_recomputed(torch_mod, lens, behind, V, FF, causal):
    print("decoder", lens, behind, V, FF, causal, flush=True)
    s = Decoder(torch_mod, lens, behind, V, FF, seed=sum(lens), causal=causal)
    s.run()
    want = s.everything()
    s.check(want)
    d, dl = s.b.d, s.dl
    for n in s.MADE + s.USED + ["lse", "lp", "best", "which", "c.n2"]:
        d.release(s.i[n], dl.EV_EVICT)
    d.recompute_segment(s.forward)
    for n in ("x0", "n1", "qkv", "ao", "f", "n2"):                                 # nothing of these is read by the gradients
        if n not in ("x0", "n1"):
            d.release(s.i[n], dl.EV_EVICT)
    d.release(s.i["lse"], dl.EV_OFFLOAD)
    d.prefetch(s.i["lse"])
    for g in s.gw.values():
        g.fill_(float("nan"))
    torch_mod.cuda.synchronize()
    d.backward_segment(s.backward)
    d.backward_join()
    d.sync()
    for n in s.USED:
        s.b.at[s.i[n]] = d.tensor_ptr(s.i[n]) - s.b.arena.data_ptr()
        assert np.array_equal(values(s.b.get(s.i[n], np.uint16, (s.T, s.wide[n])), "bf16"), want[n]), n
    for n, g in s.gw.items():
        assert np.array_equal(g.cpu().numpy().astype(np.float64), want["gw." + n]), n
    s.b.close()


def test_step_captured_into_graphs_and_replayed(torch_mod):
    """Two graphs of two contexts, their replays in turn and with eager work of both between them."""
    torch = torch_mod
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Decoder(torch, (70, 1, 129), 5, seed=9 + k, stream=st) for k, st in enumerate(streams)]
    want, graphs = [], []
    for s, st in zip(steps, streams):
        with torch.cuda.stream(st):
            s.run()
        want.append(s.everything())
        s.check(want[-1])
    for s, st in zip(steps, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s.run()
        graphs.append(g)
    for k in range(4):
        for s in steps:
            for t in s.gw.values():
                t.fill_(float("nan"))
            for n in s.MADE + s.USED + ["lse", "lp"]:
                s.b.arena[s.b.at[s.i[n]]:s.b.at[s.i[n]] + s.b.sizes[s.i[n]]].fill_(0x7F)
            s.ws.fill_(0x7F if k % 2 else 0)
        torch.cuda.synchronize()
        for g in graphs[::-1] if k % 2 else graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(steps, want):
            got = s.everything()
            for n in w:
                assert np.array_equal(got[n], w[n]), (k, n)
        for s in steps:
            s.run()
        torch.cuda.synchronize()
    del graphs
    for s in steps:
        s.b.close()


def test_captured_step_takes_other_lengths_and_tokens(torch_mod):
    """Offsets, positions and ids are read by the device: a replay follows what they hold then."""
    torch = torch_mod
    st = torch.cuda.Stream()
    s = Decoder(torch, (70, 1, 129), 5, seed=12, stream=st)
    with torch.cuda.stream(st):
        s.run()
    s.everything()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        s.run()
    rng = np.random.default_rng(3)
    for off in ([0, 5, 200, 205], [0, 0, 0, 130], [7, 100, 164, 203]):
        s.off, s.longest = np.array(off, np.int64), 205
        s.next = rng.integers(-2, s.V + 2, s.T)
        s.b.put(s.i["off"], s.off)
        s.b.put(s.i["next"], s.next.astype(np.int64))
        g.replay()
        torch.cuda.synchronize()
        s.check(s.everything())
    del g
    s.b.close()


def test_two_contexts_on_two_streams_at_once(torch_mod):
    torch = torch_mod
    steps = [Decoder(torch, (300, 211), 2, seed=20 + k, stream=torch.cuda.Stream()) for k in range(2)]
    want = []
    for s in steps:
        s.run()
        want.append(s.everything())
        s.check(want[-1])
    for _ in range(3):
        for s in steps:
            s.run()
    for s, w in zip(steps, want):
        got = s.everything()
        for n in w:
            assert np.array_equal(got[n], w[n]), n
        s.b.close()


def test_step_large_enough_for_the_second_stream(torch_mod):
    """Weight gradients of more than 1 GFLOP run on the library's own stream and use the beginning of the workspace that normalisation and attention use the end of: with
    just the largest need the streams wait for each other, with twice that they do not; the results are the same."""
    s = Decoder(torch_mod, (1700, 2301, 2500), 3, V=512, FF=640, seed=30)
    assert "second stream" in s.b.d.backward_kernel(s.backward[9])
    s.run()
    want = s.everything()
    s.check(want)
    tight = max([s.b.d.backward_workspace(d) for d in s.forward if d.op != s.dl.OP_ROTARY] + [s.b.d.backward_workspace(s.backward[4].fwd)])
    for b in s.backward:
        b.workspace_bytes = tight
    for _ in range(3):
        for g in s.gw.values():
            g.fill_(float("nan"))
        torch_mod.cuda.synchronize()
        s.run()
        got = s.everything()
        for n in want:
            assert np.array_equal(got[n], want[n]), n
    s.b.close()


# ------------------------------------------------------------------ refusals

def test_refusals_leave_everything_as_it_was(torch_mod):
    import paper_2203_15980_amd as dl
    s = Decoder(torch_mod, (20, 9), 4, seed=2)
    i, F, none, T = s.i, s.F, dl.NO_TENSOR, s.T

    def forward(of, status=dl.ERR_INVALID, **kw):
        d = dl.LayerDesc.from_buffer_copy(F[of])
        for k, v in kw.items():
            setattr(d, k, v)
        with pytest.raises(dl.DeltaError) as e:
            s.b.d.recompute_segment([d])
        assert e.value.status == status and e.value.message, kw
    for kw in (dict(Cout=s.C + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(scale=None), dict(scale=s.dev["g1"].data_ptr() + 4), dict(y2=i["s2"]), dict(y3=i["c.n2"]), dict(pack=1),
               dict(flags=1), dict(res=i["ao"]), dict(pack=3), dict(y2=i["x0"], res=i["ao"]), dict(x=9999), dict(fuse=1)):
        forward("n1", **kw)
    for kw in (dict(y2=none), dict(y3=none), dict(pack=0), dict(y2=i["n2"]), dict(y3=i["s2"]), dict(y2=i["x0"]), dict(y2=9999), dict(y3=i["lse"]), dict(res=i["qkv"]), dict(res=none)):
        forward("n2", **kw)
    for kw in (dict(res=none), dict(res=i["lp"]), dict(res=i["gp.h"]), dict(R=0), dict(R=3, S=2), dict(S=-1), dict(scale=None), dict(flags=2), dict(y2=i["lse"]), dict(y3=i["lse"]), dict(pack=1), dict(Cout=64),
               dict(y=i["qkv"]), dict(R=32, S=32)):
        forward("rot", **kw)
    for kw in (dict(res=none), dict(res=i["lp"]), dict(R=3), dict(S=3), dict(S=0), dict(dtype=dl.DTYPE_F32), dict(flags=2), dict(y2=i["lp"]), dict(y3=i["lp"]), dict(pack=2), dict(y2=i["ctx"]),
               dict(Cout=s.C // 2), dict(R=2, S=1)):
        forward("att", **kw)
    for kw in (dict(res=none), dict(res=i["off"]), dict(Cout=65), dict(Cout=-1), dict(Cout=0), dict(Cout=2), dict(y2=none), dict(y3=none), dict(y2=i["which"]), dict(y3=i["best"]), dict(flags=1),
               dict(y=i["best"]), dict(dtype=7)):
        forward("lp", **kw)
    forward("o", flags=1)                                        # an operator without flags
    for of in ("n1", "rot", "att", "lp"):                        # rows that wrap around in 64 bits
        forward(of, N=2 ** 30, H=2 ** 30, W=2)
        forward(of, N=2 ** 31 - 1, H=2 ** 31 - 1, W=2 ** 31 - 1)
    s.b.d.release(i["pos"], dl.EV_OFFLOAD)
    forward("rot", status=dl.ERR_STATE)
    s.b.d.prefetch(i["pos"])

    def backward(k, status=dl.ERR_INVALID, fwd=None, **kw):
        D = dl.BwdDesc.from_buffer_copy(s.backward[k])
        for n, v in kw.items():
            setattr(D, n, v)
        for n, v in (fwd or {}).items():
            setattr(D.fwd, n, v)
        with pytest.raises(dl.DeltaError) as e:
            s.b.d.backward_segment([D])
        assert e.value.status == status and e.value.message, (k, kw)
    for k in (0, 7, 8):
        for kw in (dict(gx=none), dict(gx_add=i["s2"]), dict(gw=s.gw["q"].data_ptr()), dict(mask_gx=1), dict(gy_masked=1), dict(gx=s.backward[k].fwd.x), dict(gx=s.backward[k].gy),
                   dict(gpre=i["s2"]), dict(gy=i["ids"], gpre=i["ids"]), dict(gx=i["ids"]), dict(gy=9999, gpre=9999)):
            backward(k, **kw)
    for kw in (dict(workspace=None), dict(workspace=s.ws.data_ptr() + 64), dict(workspace_bytes=256), dict(fwd=dict(y2=none))):
        backward(7, **kw)
    for kw in (dict(gx=none, gw=None, gx_add=none), dict(gx=none), dict(gx=i["s2"], gx_add=i["s2"]), dict(gx=i["ao"]), dict(gx=i["n2"]), dict(gx_add=i["ids"]), dict(workspace=None),
               dict(gw=s.gw["n2"].data_ptr() + 4), dict(workspace_bytes=0), dict(mask_gx=1)):
        backward(5, **kw)
    s.b.d.release(i["lse"], dl.EV_FREE)
    backward(7, status=dl.ERR_STATE)
    for n in s.MADE + s.USED:                                    # as the arena began
        assert (s.b.get(i[n], np.uint8, (-1,)) == 0xA5).all(), n
    s.b.close()


def test_an_operator_that_finds_no_room_leaves_none_of_its_outputs_resident(torch_mod):
    import paper_2203_15980_amd as dl
    torch = torch_mod
    M, C = 64, 64
    n = M * C * 2
    arena = torch.zeros(4 * n + 256, dtype=torch.uint8, device="cuda:0")           # x, res, y: no room for the sum
    d = dl.Delta(arena[:3 * n + 256], torch.cuda.current_stream().cuda_stream)
    d.bind([n, n, n, n])
    d.alloc(0)
    d.alloc(1)
    gamma = torch.ones(C, device="cuda:0")
    L = dl.LayerDesc(x=0, res=1, y=2, y2=3, y3=dl.NO_TENSOR, dtype=dl.DTYPE_BF16, N=1, H=M, W=1, Cin=C, Cout=C, R=1, S=1, stride=1, op=dl.OP_RMSNORM, eps=1e-6, scale=gamma.data_ptr())
    before = d.stats()["arena_in_use"]
    with pytest.raises(dl.DeltaError) as e:
        d.recompute_segment([L])
    assert e.value.status == dl.ERR_OOM_ARENA and "arena block" in e.value.message
    for t in (2, 3):
        with pytest.raises(dl.DeltaError):
            d.tensor_ptr(t)
    assert d.stats()["arena_in_use"] == before
    d.close()


def test_rows_that_wrap_around_are_refused_before_bytes_are_divided(torch_mod):
    """2^61 rows of 8 bytes are 2^64, and so are those of x: a tensor of no bytes has both sizes."""
    import paper_2203_15980_amd as dl
    torch = torch_mod
    arena, f = torch.zeros(4096, dtype=torch.uint8, device="cuda:0"), torch.zeros(64, device="cuda:0")
    d = dl.Delta(arena, torch.cuda.current_stream().cuda_stream)
    d.bind([0, 0, 0])
    with pytest.raises(dl.DeltaError) as e:
        d.recompute_segment([dl.LayerDesc(x=0, res=1, y=2, y2=dl.NO_TENSOR, y3=dl.NO_TENSOR, dtype=dl.DTYPE_BF16, N=2 ** 30, H=2 ** 30, W=2, Cin=16, Cout=16, R=1, S=0, stride=1,
                                          op=dl.OP_ROTARY, scale=f.data_ptr())])
    assert e.value.status == dl.ERR_INVALID and "2147483647 rows" in e.value.message
    d.close()


def test_kernel_names(torch_mod):
    s = Decoder(torch_mod, (20, 9), 3, seed=2)
    assert s.b.d.layer_kernel(s.F["n2"]).startswith("rmsnorm bf16") and s.b.d.layer_kernel(s.F["att"]).startswith("packed_attention bf16")
    assert s.b.d.layer_kernel(s.F["rot"]).startswith("rotary bf16") and s.b.d.layer_kernel(s.F["lp"]).startswith("logprob bf16")
    assert [s.b.d.backward_kernel(s.backward[k]) for k in (0, 5, 8)] == ["gx: logprob", "gx, gw: rmsnorm", "gx: rotary"]
    assert s.b.d.backward_kernel(s.backward[7]).startswith("gx: packed_attention")
    s.b.close()
