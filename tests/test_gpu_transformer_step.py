"""The transformer's operators together, as a training step uses them: embedding, layer normalisation, linear layers with a
ReLU and a residual, checkpoints in 8 bits of what the backward pass reads, the tensors themselves released; the backward pass from the checkpoints; captured
into a graph and replayed; two contexts side by side; beside weight gradients on the library's second stream.

Each tensor is compared with float64 on the operands that the GPU itself stored, so that every operator's own rounding is the bar:
2^-8 of a bf16 value and what fp32 sums may add (rowops_util)."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, layernorm_noise, storage, values

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


class Step:
    """ids -> x0 = embedding -> n1 = layernorm(x0) -> h = relu(n1 w1 + b1) -> f = h w2 + b2 + x0 -> n2 = layernorm(f); gy = dL/dn2.
    n1 and h go into checkpoints (int8, E4M3), x0 and f too; the backward pass reads those (h itself as its own ReLU mask)."""
    NAMES = ["ids", "x0", "n1", "h", "f", "n2", "c.x0", "c.n1", "c.h", "c.f", "g.n2", "g.f", "g.h", "gp.h", "g.n1", "g.x0"]

    def __init__(self, torch, tokens=300, V=500, C=256, FF=512, seed=1, stream=None):
        import paper_2203_15980_amd as dl
        self.dl, self.torch = dl, torch
        rng = np.random.default_rng(seed)
        self.T, self.V, self.C, self.FF = tokens, V, C, FF
        big = {"h", "g.h", "gp.h"}
        size = lambda n: tokens * 8 if n == "ids" else ro.packed_bytes(tokens, FF if n == "c.h" else C) if n.startswith("c.") else \
            tokens * (FF if n in big else C) * 2                                 # noqa: E731
        self.i = {n: k for k, n in enumerate(self.NAMES)}
        self.b = b = Bench(torch, [size(n) for n in self.NAMES], stream=stream)
        ids = np.minimum(V - 1, np.floor((V + 3.0) ** rng.random(tokens) - 1)).astype(np.int64)
        ids[rng.random(tokens) < 0.1] = -1
        gy = storage(rng.normal(size=(tokens, C)), "bf16")
        b.put(self.i["ids"], ids)
        b.put(self.i["g.n2"], gy)
        self.ids = ids
        P = self.P = {}
        P["table"] = storage(rng.normal(size=(V, C)) * 0.02, "bf16")
        P["w1"], P["w2"] = storage(rng.normal(size=(FF, C)) / 16, "bf16"), storage(rng.normal(size=(C, FF)) / 22, "bf16")
        f32 = lambda a: a.astype(np.float32)                                     # noqa: E731
        P["scale"] = np.full(C, 16.0, np.float32)
        for k, n in (("1", FF), ("2", C)):
            P["one" + k], P["b" + k] = np.ones(n, np.float32), f32(rng.normal(size=n) * 0.02)
            P["g" + k], P["be" + k] = f32(rng.uniform(0.5, 1.5, C)), f32(rng.normal(size=C) * 0.1)
        self.dev = {k: b.dev(v.view(np.int16) if v.dtype == np.uint16 else v) for k, v in P.items()}
        self.wt = {"1": b.dev(np.zeros((C, FF), np.int16)), "2": b.dev(np.zeros((FF, C), np.int16))}
        p, i = (lambda n: self.dev[n].data_ptr()), self.i
        L = lambda op, x, y, cin, cout, **kw: b.layer(op, tokens, cin, cout, i[x], i[y], **kw)     # noqa: E731
        emb = L(dl.OP_EMBEDDING, "ids", "x0", V, C, w=p("table"), scale=p("scale"))
        ln1 = L(dl.OP_LAYERNORM, "x0", "n1", C, C, scale=p("g1"), shift=p("be1"), eps=EPS)
        l1 = L(dl.OP_CONV, "n1", "h", C, FF, w=p("w1"), scale=p("one1"), shift=p("b1"), relu=1)
        l2 = L(dl.OP_CONV, "h", "f", FF, C, w=p("w2"), scale=p("one2"), shift=p("b2"), res=i["x0"])
        ln2 = L(dl.OP_LAYERNORM, "f", "n2", C, C, scale=p("g2"), shift=p("be2"), eps=EPS)
        pk = lambda n, c, fmt: L(dl.OP_PACK8, n, "c." + n, c, c, pack=fmt)       # noqa: E731
        self.forward = [emb, ln1, l1, l2, ln2, pk("x0", C, dl.PACK_INT8), pk("n1", C, dl.PACK_INT8), pk("h", FF, dl.PACK_E4M3), pk("f", C, dl.PACK_E4M3)]
        self.fmt = {"x0": "int8", "n1": "int8", "h": "e4m3", "f": "e4m3"}

        def held(layer, n):
            d = dl.LayerDesc.from_buffer_copy(layer)
            d.x, d.pack = i["c." + n], {"int8": dl.PACK_INT8, "e4m3": dl.PACK_E4M3}[self.fmt[n]]
            return d
        self.held = dict(ln2=held(ln2, "f"), l2=held(l2, "h"), l1=held(l1, "n1"), ln1=held(ln1, "x0"), emb=emb)
        need = [b.d.backward_workspace(d) for d in self.held.values()]
        self.ws, self.whole = b.workspace(2 * max(need) + 256)
        self.gw = {n: b.guarded(k)[0] for n, k in (("ln2", 2 * C), ("l2", C * FF), ("l1", FF * C), ("ln1", 2 * C), ("emb", V * C))}
        b.d.bwd_weights(l1, self.wt["1"].data_ptr())
        b.d.bwd_weights(l2, self.wt["2"].data_ptr())
        h, kw = self.held, dict(ws=self.ws)
        self.backward = [
            b.bwd(h["ln2"], i["g.n2"], gx=i["g.f"], gw=self.gw["ln2"], **kw),
            b.bwd(h["l2"], i["g.f"], gx=i["g.h"], gw=self.gw["l2"], wt=self.wt["2"].data_ptr(), **kw),
            b.bwd(h["l1"], i["g.h"], gx=i["g.n1"], gw=self.gw["l1"], wt=self.wt["1"].data_ptr(), gpre=i["gp.h"], **kw),
            b.bwd(h["ln1"], i["g.n1"], gx=i["g.x0"], add=i["g.f"], gw=self.gw["ln1"], **kw),     # and the residual's gradient
            b.bwd(h["emb"], i["g.x0"], gw=self.gw["emb"], **kw)]

    def run(self):
        self.b.d.recompute_segment(self.forward)
        self.b.d.backward_segment(self.backward)
        self.b.d.backward_join()

    def get(self, n, c=None):
        return values(self.b.get(self.i[n], np.uint16, (self.T, c or (self.FF if n in ("h", "g.h", "gp.h") else self.C))), "bf16")

    def everything(self):
        self.b.d.sync()
        out = {n: self.get(n).copy() for n in ("x0", "n1", "h", "f", "n2", "g.f", "g.h", "gp.h", "g.n1", "g.x0")}
        out.update({"gw." + n: t.cpu().numpy().astype(np.float64) for n, t in self.gw.items()})
        return out

    def check(self, o):
        """Every tensor against float64 on the stored operands of its operator."""
        P = {k: (values(v, "bf16") if v.dtype == np.uint16 else v.astype(np.float64)) for k, v in self.P.items()}
        T = self.T

        def near(got, ref, noise):
            tol = 2.0 ** -8 * np.abs(ref) + noise
            assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) / tol).max())
        near(o["x0"], ro.embedding(self.ids, P["table"], P["scale"]), 0)
        for x, y, k in (("x0", "n1", "1"), ("f", "n2", "2")):
            X = o[x]
            c = X - X.mean(axis=1, keepdims=True)
            r = 1 / np.sqrt((c * c).mean(axis=1, keepdims=True) + EPS)
            near(o[y], ro.layernorm(X, P["g" + k], P["be" + k], EPS),
                 40 * EPS24 * (np.abs(X).max(axis=1, keepdims=True) * r + np.abs(c * r)) * P["g" + k] + 2 * EPS24 * np.abs(P["be" + k]))
        pre = o["n1"] @ P["w1"].T + P["b1"]
        near(o["h"], np.maximum(pre, 0), self.C * EPS24 * (np.abs(o["n1"]) @ np.abs(P["w1"]).T + np.abs(P["b1"])))
        near(o["f"], o["h"] @ P["w2"].T + P["b2"] + o["x0"], self.FF * EPS24 * (np.abs(o["h"]) @ np.abs(P["w2"]).T + np.abs(P["b2"]) + np.abs(o["x0"])))
        C = {n: ro.unpack(*ro.pack(o[n], f), f) for n, f in self.fmt.items()}    # what the checkpoints hold
        for x, gy, gx, k, n in (("f", self.get("g.n2"), "g.f", "2", "ln2"), ("x0", o["g.n1"], "g.x0", "1", "ln1")):
            add = o["g.f"] if n == "ln1" else np.zeros((T, self.C))
            rgx, rdg, rdb = ro.layernorm_bwd(C[x], gy, P["g" + k], EPS, add)
            ngx, ndg, ndb = layernorm_noise(C[x], gy, P["g" + k], EPS)
            near(o[gx], rgx, 2 * ngx + EPS24 * np.abs(add))
            assert (np.abs(o["gw." + n][:self.C] - rdg) <= ndg).all() and (np.abs(o["gw." + n][self.C:] - rdb) <= ndb).all()
        near(o["g.h"], o["g.f"] @ P["w2"], self.C * EPS24 * (np.abs(o["g.f"]) @ np.abs(P["w2"])))
        assert np.array_equal(o["gp.h"], np.where(o["h"] > 0, o["g.h"], 0))
        near(o["g.n1"], o["gp.h"] @ P["w1"], self.FF * EPS24 * (np.abs(o["gp.h"]) @ np.abs(P["w1"])))
        for n, g, x in (("l2", o["g.f"], C["h"]), ("l1", o["gp.h"], C["n1"])):
            got = o["gw." + n].reshape(g.shape[1], x.shape[1])
            assert (np.abs(got - g.T @ x) <= T * EPS24 * (np.abs(g).T @ np.abs(x))).all()
        got, size = o["gw.emb"].reshape(self.V, self.C), ro.embedding_bwd(self.ids, np.abs(o["g.x0"]), P["scale"], self.V)
        assert (np.abs(got - ro.embedding_bwd(self.ids, o["g.x0"], P["scale"], self.V)) <= T * EPS24 * size).all()


@pytest.mark.parametrize("tokens,V,C,FF", [(300, 500, 256, 512), (1, 40, 64, 64), (77, 30, 768, 128), (2500, 3000, 128, 192)])
def test_step_with_the_activations_released(torch_mod, tokens, V, C, FF):
    print("tokens", tokens, "V", V, "C", C, "FF", FF, flush=True)
    s = Step(torch_mod, tokens, V, C, FF, seed=tokens)
    s.run()
    want = s.everything()
    s.check(want)
    # once more, with everything that has a checkpoint (and the gradients) gone before the backward pass
    d, dl = s.b.d, s.dl
    d.recompute_segment(s.forward)
    for n in ("x0", "n1", "f", "n2", "g.f", "g.h", "gp.h", "g.n1", "g.x0"):
        d.release(s.i[n], dl.EV_EVICT)
    d.release(s.i["c.n1"], dl.EV_OFFLOAD)
    d.prefetch(s.i["c.n1"])
    for g in s.gw.values():
        g.fill_(float("nan"))
    torch_mod.cuda.synchronize()
    d.backward_segment(s.backward)
    d.backward_join()
    d.sync()
    for n in ("g.f", "g.h", "gp.h", "g.n1", "g.x0"):
        s.b.at[s.i[n]] = d.tensor_ptr(s.i[n]) - s.b.arena.data_ptr()
        assert np.array_equal(s.get(n), want[n]), n
    for n, g in s.gw.items():
        assert np.array_equal(g.cpu().numpy().astype(np.float64), want["gw." + n]), n
    s.b.close()


def test_step_captured_into_a_graph_and_replayed(torch_mod):
    torch = torch_mod
    stream = torch.cuda.Stream()
    s = Step(torch, 300, 500, 256, 512, seed=9, stream=stream)
    with torch.cuda.stream(stream):
        s.run()                                              # identity factors and attributes are made here, not in the capture
    want = s.everything()
    s.check(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        s.run()
    other = Step(torch, 64, 100, 64, 64, seed=10)            # eager work of another context between the replays
    for k in range(4):
        for t in s.gw.values():
            t.fill_(float("nan"))
        for n in ("x0", "n1", "g.f", "g.x0", "c.h"):
            s.b.arena[s.b.at[s.i[n]]:s.b.at[s.i[n]] + s.b.sizes[s.i[n]]].fill_(0x7F)
        s.ws.fill_(0x7F if k % 2 else 0)
        torch.cuda.synchronize()
        g.replay()
        other.run()
        torch.cuda.synchronize()
        got = s.everything()
        for n in want:
            assert np.array_equal(got[n], want[n]), (k, n)
    del g
    other.b.close()
    s.b.close()


def test_two_contexts_on_two_streams_at_once(torch_mod):
    torch = torch_mod
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Step(torch, 700, 900, 256, 256, seed=20 + k, stream=st) for k, st in enumerate(streams)]
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
    """Linear layers of more than 1 GFLOP: their weight gradients run on the library's own stream and use the beginning of the workspace
    that layer normalisation and the embedding use the end of: one workspace of just the largest need makes the streams wait for each other, one of
    twice that does not; the results are the same."""
    s = Step(torch_mod, 4000, 700, 512, 512, seed=30)
    assert "second stream" in s.b.d.backward_kernel(s.backward[1])
    s.run()
    want = s.everything()
    s.check(want)
    tight = max(s.b.d.backward_workspace(d) for d in s.held.values())
    for bw in s.backward:
        bw.workspace_bytes = tight
    for _ in range(3):
        for g in s.gw.values():
            g.fill_(float("nan"))
        torch_mod.cuda.synchronize()
        s.run()
        got = s.everything()
        for n in want:
            assert np.array_equal(got[n], want[n]), n
    s.b.close()
