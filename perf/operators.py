"""The operators of a transformer's training step that are measured here: layer normalisation and its
gradients, activation checkpoints in 8 bits and their use in the backward pass, embedding lookup and
its gradient, each through the C ABI's binding as a training program calls it (`own`), and in plain
torch operations.

The checkpoint format: a row's channels in blocks of 32 (the last may be shorter); a block has one
scale 2^e, e the smallest integer in [-120, 127] with max|x| <= M * 2^e; a value is stored as
round(x / 2^e) to the nearest representable one, ties to even: whole numbers up to M = 127 in "int8",
OCP E4M3 numbers up to M = 448 in "e4m3".
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-12
SYNC_EVERY = 16      # passes between two delta_sync calls: a program syncs where it reads its loss; events are recycled there


def listed():
    return [
        # one short odd sequence through a normalisation of the encoder (768 channels): launches and latency
        dict(name="ln_backward_b1_77", kind="layernorm", do="backward", dtype="bf16", N=1, S=77, C=768, add=False, pack=""),
        # the encoder layer of configuration 5 at 32 x 512 tokens: both gradients from the stored input
        dict(name="ln_backward_b32_512", kind="layernorm", do="backward", dtype="bf16", N=32, S=512, C=768, add=False, pack=""),
        # fp32, odd rows, channels that no power of two divides: forward and backward
        dict(name="ln_both_f32_b3_211", kind="layernorm", do="both", dtype="f32", N=3, S=211, C=1000, add=False, pack=""),
        # a wide hidden state before a residual branch: forward, backward and the branch's gradient added on the way
        dict(name="ln_both_b8_1024_c8192", kind="layernorm", do="both", dtype="bf16", N=8, S=1024, C=8192, add=True, pack=""),
        # an activation of configuration 5 into its checkpoint and back
        dict(name="pack_int8_b32_512", kind="pack", fmt="int8", dtype="bf16", N=32, S=512, C=768),
        # an fp32 activation with a short last block and odd rows
        dict(name="pack_e4m3_f32_b5_333", kind="pack", fmt="e4m3", dtype="f32", N=5, S=333, C=1016),
        # the encoder's normalisation again, its input held as a checkpoint
        dict(name="ln_backward_int8_b32_512", kind="layernorm", do="backward", dtype="bf16", N=32, S=512, C=768, add=False, pack="int8"),
        # the attention output layer's weight gradient from a checkpoint of its input
        dict(name="linear_int8_b32_512", kind="linear", fmt="int8", N=32, S=512, Cin=768, Cout=768),
        # a small layer on one odd sequence
        dict(name="linear_e4m3_b1_333", kind="linear", fmt="e4m3", N=1, S=333, Cin=1024, Cout=256),
        # one short odd sequence through an fp32 table and back
        dict(name="embedding_both_f32_b1_77", kind="embedding", do="both", dtype="f32", N=1, S=77, V=30522, C=768),
        # configuration 5's tokens through a table of BERT-base's size and back: a training step's first and last operators
        dict(name="embedding_both_b32_512", kind="embedding", do="both", dtype="bf16", N=32, S=512, V=30522, C=768),
        # a large vocabulary and a long batch: the gradient
        dict(name="embedding_backward_b8_4096_v131072", kind="embedding", do="backward", dtype="bf16", N=8, S=4096, V=131072, C=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layernorm"] * 3 + ["pack", "linear", "linear", "embedding", "embedding"])
    N, S = _log(rng, 1, 32), _log(rng, 1, 512)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "layernorm":
        C = 64 * _log(rng, 33, 128) if rng.random() < 0.3 else 8 * _log(rng, 1, 256)
        if C > 2048:
            S = min(S, (4096 if dtype == "f32" else 8192) // N)
        return dict(kind=kind, do=rng.choice(["backward", "both"]), dtype=dtype, N=N, S=S, C=C, add=rng.random() < 0.4,
                    pack=rng.choice(["", "", "int8", "e4m3"]))
    if kind == "pack":
        return dict(kind=kind, fmt=rng.choice(["int8", "e4m3"]), dtype=dtype, N=N, S=S, C=8 * _log(rng, 1, 512))
    if kind == "linear":
        return dict(kind=kind, fmt=rng.choice(["int8", "e4m3"]), N=N, S=S, Cin=64 * _log(rng, 1, 32), Cout=64 * _log(rng, 1, 32))
    return dict(kind=kind, do=rng.choice(["forward", "backward", "both"]), dtype=dtype, N=N, S=S * rng.choice([1, 2]),
                V=_log(rng, 100, 131072), C=8 * _log(rng, 8, 256))


# ------------------------------------------------------------------ inputs

def _tdtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _inputs(case, seed):
    """Every input of a case, from the seed alone: name -> GPU tensor."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    t, k = _tdtype(case), case["kind"]
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)                       # noqa: E731
    un = lambda lo, hi, n: lo + (hi - lo) * torch.rand(n, device=DEV, generator=g)  # noqa: E731
    M, v = case["N"] * case["S"], {}
    if k == "embedding":
        V, C = case["V"], case["C"]
        # ids by falling frequency, as a vocabulary is numbered: id k is met about as often as 1 / (k + 3); the
        # sequences of a batch have different lengths, and -1 stands behind their ends
        u = torch.rand(M, device=DEV, generator=g, dtype=torch.float64)
        ids = (3.0 * ((V + 3) / 3.0) ** u - 3.0).floor().clamp_(0, V - 1).to(torch.int64).reshape(case["N"], case["S"])
        if case["N"] > 1:
            length = (case["S"] * un(0.5, 1.0, case["N"])).ceil()
            ids[torch.arange(case["S"], device=DEV)[None, :] >= length[:, None]] = -1
        v["ids"] = ids
        v["w"] = (0.02 * rn(V, C)).to(t)
        v["scale"] = torch.full((C,), math.sqrt(C), device=DEV)
        if case["do"] != "forward":
            v["gy"] = rn(M, C).to(t)
        return v
    C = case["Cin"] if k == "linear" else case["C"]
    # a hidden state: rows with a mean, channels of different spread, a few of them large
    spread = un(0.5, 1.5, C) * torch.where(torch.rand(C, device=DEV, generator=g) < 0.01, 12.0, 1.0)
    v["x"] = (rn(M, C) * spread + 0.3 * rn(C)).to(t)
    if k == "layernorm":
        v["gy"] = rn(M, C).to(t)
        v["gamma"], v["beta"] = un(0.5, 1.5, C), 0.1 * rn(C)
        if case["add"]:
            v["add"] = rn(M, C).to(t)
    elif k == "linear":
        v["gy"] = rn(M, case["Cout"]).to(t)
    return v


# ------------------------------------------------------------------ plain form

def _power(e):
    """2^e in fp32, from its bits: pow() and ldexp() of a GPU may be off in the last place."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_pack(x, fmt):
    """(stored values, exponents) of x [M, C]."""
    M, C = x.shape
    nb = (C + 31) // 32
    xb = torch.nn.functional.pad(x.float(), (0, nb * 32 - C)).reshape(M, nb, 32)
    most = 127.0 if fmt == "int8" else 448.0
    m, p = torch.frexp(xb.abs().amax(dim=2))                     # amax = m 2^p, m in [0.5, 1)
    unit, top = math.frexp(most)                                 # most = unit 2^top
    e = torch.where(m <= unit, p - top, p - top + 1)
    e = torch.where(m == 0, -120, e).clamp(-120, 127)
    q = xb * _power(-e)[:, :, None]
    q = torch.round(q).to(torch.int8) if fmt == "int8" else q.to(torch.float8_e4m3fn)
    return q, e.to(torch.int8)


def _plain_unpack(packed, C):
    q, e = packed
    return (q.float() * _power(e)[:, :, None]).reshape(q.shape[0], -1)[:, :C]


def _run_plain(state):
    case, v = state["case"], state["v"]
    t, k = _tdtype(case), case["kind"]
    if k == "pack":
        return _plain_unpack(_plain_pack(v["x"], case["fmt"]), case["C"]).to(t)
    if k == "linear":
        x = _plain_unpack(state["packed"], case["Cin"])
        return v["gy"].float().t() @ x
    if k == "layernorm":
        x = _plain_unpack(state["packed"], case["C"]) if case["pack"] else v["x"].float()
        mean = x.mean(dim=1, keepdim=True)
        c = x - mean
        rstd = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + EPS)
        xh = c * rstd
        out = []
        if case["do"] == "both":
            out.append((xh * v["gamma"] + v["beta"]).to(t))
        gy = v["gy"].float()
        g = gy * v["gamma"]
        gx = rstd * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
        if case["add"]:
            gx = gx + v["add"].float()
        out += [gx.to(t), torch.cat([(gy * xh).sum(dim=0), gy.sum(dim=0)])]
        return out
    ids = v["ids"].reshape(-1)
    there = (ids >= 0).float()[:, None]
    at = ids.clamp(min=0)
    out = []
    if case["do"] != "backward":
        out.append((v["w"][at].float() * v["scale"] * there).to(t))
    if case["do"] != "forward":
        gw = torch.zeros(case["V"], case["C"], device=DEV)
        out.append(gw.index_add_(0, at, v["gy"].float() * there) * v["scale"])
    return out


# ------------------------------------------------------------------ the framework's operators

class Program:
    """A context, its arena and its tensor table; outputs are views of the arena."""

    def __init__(self, sizes):
        import paper_2203_15980_amd as dl
        self.ids = {n: i for i, n in enumerate(sizes)}
        self.meta = sizes
        nb = [math.prod(s) * torch.empty((), dtype=dt).element_size() for s, dt in sizes.values()]
        self.arena = torch.empty(sum((b + 255) // 256 * 256 for b in nb) + (1 << 20), dtype=torch.uint8, device=DEV)
        self.d = dl.Delta(self.arena, torch.cuda.current_stream().cuda_stream)
        self.d.bind(nb)
        for i in range(len(nb)):
            self.d.alloc(i)
        self.passes = 0

    def view(self, name):
        shape, dt = self.meta[name]
        off = self.d.tensor_ptr(self.ids[name]) - self.arena.data_ptr()
        return self.arena[off:off + math.prod(shape) * torch.empty((), dtype=dt).element_size()].view(dt).reshape(shape)

    def put(self, name, value):
        self.view(name).copy_(value.reshape(self.meta[name][0]))

    def begin(self):
        self.passes += 1
        if self.passes % SYNC_EVERY == 0:
            self.d.sync()


def _packed_bytes(dl, rows, C):
    d = dl.Delta()
    n = d.packed_bytes(rows, C)
    d.close()
    return n


def _prepare_own(case, v):
    import paper_2203_15980_amd as dl
    k, t, M = case["kind"], _tdtype(case), case["N"] * case["S"]
    code = dl.DTYPE_F32 if t == torch.float32 else dl.DTYPE_BF16
    fmt = {"": 0, "int8": dl.PACK_INT8, "e4m3": dl.PACK_E4M3}[case.get("fmt", case.get("pack", ""))]
    geo = dict(res=dl.NO_TENSOR, dtype=code, N=case["N"], H=case["S"], W=1, R=1, S=1, stride=1, pad=0, relu=0)
    none = dl.NO_TENSOR
    sizes = {}
    if k == "embedding":
        C = case["C"]
        sizes["ids"], sizes["y"] = (tuple(v["ids"].shape), torch.int64), ((M, C), t)
        if "gy" in v:
            sizes["gy"] = ((M, C), t)
    else:
        C = case["Cin"] if k == "linear" else case["C"]
        sizes["x"] = ((M, C), t)
        if fmt:
            sizes["packed"] = ((_packed_bytes(dl, M, C),), torch.uint8)
        if k == "linear":
            sizes["y"], sizes["gy"] = ((M, case["Cout"]), t), ((M, case["Cout"]), t)
        else:
            sizes["y"] = ((M, C), t)
        if k == "layernorm":
            sizes["gy"], sizes["gx"] = ((M, C), t), ((M, C), t)
            if case["add"]:
                sizes["add"] = ((M, C), t)
    p = Program(sizes)
    for n in sizes:
        if n in v:
            p.put(n, v[n])
    i = p.ids
    p.forward, p.backward, p.out, p.v = None, [], [], v
    pack = dl.LayerDesc(x=i.get("x", 0), y=i.get("packed", 0), Cin=C, Cout=C, op=dl.OP_PACK8, pack=fmt, **geo)
    if k == "pack":
        p.forward = dl.layer_array([pack, dl.LayerDesc(x=i["packed"], y=i["y"], Cin=C, Cout=C, op=dl.OP_UNPACK8, pack=fmt, **geo)])
        p.out = [p.view("y")]
        return p
    if fmt:                                                      # the checkpoint that the forward pass left
        p.d.recompute_segment([pack])
    if k == "embedding":
        fwd = dl.LayerDesc(x=i["ids"], y=i["y"], Cin=case["V"], Cout=C, op=dl.OP_EMBEDDING, w=v["w"].data_ptr(), scale=v["scale"].data_ptr(),
                           **geo)
        gw = (case["V"], C)
    elif k == "linear":
        p.ones, p.zeros = torch.ones(case["Cout"], device=DEV), torch.zeros(case["Cout"], device=DEV)
        p.w = torch.zeros(case["Cout"], C, device=DEV, dtype=t)
        fwd = dl.LayerDesc(x=i["packed"], y=i["y"], Cin=C, Cout=case["Cout"], op=dl.OP_CONV, w=p.w.data_ptr(), scale=p.ones.data_ptr(),
                           shift=p.zeros.data_ptr(), pack=fmt, **geo)
        gw = (case["Cout"], C)
    else:
        fwd = dl.LayerDesc(x=i["packed" if fmt else "x"], y=i["y"], Cin=C, Cout=C, op=dl.OP_LAYERNORM, scale=v["gamma"].data_ptr(),
                           shift=v["beta"].data_ptr(), eps=EPS, pack=fmt, **geo)
        gw = (2 * C,)
    if case.get("do") in ("forward", "both"):
        if fmt:                                                  # a forward pass from a checkpoint restores it first
            there = dl.LayerDesc(x=i["packed"], y=i["x"], Cin=C, Cout=C, op=dl.OP_UNPACK8, pack=fmt, **geo)
            plain = dl.LayerDesc.from_buffer_copy(fwd)
            plain.x, plain.pack = i["x"], 0
            p.forward = dl.layer_array([there, plain])
        else:
            p.forward = dl.layer_array([fwd])
        p.out.append(p.view("y"))
    if case.get("do") != "forward":
        need = p.d.backward_workspace(fwd)
        p.gw, p.work = torch.empty(*gw, device=DEV), torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        gx = i["gx"] if k == "layernorm" else none
        p.backward = [dl.BwdDesc(fwd=fwd, gy=i["gy"], gpre=i["gy"], gx=gx, gx_add=i.get("add", none), gw=p.gw.data_ptr(),
                                 workspace=p.work.data_ptr(), workspace_bytes=p.work.numel())]
        if k == "layernorm":
            p.out.append(p.view("gx"))
        p.out.append(p.gw)
    if k == "embedding" and len(p.out) == 1:
        p.out = [p.out]                                          # a list also where it is one output, as in the plain form
    return p


def prepare(case, seed):
    v = _inputs(case, seed)
    if own:
        p = _prepare_own(case, v)
        torch.cuda.synchronize()
        return p
    state = dict(case=case, v=v)
    fmt = case.get("pack") or (case.get("fmt") if case["kind"] == "linear" else "")
    if fmt:
        state["packed"] = _plain_pack(v["x"], fmt)
    torch.cuda.synchronize()
    return state


def run(state):
    if not own:
        return _run_plain(state)
    p = state
    p.begin()
    if p.forward is not None:
        p.d.recompute_segment(p.forward)
    if p.backward:
        p.d.backward_segment(p.backward)
        p.d.backward_join()
    return p.out[0] if len(p.out) == 1 else p.out


# ------------------------------------------------------------------ work

def work(case):
    k, M = case["kind"], case["N"] * case["S"]
    es = 4 if case.get("dtype") == "f32" else 2
    packed = lambda C: M * (C + (C + 31) // 32)                                    # noqa: E731
    if k == "pack":
        return dict(bytes=M * case["C"] * 2 * es + packed(case["C"]), flops=6 * M * case["C"])
    if k == "linear":
        return dict(bytes=M * case["Cout"] * 2 + packed(case["Cin"]) + case["Cin"] * case["Cout"] * 4,
                    flops=2 * M * case["Cin"] * case["Cout"])
    C = case["C"]
    if k == "layernorm":
        n = M * C
        bytes_ = n * es * 2 + (packed(C) if case["pack"] else n * es) + C * 12 + (n * es if case["add"] else 0)     # gy, gx; x; gamma and its gradients
        flops = 18 * n
        if case["do"] == "both":
            bytes_, flops = bytes_ + n * es + C * 4, flops + 8 * n
        return dict(bytes=bytes_, flops=flops)
    bytes_ = M * 8 + C * 4
    rows = min(M, case["V"])
    if case["do"] != "backward":
        bytes_ += M * C * es + rows * C * es
    if case["do"] != "forward":
        bytes_ += M * C * es + case["V"] * C * 4
    return dict(bytes=bytes_, flops=2 * M * C)


# ------------------------------------------------------------------ exact

def _power64(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_checkpoint(x, fmt):
    """x as its checkpoint holds it, in 64 bits: the scale by counting the powers of two that are too small, the value by its own grid."""
    M, C = x.shape
    out = torch.empty(M, C, dtype=torch.float64, device=DEV)
    most = 127.0 if fmt == "int8" else 448.0
    for lo in range(0, C, 32):
        b = x[:, lo:lo + 32].double()
        ratio = b.abs().max(dim=1, keepdim=True).values / most
        e = torch.ceil(torch.log2(ratio.clamp(min=2.0 ** -120))).clamp(-120, 127)
        e = torch.where(_power64(e) < ratio, e + 1, e)                              # log2 may be off by its last bit
        e = torch.where((_power64(e - 1) >= ratio) & (e > -120), e - 1, e)
        s = _power64(e)
        q = b / s
        if fmt == "int8":
            out[:, lo:lo + 32] = torch.round(q) * s
        else:
            k = torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6)))              # binade of a value, subnormals in the lowest
            k = torch.where(_power64(k) > q.abs().clamp(min=2.0 ** -6), k - 1, k)
            k = torch.where(_power64(k + 1) <= q.abs(), k + 1, k)
            step = _power64(k - 3)
            out[:, lo:lo + 32] = torch.round(q / step) * step * s
    return out


def exact(case, seed):
    v, k = _inputs(case, seed), case["kind"]
    if k == "pack":
        return _exact_checkpoint(v["x"], case["fmt"])
    if k == "linear":
        return torch.matmul(v["gy"].double().t().contiguous(), _exact_checkpoint(v["x"], case["fmt"]))
    if k == "layernorm":
        x = _exact_checkpoint(v["x"], case["pack"]) if case["pack"] else v["x"].double()
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        inv = (var + EPS).rsqrt()
        n = (x - mean) * inv
        gamma, gy = v["gamma"].double(), v["gy"].double()
        out = [n * gamma + v["beta"].double()] if case["do"] == "both" else []
        C = float(case["C"])
        h = gy * gamma
        gx = (C * h - h.sum(1, keepdim=True) - n * (h * n).sum(1, keepdim=True)) * inv / C
        if case["add"]:
            gx = gx + v["add"].double()
        return out + [gx, torch.cat([(gy * n).sum(0), gy.sum(0)])]
    ids, scale = v["ids"].reshape(-1), v["scale"].double()
    keep = ids >= 0
    out = []
    if case["do"] != "backward":
        y = torch.zeros(ids.numel(), case["C"], dtype=torch.float64, device=DEV)
        y[keep] = v["w"][ids[keep]].double() * scale
        out.append(y)
    if case["do"] != "forward":
        gw = torch.zeros(case["V"], case["C"], dtype=torch.float64, device=DEV)
        gw.index_put_((ids[keep],), v["gy"][keep].double() * scale, accumulate=True)
        out.append(gw)
    return out
