"""The operators of a decoder layer's training step that are measured here: root-mean-square normalisation with the residual's
addition and an output in 8 bits, rotary positions with several axes, attention over packed sequences with grouped heads, log
probabilities of given tokens with entropy and top alternatives, each with its gradients, through the C ABI's binding as a training
program calls it (`own`), and in plain torch operations.

Checkpoint format of the 8-bit output: a row's channels in blocks of 32 (the last may be shorter); a block has one scale 2^e, e the
smallest integer in [-120, 127] with max|x| <= M * 2^e; a value is stored as round(x / 2^e), ties to even: whole numbers up to
M = 127 in "int8", OCP E4M3 numbers up to M = 448 in "e4m3".
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
SYNC_EVERY = 16      # passes between two delta_sync calls: a program syncs where it reads its loss; events are recycled there


def listed():
    return [
        # one short odd sequence through an attention of the encoder's shape, causal: launches and latency
        dict(name="attention_both_b1_77", kind="attention", do="both", seqs=1, longest=77, even=True, tail=0, heads=12, kv=12, D=64, causal=True),
        # a batch of configuration 5 without its padding: 32 sequences of up to 512, all positions see each other
        dict(name="attention_both_full_b32_512", kind="attention", do="both", seqs=32, longest=512, even=False, tail=0, heads=12, kv=12, D=64,
             causal=False),
        # documents of different lengths packed into one row of tokens, with room behind the last; a forward pass that a recomputation runs again
        dict(name="attention_forward_packed_9_1531", kind="attention", do="forward", seqs=9, longest=1531, even=False, tail=37, heads=16, kv=2, D=128,
             causal=True),
        # one long document
        dict(name="attention_both_b1_8192", kind="attention", do="both", seqs=1, longest=8192, even=True, tail=0, heads=32, kv=8, D=128, causal=True),
        # one short odd sequence through a normalisation behind a residual
        dict(name="rmsnorm_both_b77_c768", kind="rmsnorm", do="both", dtype="bf16", M=77, C=768, res=True, add=True, pack=""),
        # a wide hidden state: forward with the checkpoint that the next linear layer keeps, backward with the residual's gradient added
        dict(name="rmsnorm_both_int8_b8192_c4096", kind="rmsnorm", do="both", dtype="bf16", M=8192, C=4096, res=True, add=True, pack="int8"),
        # fp32, odd rows, channels that no power of two divides, a short last block
        dict(name="rmsnorm_both_e4m3_f32_b633_c1000", kind="rmsnorm", do="both", dtype="f32", M=633, C=1000, res=False, add=False, pack="e4m3"),
        # one short text, the queries and keys of 12 heads beside values that are not rotated, neighbouring channels paired
        dict(name="rotary_both_b77", kind="rotary", do="both", dtype="bf16", M=77, axes=1, heads=24, rest=12, D=64, pairs=True),
        # frames of a video by time, height and width, grouped heads
        dict(name="rotary_both_video_b8192", kind="rotary", do="both", dtype="bf16", M=8192, axes=3, heads=40, rest=8, D=128, pairs=False),
        # one next token's alternatives over a vocabulary of BERT-base's size
        dict(name="logprob_forward_b1_v30522", kind="logprob", do="forward", dtype="f32", M=1, V=30522, K=20, masked=0),
        # scores of a rewarded answer: odd rows and vocabulary, entropy and alternatives, gradients
        dict(name="logprob_both_b333_v50001", kind="logprob", do="both", dtype="f32", M=333, V=50001, K=5, masked=17),
        # the loss of a batch over a large vocabulary
        dict(name="logprob_both_b4096_v131072", kind="logprob", do="both", dtype="bf16", M=4096, V=131072, K=0, masked=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention"] * 3 + ["rmsnorm", "rotary", "logprob", "logprob"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    do = rng.choice(["forward", "both", "both"])
    if kind == "attention":
        longest = _log(rng, 1, 4096)
        seqs = _log(rng, 1, max(1, min(64, 8192 // longest)))
        kv, group = rng.choice([1, 2, 3, 4, 8, 12]), rng.choice([1, 1, 2, 4, 8])
        while kv * group > 32:
            group //= 2
        return dict(kind=kind, do=do, seqs=seqs, longest=longest, even=rng.random() < 0.3, tail=rng.choice([0, 0, 1, 19, 130]), heads=kv * group, kv=kv,
                    D=rng.choice([64, 128]), causal=rng.random() < 0.7)
    if kind == "rmsnorm":
        return dict(kind=kind, do=do, dtype=dtype, M=_log(rng, 1, 8192), C=8 * _log(rng, 1, 512), res=rng.random() < 0.6, add=rng.random() < 0.5,
                    pack=rng.choice(["", "", "int8", "e4m3"]))
    if kind == "rotary":
        heads = rng.randint(1, 40)
        return dict(kind=kind, do=do, dtype=dtype, M=_log(rng, 1, 8192), axes=rng.choice([1, 1, 2, 3]), heads=heads,
                    rest=rng.randint(0, 8), D=rng.choice([32, 64, 80, 96, 128]), pairs=rng.random() < 0.5)
    V = _log(rng, 100, 131072)
    return dict(kind=kind, do=do, dtype=dtype, M=_log(rng, 1, 1024), V=V, K=rng.choice([0, 0, 1, 5, 20, 64]), masked=rng.choice([0, 0, V // 100]))


# ------------------------------------------------------------------ inputs

def _tdtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _offsets(case):
    """Where the sequences begin, and where the last ends: a function of the case, so that its work is known.  Uneven ones are of a quarter of the
    longest to the longest, one of them (of three or more) of no token, and one of a single token."""
    r, n, top = random.Random(case["seqs"] * 10007 + case["longest"]), case["seqs"], case["longest"]
    lens = [top if case["even"] else max(1, round(top * r.uniform(0.25, 1.0))) for _ in range(n)]
    if not case["even"]:
        if n >= 3:
            lens[1] = 0
        if n >= 4:
            lens[2] = 1
        lens[-1] = top
    off = [0]
    for k in lens:
        off.append(off[-1] + k)
    return off


def _rows(case):
    return _offsets(case)[-1] + case["tail"] if case["kind"] == "attention" else case["M"]


def _inputs(case, seed):
    """Every input of a case, from the seed alone: name -> GPU tensor."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 31)
    t, k = _tdtype(case), case["kind"]
    rn = lambda *s: torch.randn(*s, device=DEV, generator=g)                       # noqa: E731
    un = lambda lo, hi, *s: lo + (hi - lo) * torch.rand(*s, device=DEV, generator=g)  # noqa: E731
    M, v = _rows(case), {}
    if k == "attention":
        H, G, D = case["heads"], case["kv"], case["D"]
        # queries and keys of a spread that gives scores of some units: a few keys of a row carry most of its weight
        spread = torch.ones((H + 2 * G) * D, device=DEV)
        spread[:(H + G) * D] = 1.4
        v["x"] = (rn(M, (H + 2 * G) * D) * spread).to(t)
        v["off"] = torch.tensor(_offsets(case), device=DEV, dtype=torch.int64)
        if case["do"] != "forward":
            v["gy"] = rn(M, H * D).to(t)
    elif k == "rmsnorm":
        C = case["C"]
        # a hidden state: channels of different spread, a few of them large
        v["x"] = (rn(M, C) * un(0.5, 1.5, C) * torch.where(torch.rand(C, device=DEV, generator=g) < 0.01, 12.0, 1.0)).to(t)
        if case["res"]:
            v["res"] = (2.0 * rn(M, C)).to(t)
        v["gamma"] = un(0.5, 1.5, C)
        if case["do"] != "forward":
            v["gy"] = rn(M, C).to(t)
            if case["add"]:
                v["add"] = rn(M, C).to(t)
    elif k == "rotary":
        A, W = case["axes"], (case["heads"] + case["rest"]) * case["D"]
        half = case["D"] // 2
        v["x"] = rn(M, W).to(t)
        m = torch.arange(M, device=DEV)
        if A == 1:                                   # texts one behind another, the first one far into its document
            start = torch.randint(0, 30000, (1,), device=DEV, generator=g)
            pos = (m + start)[:, None]
        else:                                        # a grid, from a corner of the seed's own
            side = max(1, math.isqrt(M) // (1 if A == 2 else 2))
            axes = [m % side, (m // side) % side, m // (side * side)] if A == 3 else [m % side, m // side]
            pos = torch.stack(axes, dim=1) + torch.randint(0, 500, (1, A), device=DEV, generator=g)
        v["pos"] = pos.to(torch.int64)
        freq = torch.zeros(A, half, device=DEV)      # each pair of channels turns with one axis
        i = torch.arange(half, device=DEV)
        freq[i % A, i] = (10000.0 ** (-(i.double() / half))).float()
        v["freq"] = freq
        if case["do"] != "forward":
            v["gy"] = rn(M, W).to(t)
    else:
        V = case["V"]
        # logits: a few large ones above a broad rest; the vocabulary's last entries stand for no token and are masked
        z = rn(M, V) * 2.0
        top = torch.randint(0, V, (M, 4), device=DEV, generator=g)
        z.scatter_add_(1, top, un(2.0, 9.0, M, 4))
        if case["masked"]:
            z[:, V - case["masked"]:] = -math.inf
        v["x"] = z.to(t)
        ids = torch.randint(0, V - case["masked"], (M,), device=DEV, generator=g)
        ids = torch.where(torch.rand(M, device=DEV, generator=g) < 0.6, top[:, 0].clamp(max=V - case["masked"] - 1), ids)
        if M > 8:                                    # padding
            ids[torch.rand(M, device=DEV, generator=g) < 0.05] = -1
        v["ids"] = ids
        if case["do"] != "forward":
            v["gy"] = torch.stack([un(-1.0, 1.0, M), 0.01 * rn(M), 0.02 * rn(M)]) / M
    return v


# ------------------------------------------------------------------ plain form

def _power(e):
    """2^e in fp32, from its bits: pow() and ldexp() of a GPU may be off in the last place."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_checkpoint(x, fmt):
    """x [M, C] as its checkpoint holds it."""
    M, C = x.shape
    nb = (C + 31) // 32
    xb = torch.nn.functional.pad(x.float(), (0, nb * 32 - C)).reshape(M, nb, 32)
    most = 127.0 if fmt == "int8" else 448.0
    m, p = torch.frexp(xb.abs().amax(dim=2))                     # amax = m 2^p, m in [0.5, 1)
    unit, top = math.frexp(most)                                 # most = unit 2^top
    e = torch.where(m <= unit, p - top, p - top + 1)
    e = torch.where(m == 0, -120, e).clamp(-120, 127)
    q = xb * _power(-e)[:, :, None]
    q = torch.round(q) if fmt == "int8" else q.to(torch.float8_e4m3fn).float()
    return (q * _power(e)[:, :, None]).reshape(M, -1)[:, :C]


def _plain_attention(case, v):
    H, G, D = case["heads"], case["kv"], case["D"]
    off, x = v["off"], v["x"]
    N, L, t = case["seqs"], case["longest"], x.dtype
    at = off[:-1, None] + torch.arange(L, device=DEV)[None, :]                     # [N, L] rows of a padded batch
    there = at < off[1:, None]
    at = torch.where(there, at, 0)
    q, k, u = x.float()[at].reshape(N, L, H + 2 * G, D).transpose(1, 2).split([H, G, G], dim=1)
    q = q.reshape(N * G, -1, D)                                  # the queries of a group's heads, one behind another
    k, u = k.reshape(N * G, L, D), u.reshape(N * G, L, D)
    R = H // G
    s = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(D)).reshape(N, G * R, L, L)
    keep = there[:, None, :].expand(N, L, L)
    if case["causal"]:
        keep = keep & torch.ones(L, L, dtype=torch.bool, device=DEV).tril()
    s.masked_fill_(~keep[:, None], -math.inf)
    m = s.amax(dim=3, keepdim=True).clamp_(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(dim=3, keepdim=True)
    lse = (m + torch.log(total)).squeeze(3)
    p.div_(total)
    o = torch.bmm(p.reshape(N * G, R * L, L), u).reshape(N, H, L, D)
    sel = there.reshape(-1).nonzero().squeeze(1)
    rows = at.reshape(-1)[sel]
    y = torch.zeros(x.shape[0], H * D, device=DEV, dtype=t)
    y[rows] = o.transpose(1, 2).reshape(N * L, H * D)[sel].to(t)
    stats = torch.zeros(H, x.shape[0], device=DEV)
    stats[:, rows] = lse.transpose(0, 1).reshape(H, N * L)[:, sel]
    out = [y, stats]
    if case["do"] == "forward":
        return out
    go = v["gy"].float()[at].mul_(there[:, :, None]).reshape(N, L, H, D).transpose(1, 2)
    delta = (go * o).sum(dim=3, keepdim=True)
    go = go.reshape(N * G, R * L, D)
    gu = torch.bmm(p.reshape(N * G, R * L, L).transpose(1, 2).contiguous(), go)
    ds = torch.bmm(go, u.transpose(1, 2).contiguous()).reshape(N, H, L, L).sub_(delta).mul_(p).mul_(1.0 / math.sqrt(D)).reshape(N * G, R * L, L)
    del p
    gq = torch.bmm(ds, k)
    gk = torch.bmm(ds.transpose(1, 2).contiguous(), q)
    all_ = torch.cat([gq.reshape(N, H, L, D), gk.reshape(N, G, L, D), gu.reshape(N, G, L, D)], dim=1).transpose(1, 2).reshape(N * L, -1)
    gx = torch.zeros_like(x)
    gx[rows] = all_[sel].to(t)
    return out + [gx]


def _plain_rmsnorm(case, v):
    t, out = _tdtype(case), []
    s = v["x"]
    if case["res"]:
        s = (s.float() + v["res"].float()).to(t)
    f = s.float()
    r = 1.0 / torch.sqrt((f * f).mean(dim=1, keepdim=True) + EPS)
    sh = f * r
    y = (sh * v["gamma"]).to(t)
    out = [y] + ([s] if case["res"] else [])
    if case["pack"]:
        out.append(_plain_checkpoint(y, case["pack"]).to(torch.bfloat16))          # exact: what a checkpoint holds has 8 bits at most
    if case["do"] == "forward":
        return out
    gy = v["gy"].float()
    g = gy * v["gamma"]
    gx = r * (g - sh * (g * sh).mean(dim=1, keepdim=True))
    if case["add"]:
        gx = gx + v["add"].float()
    return out + [gx.to(t), (gy * sh).sum(dim=0)]


def _plain_turn(x, cos, sin, case):
    """x with each pair of the rotated heads' channels turned by its angle."""
    n, D, half, M = case["heads"], case["D"], case["D"] // 2, x.shape[0]
    f = x.float()
    h = f[:, :n * D].reshape(M, n, half, 2) if case["pairs"] else f[:, :n * D].reshape(M, n, 2, half).transpose(2, 3)
    a, b = h[..., 0], h[..., 1]
    h = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=3)
    if not case["pairs"]:
        h = h.transpose(2, 3)
    return torch.cat([h.reshape(M, n * D), f[:, n * D:]], dim=1).to(x.dtype)


def _plain_logprob(case, v):
    z, ids = v["x"].float(), v["ids"]
    there = (ids >= 0)[:, None]
    at = ids.clamp(min=0)[:, None]
    m = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(dim=1, keepdim=True)
    log = torch.log(total)
    lse = m + log
    H = log + (e * torch.where(e > 0, m - z, 0.0)).sum(dim=1, keepdim=True) / total
    lp = z.gather(1, at) - lse
    out = [torch.cat([lp, H, lse], dim=1).mul(there).t().contiguous()]
    if case["K"]:
        b = (z + 0.0).view(torch.int32).long()
        key = (torch.where(b < 0, b ^ 0x7FFFFFFF, b) << 32) | (0x7FFFFFFF - torch.arange(case["V"], device=DEV))    # of equal ones the lowest first
        best = 0x7FFFFFFF - (torch.topk(key, case["K"], dim=1).values & 0xFFFFFFFF)
        out += [torch.where(there, z.gather(1, best) - lse, 0.0), torch.where(there, best, -1)]
    if case["do"] == "forward":
        return out
    g1, g2, g3 = (g[:, None] for g in v["gy"])
    p = e / total
    gz = p * ((g3 - g1) - g2 * torch.where(e > 0, z - lse + H, 0.0))
    gz.scatter_add_(1, at, g1)
    return out + [gz.masked_fill_(~there, 0.0).to(v["x"].dtype)]


def _run_plain(state):
    case, v = state["case"], state["v"]
    k = case["kind"]
    if k == "attention":
        return _plain_attention(case, v)
    if k == "rmsnorm":
        return _plain_rmsnorm(case, v)
    if k == "logprob":
        return _plain_logprob(case, v)
    angle = (v["pos"].double() @ v["freq"].double())[:, None, :]                   # [M, 1, D / 2], in 64 bits: positions are far
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = [_plain_turn(v["x"], cos, sin, case)]
    if case["do"] != "forward":
        out.append(_plain_turn(v["gy"], cos, -sin, case))
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
    k, t, M = case["kind"], _tdtype(case), _rows(case)
    none = dl.NO_TENSOR
    sizes = {n: (tuple(v[n].shape), v[n].dtype) for n in ("x", "off", "res", "pos", "ids", "gy", "add") if n in v}
    given = list(sizes)
    back, W = case["do"] != "forward", v["x"].shape[1]
    wide = {"attention": case.get("heads", 0) * case.get("D", 0), "logprob": 0}.get(k, W)
    sizes["y"] = ((3, M), torch.float32) if k == "logprob" else ((M, wide), t)
    if back:
        sizes["gx"] = ((M, W), t)
    if k == "attention":
        sizes["lse"] = ((case["heads"], M), torch.float32)
    if k == "rmsnorm" and case["res"]:
        sizes["sum"] = ((M, W), t)
    if k == "rmsnorm" and case["pack"]:
        sizes["packed"], sizes["held"] = ((_packed_bytes(dl, M, W),), torch.uint8), ((M, W), torch.bfloat16)
    if k == "logprob" and case["K"]:
        sizes["best"], sizes["which"] = ((M, case["K"]), torch.float32), ((M, case["K"]), torch.int64)
    p = Program(sizes)
    for n in given:
        p.put(n, v[n])
    i = p.ids
    common = dict(x=i["x"], y=i["y"], dtype=dl.DTYPE_F32 if t == torch.float32 else dl.DTYPE_BF16, N=1, H=M, W=1, Cin=W, stride=1, pad=0, relu=0)
    if k == "attention":
        for n in ("y", "lse", "gx"):
            if n in i:
                p.view(n).fill_(math.nan)            # all of them are the operator's to write, also rows of no sequence
        fwd = dl.LayerDesc(op=dl.OP_ATTENTION_PACKED, res=i["off"], y2=i["lse"], y3=none, Cout=wide, R=case["heads"], S=case["kv"],
                           flags=dl.ATTENTION_CAUSAL if case["causal"] else 0, **common)
    elif k == "rmsnorm":
        fwd = dl.LayerDesc(op=dl.OP_RMSNORM, res=i.get("res", none), y2=i.get("sum", none), y3=i.get("packed", none), Cout=W, R=1, S=1,
                           scale=v["gamma"].data_ptr(), eps=EPS, pack={"": 0, "int8": dl.PACK_INT8, "e4m3": dl.PACK_E4M3}[case["pack"]], **common)
    elif k == "rotary":
        fwd = dl.LayerDesc(op=dl.OP_ROTARY, res=i["pos"], y2=none, y3=none, Cout=W, R=case["heads"], S=case["rest"], scale=v["freq"].data_ptr(),
                           flags=dl.ROTARY_PAIRS if case["pairs"] else 0, **common)
    else:
        fwd = dl.LayerDesc(op=dl.OP_LOGPROB, res=i["ids"], y2=i.get("best", none), y3=i.get("which", none), Cout=case["K"], R=1, S=1, **common)
    layers = [fwd]
    if "held" in i:
        layers.append(dl.LayerDesc(op=dl.OP_UNPACK8, x=i["packed"], res=none, y=i["held"], dtype=dl.DTYPE_BF16, N=1, H=M, W=1, Cin=W, Cout=W, R=1, S=1, stride=1,
                                   pad=0, relu=0, pack=fwd.pack))
    p.forward, p.backward, p.v = dl.layer_array(layers), [], v
    p.out = [p.view(n) for n in ("y", "lse", "sum", "held", "best", "which") if n in i]
    if back:
        need = p.d.backward_workspace(fwd)
        p.work = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        p.gw = torch.empty(W, device=DEV) if k == "rmsnorm" else None
        p.backward = [dl.BwdDesc(fwd=fwd, gy=i["gy"], gpre=i["gy"], gx=i["gx"], gx_add=i.get("add", none),
                                 gw=p.gw.data_ptr() if p.gw is not None else None, workspace=p.work.data_ptr(), workspace_bytes=p.work.numel())]
        p.out += [p.view("gx")] + ([p.gw] if p.gw is not None else [])
    return p


def prepare(case, seed):
    v = _inputs(case, seed)
    state = _prepare_own(case, v) if own else dict(case=case, v=v)
    torch.cuda.synchronize()
    return state


def run(state):
    if not own:
        return _run_plain(state)
    p = state
    p.begin()
    p.d.recompute_segment(p.forward)
    if p.backward:
        p.d.backward_segment(p.backward)
        p.d.backward_join()
    return p.out


# ------------------------------------------------------------------ work

def work(case):
    k, M = case["kind"], _rows(case)
    es = 4 if case.get("dtype") == "f32" else 2
    back = case["do"] != "forward"
    if k == "attention":
        off = _offsets(case)
        lens = [b - a for a, b in zip(off, off[1:])]
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
        H, G, D, T = case["heads"], case["kv"], case["D"], off[-1]
        bytes_ = T * ((H + 2 * G) * D * 2 + H * D * 2 + H * 4) + len(off) * 8
        if back:
            bytes_ += T * (H * D * 2 + (H + 2 * G) * D * 2)
        return dict(bytes=bytes_, flops=(14 if back else 4) * D * H * pairs)
    if k == "rmsnorm":
        n = M * case["C"]
        bytes_, flops = n * es * (4 if case["res"] else 2) + case["C"] * 4, 4 * n
        if case["pack"]:
            bytes_, flops = bytes_ + M * (case["C"] + (case["C"] + 31) // 32) + n * 2, flops + 6 * n
        if back:
            bytes_, flops = bytes_ + n * es * (3 if case["add"] else 2) + case["C"] * 4, flops + 9 * n
        return dict(bytes=bytes_, flops=flops)
    if k == "rotary":
        n = M * (case["heads"] + case["rest"]) * case["D"]
        turned = M * case["heads"] * case["D"]
        times = 2 if back else 1
        return dict(bytes=times * 2 * n * es + M * case["axes"] * 8 + case["axes"] * case["D"] * 2, flops=times * 3 * turned)
    n = M * case["V"]
    bytes_, flops = n * es + M * 20 + M * case["K"] * 12, 6 * n
    if back:
        bytes_, flops = bytes_ + n * es + M * 12, flops + 6 * n
    return dict(bytes=bytes_, flops=flops)


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


def _exact_attention(case, v):
    """Sequence by sequence and head by head."""
    H, G, D, T = case["heads"], case["kv"], case["D"], v["x"].shape[0]
    y, stats = torch.zeros(T, H * D, dtype=torch.float64, device=DEV), torch.zeros(H, T, dtype=torch.float64, device=DEV)
    gx = torch.zeros(v["x"].shape, dtype=torch.float64, device=DEV)
    off = _offsets(case)
    for a, b in zip(off, off[1:]):
        if a == b:
            continue
        x = v["x"][a:b].double()
        for h in range(H):
            j = h // (H // G)
            cols = [slice(h * D, h * D + D), slice((H + j) * D, (H + j + 1) * D), slice((H + G + j) * D, (H + G + j + 1) * D)]
            q, k, u = (x[:, c] for c in cols)
            s = q @ k.t() * D ** -0.5
            if case["causal"]:
                s = s + torch.full((b - a, b - a), -math.inf, dtype=torch.float64, device=DEV).triu_(1)
            lse = torch.logsumexp(s, dim=1)
            p = torch.exp(s - lse[:, None])
            o = p @ u
            y[a:b, cols[0]], stats[h, a:b] = o, lse
            if case["do"] == "forward":
                continue
            go = v["gy"][a:b, cols[0]].double()
            gx[a:b, cols[2]] += p.t() @ go
            dp = go @ u.t()
            ds = p * (dp - (p * dp).sum(dim=1, keepdim=True)) * D ** -0.5
            gx[a:b, cols[0]] = ds @ k
            gx[a:b, cols[1]] += ds.t() @ q
    return [y, stats] + ([gx] if case["do"] != "forward" else [])


def exact(case, seed):
    v, k = _inputs(case, seed), case["kind"]
    if k == "attention":
        return _exact_attention(case, v)
    if k == "rmsnorm":
        t, C = _tdtype(case), case["C"]
        s = v["x"].double()
        if case["res"]:
            s = (s + v["res"].double()).to(t).double()                             # the stored sum is what is normalised
        inv = (s.square().sum(1, keepdim=True) / C + EPS).rsqrt()
        n, gamma = s * inv, v["gamma"].double()
        out = [n * gamma] + ([s] if case["res"] else [])
        if case["pack"]:
            out.append(_exact_checkpoint((n * gamma).to(t), case["pack"]))
        if case["do"] != "forward":
            gy = v["gy"].double()
            h = gy * gamma
            gx = (C * h - n * (h * n).sum(1, keepdim=True)) * inv / C
            out += [gx + v["add"].double() if case["add"] else gx, (gy * n).sum(0)]
        return out
    if k == "rotary":
        theta = torch.zeros(case["M"], case["D"] // 2, dtype=torch.float64, device=DEV)
        for a in range(case["axes"]):
            theta += v["pos"][:, a:a + 1].double() * v["freq"][a].double()
        turn = torch.polar(torch.ones_like(theta), theta)[:, None, :]
        n, D = case["heads"], case["D"]

        def turned(x, by):
            x = x.double()
            h = x[:, :n * D].reshape(-1, n, D)
            re, im = (h[..., 0::2], h[..., 1::2]) if case["pairs"] else (h[..., :D // 2], h[..., D // 2:])
            w = torch.complex(re.contiguous(), im.contiguous()) * by
            o = torch.empty_like(h)
            if case["pairs"]:
                o[..., 0::2], o[..., 1::2] = w.real, w.imag
            else:
                o[..., :D // 2], o[..., D // 2:] = w.real, w.imag
            return torch.cat([o.reshape(-1, n * D), x[:, n * D:]], dim=1)
        return [turned(v["x"], turn)] + ([turned(v["gy"], turn.conj())] if case["do"] != "forward" else [])
    V, K = case["V"], case["K"]
    rows, best, which, gz = [], [], [], []
    for lo in range(0, case["M"], 512):                                            # some rows at a time
        z, ids = v["x"][lo:lo + 512].double(), v["ids"][lo:lo + 512]
        keep = ids >= 0
        lp = torch.log_softmax(z, dim=1)
        p = lp.exp()
        H = -(p * torch.nan_to_num(lp, neginf=0.0)).sum(1)
        mine = lp[torch.arange(len(ids), device=DEV), ids.clamp(min=0)]
        rows.append(torch.stack([mine, H, torch.logsumexp(z, dim=1)]) * keep)
        if K:
            order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
            best.append(lp.gather(1, order) * keep[:, None])
        if case["do"] != "forward":
            g = v["gy"][:, lo:lo + 512].double()
            hot = torch.zeros_like(p)
            hot[torch.arange(len(ids), device=DEV), ids.clamp(min=0)] = 1.0
            dz = g[0][:, None] * (hot - p) + g[2][:, None] * p - g[1][:, None] * p * (torch.nan_to_num(lp, neginf=0.0) + H[:, None])
            gz.append(dz * keep[:, None])
    out = [torch.cat(rows, dim=1)]
    if K:
        out += [torch.cat(best), None]
    return out + ([torch.cat(gz)] if gz else [])
