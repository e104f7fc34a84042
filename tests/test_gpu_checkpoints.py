"""Activation checkpoints in 8 bits through the C ABI: every stored bit against oracle/rowops.py, and the backward
operators that read them: layer normalisation's gradients and a linear layer's weight gradient.

Packing and unpacking are exact functions: equality.  The gradients: as those of the unpacked tensor."""
import numpy as np
import pytest

from oracle import rowops as ro
from rowops_util import EPS24, Bench, half_step, layernorm_noise, storage, values

pytestmark = pytest.mark.gpu

EPS = 1e-5
FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


def _code(dl, fmt):
    return {"int8": dl.PACK_INT8, "e4m3": dl.PACK_E4M3}[fmt]


def _wild(rows, C, dtype, seed):
    """Values over the whole range of magnitudes, blocks of zeros, subnormals, the limits of a scale, infinities and NaN."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, C)) * np.exp2(rng.integers(-12, 12, (rows, 1)))
    x[rng.random((rows, C)) < 0.02] *= 300
    x = x.astype(np.float32)
    if rows > 8:
        x[1] = 0.0
        x[2] = np.float32(2.0 ** -140)
        x[3] *= np.float32(1e37)                             # some overflow to infinity here, some only when rounded
        x[4, 0] = np.inf
        x[5, C - 1] = np.nan
        x[6] = np.round(x[6] * 100)
        x[6, ::8] = 127.0
        x[7] = np.float32(2.0 ** -126)
        x[8, ::3] = -0.0
    return storage(x, dtype)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(1, 8), (1, 32), (1, 768), (2, 24), (9, 40), (11, 200), (77, 768), (130, 1016), (13, 2064), (4097, 64), (1000, 96)])
def test_every_bit_of_a_checkpoint(torch_mod, rows, C, dtype, fmt):
    print("rows", rows, "C", C, dtype, fmt, flush=True)
    x = _wild(rows, C, dtype, 10 * rows + C)
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C), x.nbytes])
    assert b.d.packed_bytes(rows, C) == b.sizes[1]
    b.put(0, x)
    b.put(1, np.full(b.sizes[1], 0x5C, np.uint8))
    k = _code(b.dl, fmt)
    pack = b.layer(b.dl.OP_PACK8, rows, C, C, 0, 1, dtype, pack=k)
    unpack = b.layer(b.dl.OP_UNPACK8, rows, C, C, 1, 2, dtype, pack=k)
    assert b.d.layer_kernel(pack) == "pack8 " + fmt and b.d.layer_kernel(unpack) == "unpack8 " + fmt
    b.d.recompute_segment([pack, unpack])
    raw = b.get(1, np.uint8, (b.sizes[1],))
    pay, sc = ro.split_packed(raw, rows, C)
    X = values(x, dtype)
    want_pay, want_sc = ro.pack(X, fmt)
    assert np.array_equal(sc, want_sc)
    good = np.repeat(want_sc != 255, 32, axis=1)[:, :C]
    differ = (pay != want_pay) & good
    assert not differ.any(), (int(differ.sum()), X[differ][:4], pay[differ][:4], want_pay[differ][:4])
    nb = -(-C // 32)
    used = np.zeros(raw.size, bool)                          # the padding keeps what was there
    used[:rows * C] = True
    used[(rows * C + 15) // 16 * 16:][:rows * nb] = True
    assert (raw[~used] == 0x5C).all()
    # what rounds up to 2^128 is an infinity in both storage types, as in any rounding to them
    back, want = values(b.get(2, x.dtype, x.shape), dtype), values(storage(ro.unpack(want_pay, want_sc, fmt), dtype), dtype)
    assert np.array_equal(back, np.where(good, want, np.nan), equal_nan=True)
    assert b.untouched()
    b.close()


def test_the_checkpoint_of_what_a_checkpoint_holds_is_the_same(torch_mod):
    rows, C = 300, 328
    rng = np.random.default_rng(3)
    for fmt in FORMATS:
        x = storage(rng.normal(size=(rows, C)), "bf16")
        b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C), x.nbytes, ro.packed_bytes(rows, C), x.nbytes])
        b.put(0, x)
        k = _code(b.dl, fmt)
        L = lambda op, i, o: b.layer(op, rows, C, C, i, o, "bf16", pack=k)       # noqa: E731
        b.d.recompute_segment([L(b.dl.OP_PACK8, 0, 1), L(b.dl.OP_UNPACK8, 1, 2), L(b.dl.OP_PACK8, 2, 3), L(b.dl.OP_UNPACK8, 3, 4)])
        assert np.array_equal(b.get(2, np.uint16, x.shape), b.get(4, np.uint16, x.shape))
        b.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,C,dtype", [(1, 8, "bf16"), (77, 768, "bf16"), (9, 1000, "bf16"), (33, 520, "f32"), (5, 1032, "bf16"), (3, 8192, "bf16"),
                                          (17, 2112, "f32"), (4500, 96, "bf16"), (1029, 1544, "bf16"), (1024, 2048, "f32"), (1023, 2048, "bf16")])
def test_layernorm_gradients_from_a_checkpoint(torch_mod, rows, C, dtype, fmt):
    print("rows", rows, "C", C, dtype, fmt, flush=True)
    rng = np.random.default_rng(rows + C)
    x, gy, add = (storage(rng.normal(size=(rows, C)) + s, dtype) for s in (1.0, 0.0, 0.0))
    gamma = rng.uniform(0.5, 1.5, C).astype(np.float32)
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C), x.nbytes, x.nbytes, x.nbytes, x.nbytes, x.nbytes])
    b.put(0, x); b.put(3, gy); b.put(5, add)
    g = b.dev(gamma)
    k = _code(b.dl, fmt)
    kw = dict(scale=g.data_ptr(), shift=g.data_ptr(), eps=EPS)
    b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, C, C, 0, 1, dtype, pack=k), b.layer(b.dl.OP_UNPACK8, rows, C, C, 1, 6, dtype, pack=k)])
    fwd = b.layer(b.dl.OP_LAYERNORM, rows, C, C, 1, 2, dtype, pack=k, **kw)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    gw, _ = b.guarded(2 * C)
    desc = b.bwd(fwd, 3, gx=4, add=5, gw=gw, ws=ws)
    assert b.d.backward_kernel(desc) == "gx, gw: layernorm from " + fmt
    b.d.backward_segment([desc])
    X = ro.unpack(*ro.pack(values(x, dtype), fmt), fmt)
    GY, ADD = values(gy, dtype), values(add, dtype)
    rgx, rdg, rdb = ro.layernorm_bwd(X, GY, gamma, EPS, ADD)
    ngx, ndg, ndb = layernorm_noise(X, GY, gamma, EPS)
    gx, got = values(b.get(4, x.dtype, x.shape), dtype), gw.cpu().numpy().astype(np.float64)
    assert (np.abs(gx - rgx) <= half_step(dtype) * np.abs(rgx) + 2 * ngx + EPS24 * np.abs(ADD)).all()
    assert (np.abs(got[:C] - rdg) <= ndg).all() and (np.abs(got[C:] - rdb) <= ndb).all()
    # the same bits as from the unpacked tensor: the same values in the same order
    first, gw2 = b.get(4, x.dtype, x.shape).copy(), b.guarded(2 * C)[0]
    b.d.backward_segment([b.bwd(b.layer(b.dl.OP_LAYERNORM, rows, C, C, 6, 2, dtype, **kw), 3, gx=4, add=5, gw=gw2, ws=ws)])
    assert np.array_equal(b.get(4, x.dtype, x.shape), first) and np.array_equal(gw2.cpu().numpy(), got.astype(np.float32))
    assert b.untouched()
    b.close()


# every tile shape: channel counts of 64 (odd), 128 (not 256), 256; one pixel, ragged slices, several slices to a worker
LINEAR = [(1, 64, 64), (63, 64, 64), (65, 128, 64), (64, 256, 64), (130, 64, 128), (333, 1024, 256), (31, 64, 256), (129, 128, 128),
          (3001, 576, 576), (2900, 640, 576), (2999, 768, 576), (3003, 576, 640), (2950, 576, 768), (4100, 1024, 1024), (700, 2048, 1024)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,Cin,Cout", LINEAR)
def test_linear_weight_gradient_from_a_checkpoint_is_exact_on_whole_numbers(torch_mod, rows, Cin, Cout, fmt):
    """x and gy whole numbers (x at most 15, held exactly by both formats), so that every product and every sum of up to 2^24
    is exact in fp32 whatever the order: equality."""
    print("rows", rows, Cin, "->", Cout, fmt, flush=True)
    rng = np.random.default_rng(rows + Cin + Cout)
    xi, gi = rng.integers(-15, 16, (rows, Cin)).astype(np.float32), rng.integers(-3, 4, (rows, Cout)).astype(np.float32)
    xi *= np.exp2(rng.integers(-2, 3, (rows, Cin // 32)).repeat(32, axis=1)).astype(np.float32)     # another scale in each block; sums stay below 2^24 / 4
    x, gy = storage(xi, "bf16"), storage(gi, "bf16")
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, Cin), gy.nbytes, gy.nbytes])
    b.put(0, x); b.put(3, gy)
    k = _code(b.dl, fmt)
    b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, Cin, Cin, 0, 1, pack=k)])
    assert np.array_equal(ro.unpack(*ro.pack(xi, fmt), fmt), xi)
    scale = b.dev(np.exp2(rng.integers(-1, 2, Cout)).astype(np.float32))
    w = b.dev(np.zeros((Cout, Cin), np.uint16).view(np.int16))
    fwd = b.layer(b.dl.OP_CONV, rows, Cin, Cout, 1, 2, pack=k, w=w.data_ptr(), scale=scale.data_ptr(), shift=scale.data_ptr())
    need = b.d.backward_workspace(fwd)
    ws, whole = b.workspace(need)
    gw, guard = b.guarded(Cout * Cin)
    desc = b.bwd(fwd, 3, gw=gw, ws=ws)
    assert b.d.backward_kernel(desc).startswith("gw: wgrad1x1 from " + fmt)
    for _ in range(2):
        gw.fill_(float("nan"))
        torch_mod.cuda.synchronize()
        b.d.backward_segment([desc])
        b.d.sync()
        want = (gi.astype(np.float64).T @ xi.astype(np.float64)) * scale.cpu().numpy().astype(np.float64)[:, None]
        got = gw.cpu().numpy().reshape(Cout, Cin)
        assert np.array_equal(got, want), (int((got != want).sum()), got.size)
    assert (guard[:64] == 12345.0).all() and (guard[64 + Cout * Cin:] == 12345.0).all() and (whole[max(need, 256):] == 0x7F).all()
    assert b.untouched()
    b.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_linear_gradients_from_a_checkpoint_beside_the_data_gradient(torch_mod, fmt):
    """A linear layer with a ReLU and a residual: gpre, gx and gw in one call, x a checkpoint; gx and gpre are those of the call with x itself."""
    rows, Cin, Cout = 700, 256, 192
    rng = np.random.default_rng(12)
    x, gy, y = (storage(rng.normal(size=(rows, c)), "bf16") for c in (Cin, Cout, Cout))
    y = storage(np.maximum(values(y, "bf16"), 0), "bf16")
    w = storage(rng.normal(size=(Cout, Cin)) / 16, "bf16")
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, Cin), y.nbytes, gy.nbytes, gy.nbytes, x.nbytes, x.nbytes])
    b.put(0, x); b.put(2, y); b.put(3, gy)
    k, one, wd = _code(b.dl, fmt), b.dev(np.ones(Cout, np.float32)), b.dev(w.view(np.int16))
    b.d.recompute_segment([b.layer(b.dl.OP_PACK8, rows, Cin, Cin, 0, 1, pack=k)])
    wt = b.dev(np.zeros((Cin, Cout), np.int16))
    kw = dict(w=wd.data_ptr(), scale=one.data_ptr(), shift=one.data_ptr(), relu=1)
    plain, held = b.layer(b.dl.OP_CONV, rows, Cin, Cout, 0, 2, **kw), b.layer(b.dl.OP_CONV, rows, Cin, Cout, 1, 2, pack=k, **kw)
    b.d.bwd_weights(plain, wt.data_ptr())
    ws, _ = b.workspace(max(b.d.backward_workspace(plain), b.d.backward_workspace(held)))
    out = []
    for fwd in (plain, held):
        gw, _ = b.guarded(Cout * Cin)
        b.d.backward_segment([b.bwd(fwd, 3, gx=5, gw=gw, ws=ws, gpre=4, wt=wt.data_ptr())])
        out.append((b.get(4, np.uint16, gy.shape).copy(), values(b.get(5, np.uint16, x.shape), "bf16"), gw.cpu().numpy().reshape(Cout, Cin).astype(np.float64)))
    assert np.array_equal(out[0][0], out[1][0])
    G, W = values(out[0][0], "bf16"), values(w, "bf16")
    bound = Cout * EPS24 * (np.abs(G) @ np.abs(W))
    for o in out:
        assert (np.abs(o[1] - G @ W) <= 2.0 ** -8 * np.abs(G @ W) + bound).all()
    X = ro.unpack(*ro.pack(values(x, "bf16"), fmt), fmt)
    assert (np.abs(out[1][2] - G.T @ X) <= rows * EPS24 * (np.abs(G).T @ np.abs(X))).all()
    b.close()


def test_a_released_and_reloaded_checkpoint(torch_mod):
    """The checkpoint is a tensor of the table: offloaded, its block reused, reloaded, and read."""
    rows, C = 64, 256
    x = storage(np.random.default_rng(4).normal(size=(rows, C)), "bf16")
    b = Bench(torch_mod, [x.nbytes, ro.packed_bytes(rows, C), x.nbytes])
    dl = b.dl
    b.put(0, x)
    pack, unpack = (b.layer(op, rows, C, C, i, o, pack=dl.PACK_INT8) for op, i, o in ((dl.OP_PACK8, 0, 1), (dl.OP_UNPACK8, 1, 2)))
    b.d.recompute_segment([pack])
    b.d.release(0, dl.EV_FREE)
    b.d.release(1, dl.EV_OFFLOAD)
    with pytest.raises(dl.DeltaError) as e:
        b.d.recompute_segment([unpack])
    assert e.value.status == dl.ERR_STATE
    b.d.prefetch(1)
    b.d.recompute_segment([unpack])
    got = b.get(2, np.uint16, x.shape)
    assert np.array_equal(values(got, "bf16"), ro.unpack(*ro.pack(values(x, "bf16"), "int8"), "int8"))
    b.close()


def test_refusals(torch_mod):
    rows, C = 16, 64
    nb, pb = rows * C * 2, ro.packed_bytes(rows, C)
    b = Bench(torch_mod, [nb, pb, nb, nb, nb, rows * 12 * 2, rows * 12 * 2])
    dl = b.dl
    one = torch_mod.ones(4096, device="cuda:0")

    def refused(call, desc):
        with pytest.raises(dl.DeltaError) as e:
            call([desc])
        assert e.value.status == dl.ERR_INVALID, e.value.message
    fw, bw = b.d.recompute_segment, b.d.backward_segment
    for pack in (0, 3, 77):
        refused(fw, b.layer(dl.OP_PACK8, rows, C, C, 0, 1, pack=pack))
        refused(fw, b.layer(dl.OP_UNPACK8, rows, C, C, 1, 0, pack=pack))
    refused(fw, b.layer(dl.OP_PACK8, rows, C, C, 0, 2, pack=1))                  # not a checkpoint's size
    refused(fw, b.layer(dl.OP_UNPACK8, rows, C, C, 0, 2, pack=1))
    refused(fw, b.layer(dl.OP_PACK8, rows, C, 2 * C, 0, 1, pack=1))
    refused(fw, b.layer(dl.OP_PACK8, rows, C, C, 0, 1, pack=1, res=2))
    refused(fw, b.layer(dl.OP_PACK8, rows, C, C, 1, 1, pack=1))
    refused(fw, b.layer(dl.OP_PACK8, rows, 12, 12, 5, 6, pack=1))                # channels
    kw = dict(scale=one.data_ptr(), shift=one.data_ptr(), eps=EPS)
    refused(fw, b.layer(dl.OP_LAYERNORM, rows, C, C, 1, 2, pack=1, **kw))        # a forward pass reads the tensor itself
    refused(fw, b.layer(dl.OP_RELU, rows, C, C, 1, 2, pack=1))
    lin = dict(w=one.data_ptr(), scale=one.data_ptr(), shift=one.data_ptr())
    refused(fw, b.layer(dl.OP_CONV, rows, C, C, 1, 2, pack=1, **lin))
    gw, _ = b.guarded(C * C)
    fwd = b.layer(dl.OP_CONV, rows, C, C, 1, 2, pack=1, **lin)
    ws, _ = b.workspace(b.d.backward_workspace(fwd))
    refused(bw, b.bwd(fwd, 3, gw=gw, ws=ws, gx=4, mask_gx=1, wt=one.data_ptr()))
    refused(bw, b.bwd(fwd, 3, gw=gw, ws=ws, workspace_bytes=128))
    refused(bw, b.bwd(fwd, 3, gw=gw))
    refused(bw, b.bwd(b.layer(dl.OP_RELU, rows, C, C, 1, 2, pack=1), 3, gx=4))
    refused(bw, b.bwd(b.layer(dl.OP_CONV, rows // 4, C, C, 1, 2, pack=1, W=4, R=3, S=3, pad=1, **lin), 3, gw=gw, ws=ws))
    b.close()


@pytest.mark.parametrize("shape", [dict(N=16, H=1), dict(N=1, H=16)])
def test_making_and_restoring_a_checkpoint_have_no_backward(torch_mod, shape):
    """Neither is taken for the classifier, whose layers are [N, 1, 1] too and which reads weights that these have not."""
    rows, C = 16, 8
    nb, pb = rows * C * 2, ro.packed_bytes(rows, C)
    b = Bench(torch_mod, [nb, pb, nb, nb, pb, nb])
    dl = b.dl
    gw, _ = b.guarded(C * C)
    ws, _ = b.workspace(4096)
    for i in (0, 1, 2, 4):
        b.put(i, np.zeros((nb, pb, nb, nb, pb)[i], np.uint8))
    for op, x, y, gy, gx in ((dl.OP_PACK8, 0, 1, 4, 3), (dl.OP_UNPACK8, 1, 2, 0, 4)):
        fwd = b.layer(op, rows, C, C, x, y, pack=dl.PACK_INT8, **shape)
        for desc in (b.bwd(fwd, gy, gx=gx), b.bwd(fwd, gy, gw=gw, ws=ws), b.bwd(fwd, gy, gx=gx, gw=gw, ws=ws)):
            for call in (lambda: b.d.backward_segment([desc]), lambda: b.d.backward_kernel(desc)):
                with pytest.raises(dl.DeltaError) as e:
                    call()
                assert e.value.status == dl.ERR_INVALID, e.value.message
    b.close()
