"""What the GPU tests of the row operators share: a context over a small arena whose tensors are filled and read as
numpy arrays, storage conversions, and the operators' descriptors."""
import numpy as np

import synth

EPS24 = 2.0 ** -24          # half a step of fp32, relative


def storage(a, dtype):
    """float array -> stored array (fp32, or bf16 bits as uint16)."""
    a = np.ascontiguousarray(a, np.float32)
    return a if dtype == "f32" else synth.f32_to_bf16_bits(a).reshape(a.shape)


def values(stored, dtype):
    return np.asarray(stored, np.float64) if dtype == "f32" else synth.bf16_bits_to_f32(stored).astype(np.float64).reshape(stored.shape)


def half_step(dtype):
    """Relative rounding of the storage type: half of finfo.eps."""
    return EPS24 if dtype == "f32" else 2.0 ** -8


class Bench:
    """A context over tensors of the given byte sizes, all resident; every byte of the arena starts as 0xA5."""

    def __init__(self, torch, sizes, stream=None, extra=1 << 20):
        import paper_2203_15980_amd as dl
        self.torch, self.dl, self.sizes = torch, dl, [int(s) for s in sizes]
        room = sum((s + 255) // 256 * 256 for s in self.sizes) + extra
        self.arena = torch.full((room,), 0xA5, dtype=torch.uint8, device="cuda:0")
        torch.cuda.synchronize()
        self.d = dl.Delta(self.arena, (stream or torch.cuda.current_stream()).cuda_stream)
        self.d.bind(self.sizes)
        self.keep = []
        self.at = []
        for i in range(len(self.sizes)):
            self.at.append(self.d.alloc(i) - self.arena.data_ptr())

    def put(self, i, a):
        a = np.ascontiguousarray(a)
        assert a.nbytes == self.sizes[i]
        self.arena[self.at[i]:self.at[i] + a.nbytes].copy_(self.torch.from_numpy(a.view(np.uint8).reshape(-1)))
        self.torch.cuda.synchronize()

    def get(self, i, dtype, shape):
        self.d.sync()
        return self.arena[self.at[i]:self.at[i] + self.sizes[i]].cpu().numpy().view(dtype).reshape(shape)

    def dev(self, a):
        t = self.torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
        self.keep.append(t)
        return t

    def untouched(self):
        """No byte outside the tensors has been written."""
        self.d.sync()
        mask = np.ones(self.arena.numel(), bool)
        for o, s in zip(self.at, self.sizes):
            mask[o:o + s] = False
        return bool((self.arena.cpu().numpy()[mask] == 0xA5).all())

    def guarded(self, n):
        """fp32 device buffer of n values between guards; returns (view, whole)."""
        whole = self.torch.full((n + 128,), 12345.0, dtype=self.torch.float32, device="cuda:0")
        self.keep.append(whole)
        return whole[64:64 + n], whole

    def workspace(self, n):
        w = self.torch.full((max(int(n), 256) + 256,), 0x7F, dtype=self.torch.uint8, device="cuda:0")     # NaN patterns: nothing in it may be relied on
        self.keep.append(w)
        return w[:max(int(n), 256)], w

    def layer(self, op, rows, cin, cout, x, y, dtype="bf16", **kw):
        dl = self.dl
        base = dict(x=x, res=dl.NO_TENSOR, y=y, dtype=dl.DTYPE_F32 if dtype == "f32" else dl.DTYPE_BF16, N=1, H=rows, W=1, Cin=cin, Cout=cout,
                    R=1, S=1, stride=1, pad=0, relu=0, op=op)
        base.update(kw)
        return dl.LayerDesc(**base)

    def bwd(self, fwd, gy, gx=None, add=None, gw=None, ws=None, **kw):
        dl = self.dl
        base = dict(fwd=fwd, gy=gy, gpre=gy, gx=dl.NO_TENSOR if gx is None else gx, gx_add=dl.NO_TENSOR if add is None else add,
                    gw=gw.data_ptr() if gw is not None else None, workspace=ws.data_ptr() if ws is not None else None,
                    workspace_bytes=ws.numel() if ws is not None else 0)
        base.update(kw)
        return dl.BwdDesc(**base)

    def close(self):
        self.d.close()


def layernorm_noise(x, gy, gamma, eps):
    """Bounds on what fp32 arithmetic may add to gx (per row) and to dgamma and dbeta (per channel).  A sum of n values
    in a tree of depth <= 40 (8 values a lane and round, 64 lanes, 16 wavefronts, and the roundings of its terms) is off
    by 40 * 2^-24 of the sum of magnitudes; with X = max|x| r, H = max|xh|, G = max|g|: xh is off by 40 e (X + H), both means
    by 40 e G plus G times that of xh, and gx / r by the sum of its three terms' errors."""
    x, gy = np.asarray(x, np.float64), np.asarray(gy, np.float64)
    c = x - x.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    X, H = np.abs(x).max(axis=1, keepdims=True) * r, np.abs(c * r).max(axis=1, keepdims=True)
    G = np.abs(gy * gamma).max(axis=1, keepdims=True)
    e = 40 * EPS24
    gx = r * e * G * (3 + (1 + H) * (1 + X + H))
    # sums over the rows: at most rows / 8 + 80 terms in a chain
    depth = (x.shape[0] / 8 + 80) * EPS24
    dg = (np.abs(gy) * (e * (X + H) + depth * np.abs(c * r))).sum(axis=0)
    db = depth * np.abs(gy).sum(axis=0)
    return gx, dg, db
