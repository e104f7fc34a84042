"""Operators with several outputs under a full arena: a call that finds no room for one of them has computed nothing, so every output's contents, on the device and
on the host, are what they were."""
import pytest

pytestmark = pytest.mark.gpu

M, C, K = 64, 64, 32


@pytest.fixture(scope="module")
def torch_mod():
    import torch
    assert torch.cuda.is_available()
    return torch


class Case:
    """x, res and the outputs, all of 8192 bytes but log probabilities' y; room in the arena for `room` tensors of them, or for all."""

    def __init__(self, torch, op, room):
        import paper_2203_15980_amd as dl
        self.torch, n = torch, M * C * 2
        norm = op == dl.OP_RMSNORM
        sizes = [n, n, n, n] if norm else [n, M * 8, M * 12, M * K * 4, M * K * 8]
        self.sizes = sizes
        held = [(s + 255) // 256 * 256 for s in sizes]
        self.arena = torch.zeros(sum(held[:room]), dtype=torch.uint8, device="cuda:0")
        self.d = dl.Delta(self.arena, torch.cuda.current_stream().cuda_stream)
        self.d.bind(sizes)
        self.gamma = torch.ones(C, device="cuda:0")
        for t in range(2):
            self.d.alloc(t)
            self.fill(t, 0)
        self.last = len(sizes) - 1
        self.layer = dl.LayerDesc(x=0, res=1, y=2, y2=3, y3=dl.NO_TENSOR if norm else 4, dtype=dl.DTYPE_BF16, N=1, H=M, W=1, Cin=C, Cout=C if norm else K, R=1, S=1, stride=1, op=op,
                                  eps=1e-6, scale=self.gamma.data_ptr() if norm else None)

    def view(self, t):
        at = self.d.tensor_ptr(t) - self.arena.data_ptr()
        return self.arena[at:at + self.sizes[t]]

    def fill(self, t, value):
        self.view(t).fill_(value)
        self.torch.cuda.synchronize()

    def whole(self, t):
        self.d.sync()
        return self.view(t).cpu().numpy()


def operators():
    import paper_2203_15980_amd as dl
    return [dl.OP_RMSNORM, dl.OP_LOGPROB]


@pytest.mark.parametrize("resident", [False, True], ids=["offloaded", "resident"])
@pytest.mark.parametrize("op", operators(), ids=["rmsnorm", "logprob"])
def test_host_copies_outlive_a_call_that_found_no_room(torch_mod, op, resident):
    """Every output but the last has a host copy, and is resident too or not; the last finds no room."""
    import paper_2203_15980_amd as dl
    s = Case(torch_mod, op, 3 if op == dl.OP_RMSNORM else 4)
    d, some = s.d, range(2, s.last)
    for t in some:
        d.alloc(t)
        s.fill(t, 40 + t)
        d.swap_out(t)
        if not resident:
            d.release(t, dl.EV_OFFLOAD)
    d.sync()
    before = d.stats()["arena_in_use"]
    with pytest.raises(dl.DeltaError) as e:
        d.recompute_segment([s.layer])
    assert e.value.status == dl.ERR_OOM_ARENA
    assert d.stats()["arena_in_use"] == before
    for t in some:
        if resident:
            assert (s.whole(t) == 40 + t).all()
            s.fill(t, 7)
            d.release(t, dl.EV_FREE)                             # its block goes, its host copy counts
        d.prefetch(t)
        assert (s.whole(t) == 40 + t).all()
    d.close()


@pytest.mark.parametrize("op", operators(), ids=["rmsnorm", "logprob"])
def test_a_call_that_found_room_outdates_the_host_copies(torch_mod, op):
    import paper_2203_15980_amd as dl
    s = Case(torch_mod, op, 5)
    d = s.d
    for t in range(2, s.last + 1):
        d.alloc(t)
        s.fill(t, 40 + t)
        d.swap_out(t)
    d.release(3, dl.EV_OFFLOAD)
    d.recompute_segment([s.layer])
    for t in range(2, s.last + 1):
        assert not (s.whole(t) == 40 + t).all()
        d.release(t, dl.EV_FREE)
        with pytest.raises(dl.DeltaError) as e:
            d.prefetch(t)
        assert "no host copy" in e.value.message
    d.close()
