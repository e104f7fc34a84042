"""A layer's further outputs that a caller of the Python binding leaves out: none, not the tensor of id 0."""
import numpy as np
import pytest

import paper_2203_15980_amd as dl


def test_further_outputs_left_out_are_none():
    for d in (dl.LayerDesc(), dl.LayerDesc(op=dl.OP_LOGPROB, x=3), dl.LayerDesc(1, 2, 3, dl.DTYPE_F32)):
        assert d.y2 == d.y3 == dl.NO_TENSOR
        assert d.flags == d.pack == d.fuse == 0
    assert dl.LayerDesc(1, 2, 3, dl.DTYPE_F32).y == 3


def test_further_outputs_that_are_given_stay():
    names = [n for n, _ in dl.LayerDesc._fields_]
    given = dl.LayerDesc(*[0] * names.index("y2"), 5, y3=6)
    assert (given.y2, given.y3) == (5, 6)
    assert (dl.LayerDesc(y2=0).y2, dl.LayerDesc(y2=0).y3) == (0, dl.NO_TENSOR)
    both = dl.LayerDesc(*[0] * names.index("y2"), 0, 7, 1)
    assert (both.y2, both.y3, both.flags) == (0, 7, 1)


def test_descriptors_keep_them_in_arrays_and_backward_descriptors():
    arr = dl.layer_array([dict(x=1, op=dl.OP_RMSNORM), dl.LayerDesc(y2=4)])
    assert [(d.y2, d.y3) for d in arr] == [(dl.NO_TENSOR, dl.NO_TENSOR), (4, dl.NO_TENSOR)]
    assert dl.BwdDesc(fwd=dl.LayerDesc(x=2), gy=1).fwd.y2 == dl.NO_TENSOR


@pytest.mark.gpu
def test_attention_writes_no_log_sum_exp_that_nobody_asked_for():
    """Tensor 0 has just its bytes."""
    import torch
    rng = np.random.default_rng(1)
    M, H, D = 50, 2, 64
    arena = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda:0")
    d = dl.Delta(arena, torch.cuda.current_stream().cuda_stream)
    sizes = [H * M * 4, M * 3 * H * D * 2, 16, M * H * D * 2]
    d.bind(sizes)
    at = [d.alloc(i) - arena.data_ptr() for i in range(4)]
    arena[at[0]:at[0] + sizes[0]] = 0x5A
    arena[at[1]:at[1] + sizes[1]] = torch.from_numpy(rng.integers(0, 60, sizes[1]).astype(np.uint8)).to("cuda:0")
    arena[at[2]:at[2] + 16] = torch.tensor([0, M], dtype=torch.int64).view(torch.uint8).to("cuda:0")
    torch.cuda.synchronize()
    d.recompute_segment([dict(op=dl.OP_ATTENTION_PACKED, x=1, res=2, y=3, dtype=dl.DTYPE_BF16, N=1, H=M, W=1, Cin=3 * H * D, Cout=H * D, R=H, S=H, stride=1)])
    d.sync()
    assert (arena[at[0]:at[0] + sizes[0]] == 0x5A).all()
    assert arena[at[3]:at[3] + sizes[3]].any()
    d.close()
