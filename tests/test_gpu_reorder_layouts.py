"""States whose dimensions are not in the order of their memory."""
import pytest
import torch

from test_gpu_beam import check_reorder, parents, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8])
def test_transposed_caches(dtype):
    x = state((2, 4, 3, 50, 16), dtype, 1)                       # [B, W, heads, places, dim]
    check_reorder([x.transpose(2, 3)], parents(2, 4, 1))
    check_reorder([x.permute(0, 1, 4, 2, 3)], parents(2, 4, 2))
    check_reorder([x[:, :, :, :37].transpose(2, 3)], parents(2, 4, 3))
    check_reorder([x[:, :, 1].transpose(2, 3)], parents(2, 4, 4))
    check_reorder([x.transpose(2, 4), state((2, 4, 6), torch.int32, 2).transpose(0, 0)], parents(2, 4, 5))


def test_refusals():
    import paper_2102_05187_amd as comet
    par = parents(2, 4, 0)
    x = state((2, 4, 3, 4, 6), torch.float32, 0)
    with pytest.raises(ValueError):
        comet.comet_beam_reorder([x[:, :, :, :2, :3].transpose(2, 3)], par)
    with pytest.raises((ValueError, comet.CometError)):
        comet.comet_beam_reorder([x[:, :, :1].expand(2, 4, 3, 4, 6)], par)


def test_a_refused_layout_moves_none_of_the_others():
    import paper_2102_05187_amd as comet
    x = state((2, 4, 30), torch.float32, 1)
    before = x.clone()
    with pytest.raises(ValueError):
        comet.comet_beam_reorder([x, state((2, 4, 3, 4, 6), torch.float32, 0)[:, :, :, :2, :3]], parents(2, 4, 6))
    torch.cuda.synchronize()
    assert torch.equal(x, before)
