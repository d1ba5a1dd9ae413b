"""Attention where one place has nearly all of the weight and a value of 0: what comes out is the sum of many weights far below it."""
import pytest
import torch

from test_gpu_block_attend import DTYPES, check

pytestmark = pytest.mark.gpu


def make(news, places, gap, D, dtype, H=1, G=4, block=64):
    """Scores are 0 but for place 5 of every request, where they are `gap`; values are 3/4 to 1, there 0."""
    g = torch.Generator().manual_seed(int(gap * 8) + places)
    B, N, M = len(news), sum(news), -(-places // block)
    q, K, V = torch.zeros((N, H * G, D)), torch.randn((B * M, block, H, D), generator=g), torch.rand((B * M, block, H, D), generator=g) * 0.25 + 0.75
    q[:, :, 0], K[..., 0] = 1, 0
    K[::M, 5, :, 0], V[::M, 5] = gap, 0
    s = dict(q=q.to(dtype), K=K.to(dtype), V=V.to(dtype), table=torch.arange(B * M, dtype=torch.int32).view(B, M),
             pos=torch.tensor([0] + torch.tensor(news).cumsum(0).tolist(), dtype=torch.int32), length=torch.full((B,), places, dtype=torch.int32),
             sel=torch.arange(M, dtype=torch.int32).expand(N, H, M).contiguous())
    return {n: t.cuda() for n, t in s.items()}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("gap", [6.0, 10.0, 12.0, 13.0, 14.0, 15.0, 16.0, 17.5, 20.0, 26.0])
def test_many_small_weights(gap, D, dtype):
    check(make([1, 9], 2048, gap, D, dtype), scale=1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gap", [14.0, 17.5, 24.0])
def test_of_a_long_request(gap, dtype):
    check(make([2], 32768, gap, 64, dtype), scale=1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("step", [2.0, 0.25])
def test_scores_that_rise_and_fall(step, dtype):
    """The maximum is met late, and what was added up before it is scaled down; weights of all sizes."""
    s = make([1, 20], 640, 0.0, 128, dtype)
    rise = torch.arange(640, device="cuda") * step % 61
    s["K"][..., 0] = rise.view(10, 64, 1).repeat(2, 1, 1).to(dtype)
    check(s, scale=0.5)
    s["K"][..., 0] = -s["K"][..., 0]
    check(s, scale=0.5)


def test_values_below_the_normal_ones():
    s = make([1, 9], 300, 3.0, 64, torch.float16)
    s["V"] = (s["V"].float() * 2.0 ** -16).half()                    # of ten bits of 16-bit float, seven to eight are left
    out, _ = check(s, scale=1.0)
    assert bool((out > 0).all())
