"""Chosen blocks of tokens that share a workgroup, of requests with up to 1024 blocks, and of tables that are wider than their requests."""
import pytest
import torch

from test_gpu_block_select import DTYPES, check

pytestmark = pytest.mark.gpu


def make(news, lengths, H, G, D, block, dtype, seed, M=None):
    """Means alone: a cache is not needed for the choice."""
    g = torch.Generator().manual_seed(seed)
    B, N = len(news), sum(news)
    held = [-(-n // block) for n in lengths]
    M = M or max(held)
    P = sum(held) + 3
    ids = torch.randperm(P, generator=g).int()
    table = torch.full((B, M), -7, dtype=torch.int32)
    for b in range(B):
        table[b, :held[b]], ids = ids[:held[b]], ids[held[b]:]
    s = dict(q=torch.randn((N, H * G, D), generator=g).to(dtype), mean=torch.randn((P, H, D), generator=g).to(dtype), table=table,
             pos=torch.tensor([0] + torch.tensor(news).cumsum(0).tolist(), dtype=torch.int32), length=torch.tensor(lengths, dtype=torch.int32))
    return {n: t.cuda() for n, t in s.items()}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G,D", [(1, 4, 64), (2, 1, 128), (1, 2, 256), (1, 3, 72)])
@pytest.mark.parametrize("blocks", [100, 128, 129, 200, 256, 257, 400, 512, 513, 900, 1024])
def test_sixteen_tokens_a_workgroup(blocks, H, G, D, dtype):
    s = make([19, 7], [16 * blocks - 3, 16 * (blocks // 3) + 5], H, G, D, 16, dtype, seed=blocks)
    for K in (3, 32, 90):
        check(s, 16, K, first=1, last=2)


@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("blocks", [256, 512, 1024])
def test_many_of_many(blocks, equal):
    s = make([18], [16 * blocks], 1, 2, 64, 16, torch.float32, seed=blocks)
    if equal:
        s["mean"][:] = s["mean"][:1]
        s["mean"][::5] = float("nan")
    for K in (blocks // 2, blocks - 1):
        check(s, 16, K, first=2, last=3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1024, 1025, 2048, 16384])
def test_a_table_that_is_wider_than_its_requests(M, dtype):
    """The answer is that for the table cut to the longest request."""
    s = make([17, 4, 1], [1700, 700, 33], 2, 2, 64, 16, dtype, seed=3, M=M)
    wide = check(s, 16, 9)
    cut = check({**s, "table": s["table"][:, :107]}, 16, 9)
    assert torch.equal(wide, cut)


def test_prompts_that_see_more_than_1024_blocks():
    check(make([18, 5], [16 * 1300, 16 * 1030], 1, 2, 64, 16, torch.bfloat16, seed=4), 16, 50)
