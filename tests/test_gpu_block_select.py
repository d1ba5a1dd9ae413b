"""Chosen blocks: equal to the choice by exact scores."""
import math

import pytest
import torch

import cache_reference as ref
from cache_util import host, make

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def check(s, block, K, first=1, last=1, stream=None):
    sel = _comet().comet_block_select(s["q"], s["mean"], s["table"], s["pos"], s["length"], block, K, first=first, last=last, stream=stream)
    torch.cuda.synchronize()
    want = ref.block_select(host(s["q"]), host(s["mean"]), s["table"].tolist(), s["pos"].tolist(), s["length"].tolist(), block, K, first, last)
    got = sel.tolist()
    for r in want:
        assert got[r] == want[r], r
    return sel


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G,D", [(1, 1, 8), (2, 4, 64), (3, 5, 72), (8, 2, 128), (1, 16, 256)])
@pytest.mark.parametrize("news,lengths", [([1], [1]), ([1, 1, 1], [16, 17, 700]), ([3, 0, 5], [3, 40, 300]), ([70], [500]), ([20, 33], [20, 1000])])
def test_sizes(news, lengths, H, G, D, dtype):
    s = make(news, lengths, H, G, D, 16, dtype, seed=sum(news))
    for K in (2, 5, 40):
        check(s, 16, K)


@pytest.mark.parametrize("first,last,K", [(0, 1, 1), (0, 1, 7), (2, 1, 3), (0, 6, 6), (3, 4, 9), (1, 30, 40)])
def test_first_and_last(first, last, K):
    s = make([1, 18], [900, 600], 2, 3, 64, 16, torch.bfloat16)
    check(s, 16, K, first, last)


@pytest.mark.parametrize("length,block,K", [(16384, 16, 33), (40000, 16, 64), (100000, 16, 1024), (262000, 16, 500), (20000, 48, 17)])
def test_long_contexts(length, block, K):
    # a cache is not needed for the choice: means alone
    g = torch.Generator().manual_seed(length)
    M = -(-length // block)
    s = dict(q=torch.randn((3, 4, 64), generator=g).bfloat16(), mean=torch.randn((M + 2, 2, 64), generator=g).bfloat16(),
             table=torch.randperm(M + 2, generator=g)[None, :M].int(), pos=torch.tensor([0, 3], dtype=torch.int32), length=torch.tensor([length], dtype=torch.int32))
    check({n: t.cuda() for n, t in s.items()}, block, K)


@pytest.mark.parametrize("N", [1, 40])
def test_equal_scores_and_nan(N):
    s = make([N], [1000], 2, 2, 64, 16, torch.float32, seed=1)
    s["mean"][:] = 0.5
    check(s, 16, 9)                                    # all equal: the lowest
    s["mean"][s["table"][0, 10:30].long()] = math.nan
    check(s, 16, 45)
    s["mean"][s["table"][0, 3].long()] = math.inf
    s["mean"][s["table"][0, 5].long(), :, 0] = -math.inf
    check(s, 16, 9)
    s["mean"][:] = math.nan
    check(s, 16, 9)
    s["q"][:] = 0
    s["mean"][:] = torch.randn(s["mean"].shape, device="cuda")
    check(s, 16, 4)


@pytest.mark.parametrize("N", [1, 24])
def test_blocks_that_are_none(N):
    s = make([N], [700], 2, 2, 64, 16, torch.float16, seed=2)
    s["table"][0, 4], s["table"][0, 9], s["table"][0, 12] = -1, s["mean"].shape[0], 2 ** 31 - 1
    check(s, 16, 20)
    check(s, 16, 42)


def test_rows_behind_the_last_sequence_and_lengths_that_are_too_small():
    comet = _comet()
    s = make([2, 3], [100, 90], 2, 2, 64, 16, torch.bfloat16)
    s["length"][1] = 2                                 # its first token would be at place -1
    q = torch.cat([s["q"], s["q"]])
    sel = torch.full((10, 2, 4), 77, dtype=torch.int32, device="cuda")
    got = comet.comet_block_select(q, s["mean"], s["table"], s["pos"], s["length"], 16, 4, sel=sel)
    assert got is sel and bool((sel[5:] == 77).all())
    assert sel[2].tolist() == [[-1] * 4] * 2 and sel[3].tolist() == [[0, -1, -1, -1]] * 2
    want = check({**s, "length": s["length"].clone()}, 16, 4)
    assert torch.equal(want, sel[:5])


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(dtype):
    s = make([2, 17], [300, 400], 3, 2, 64, 16, dtype, seed=4)
    want = check(s, 16, 6)
    q = torch.zeros((6, 19, 72), dtype=dtype, device="cuda").transpose(0, 1)[..., :64].copy_(s["q"])
    mean = torch.zeros((3, s["mean"].shape[0], 80), dtype=dtype, device="cuda").transpose(0, 1)[..., :64].copy_(s["mean"])
    table = torch.zeros((2, 99), dtype=torch.int32, device="cuda")[:, :s["table"].shape[1]].copy_(s["table"])
    assert torch.equal(_comet().comet_block_select(q, mean, table, s["pos"], s["length"], 16, 6), want)


def test_close_scores_are_told_apart():
    """Scores that 32 bits do not tell apart: large parts that cancel."""
    s = make([20], [640], 1, 2, 64, 16, torch.float32, seed=6)
    s["q"][:, 1] = -s["q"][:, 0]
    s["q"][:, 1, 5] += 1e-4                            # the heads' sum is small
    s["mean"][:, :, :5] *= 1e4
    check(s, 16, 8)


def test_captured_and_replayed_on_another_stream():
    comet = _comet()
    s = make([1] * 8 + [40], [200 + i for i in range(8)] + [600], 2, 2, 64, 16, torch.bfloat16, seed=8)
    side = torch.cuda.Stream()
    call = lambda stream=None: comet.comet_block_select(s["q"], s["mean"], s["table"], s["pos"], s["length"], 16, 5, stream=stream)
    want = call()
    side.wait_stream(torch.cuda.current_stream())
    other = call(side)
    torch.cuda.synchronize()
    assert torch.equal(want, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(3):
        s["q"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())
        check(s, 16, 5)
