"""Attention over chosen blocks against the plain implementation in 64 bits."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref
from cache_util import host, make

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def check(s, scale=None, call=None):
    comet = _comet()
    call = call or (lambda: comet.comet_block_attend(s["q"], s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"], scale=scale))
    out, lse = call()
    torch.cuda.synchronize()
    dtype, D = s["q"].dtype, s["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    q, K, V = host(s["q"]), host(s["K"]), host(s["V"])
    want = ref.block_attend(q, K, V, s["table"].tolist(), s["pos"].tolist(), s["length"].tolist(), s["sel"].tolist(), scale)
    got, got_lse = host(out), host(lse)
    unit, half = ref.UNIT[dtype], 2.0 ** -24
    places = s["sel"].shape[2] * s["K"].shape[1]
    size = np.nanmax(np.abs(np.where(np.isfinite(K), K, 0)))
    for r, (o, l, mass) in want.items():
        # a score is a sum of D products in 32 bits, and is rounded a few times more (scaled, the maximum taken off)
        score = half * (D + 16) * scale * np.abs(q[r]).sum(1) * size * 1.5 + half * 16
        fine = np.isfinite(o)
        # a weight is off by twice that (its own score, and all others in the sum), rounded to the type before it meets the values, and
        # added up in 32 bits: the longest chain of additions is all places; the result is rounded once
        weight = 2 * score[:, None] * 1.05 + unit * (dtype != torch.float32) + half * (places + 64)
        tolerance = (weight * mass * 1.01 + unit * np.abs(o) * 1.01 + (2.0 ** -24 if dtype == torch.float16 else 1e-37))
        assert np.array_equal(np.isnan(o), np.isnan(got[r])), r
        assert np.all(np.abs(got[r] - o)[fine] <= tolerance[fine]), (r, np.max((np.abs(got[r] - o) / tolerance)[fine]))
        ok = np.isfinite(l)
        assert np.array_equal(l[~ok & ~np.isnan(l)], got_lse[r][~ok & ~np.isnan(l)]) and np.array_equal(np.isnan(l), np.isnan(got_lse[r]))
        assert np.all(np.abs(got_lse[r] - l)[ok] <= (score + half * (places + 64) + 4 * half * np.abs(l))[ok]), r
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G,D", [(1, 1, 8), (2, 4, 64), (3, 5, 72), (1, 12, 80), (2, 8, 128), (1, 3, 136), (1, 16, 256), (1, 40, 64), (1, 70, 96)])
@pytest.mark.parametrize("news,lengths,K", [([1], [1], 1), ([1, 1, 1], [16, 17, 300], 4), ([3, 0, 5, 1], [3, 40, 300, 33], 7), ([30], [100], 3), ([21, 37], [21, 400], 9)])
def test_sizes(news, lengths, K, H, G, D, dtype):
    check(make(news, lengths, H, G, D, 16, dtype, seed=sum(news) + D, K=K))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block", [16, 32, 48, 64, 128, 1024])
def test_blocks(block, dtype):
    check(make([1, 2, 9], [block, 3 * block + 1, 5 * block - 3], 2, 2, 64, block, dtype, seed=block, K=3))


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_blocks_of_one_token(dtype):
    check(make([1, 4], [6000, 5990], 2, 4, 128, 16, dtype, seed=1, K=300))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread", [0.0, 8.0, 60.0])
def test_flat_and_sharp_weights(dtype, spread):
    check(make([2, 20], [200, 150], 2, 2, 64, 32, dtype, seed=2, K=4, spread=spread))


def test_scale():
    s = make([2, 20], [200, 150], 2, 2, 64, 32, torch.bfloat16, seed=3, K=4)
    check(s, scale=0.5)
    check(s, scale=1e-20)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("news", [[1, 1], [3, 18]])
def test_choices_that_are_sets(news, dtype):
    """No order, blocks named twice, numbers that are none, rows that choose nothing."""
    s = make(news, [200, 150], 2, 4, 64, 16, dtype, seed=4, K=6)
    want = check(s)
    g = torch.Generator().manual_seed(1)
    sel = s["sel"].cpu()
    mixed = torch.cat([sel, sel.flip(2), torch.full_like(sel, -1)], 2)[:, :, torch.randperm(18, generator=g)]
    got = check({**s, "sel": mixed.cuda().contiguous()})
    unit = ref.UNIT[dtype]
    assert bool(((got[0].double() - want[0].double()).abs() <= 4 * unit * (1 + want[0].double().abs())).all())
    none = torch.tensor([-1, 13, 2 ** 31 - 1, -2 ** 31, 500, 12])
    check({**s, "sel": none[torch.randint(6, sel.shape, generator=g)].int().cuda()})
    s["sel"][::2] = -1
    out, lse = check(s)
    assert bool((out[::2] == 0).all()) and bool((lse[::2] == -math.inf).all())


def test_blocks_that_are_not_in_the_cache():
    s = make([2, 18], [200, 150], 2, 2, 64, 16, torch.float16, seed=5, K=5)
    s["table"][0, 3], s["table"][1, 2], s["table"][1, 9] = -1, s["K"].shape[0], 2 ** 31 - 1
    s["sel"][:, :, 0] = 2
    check(s)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_a_token_does_not_read_does_not_reach_it(dtype, bad):
    """Several tokens share the work: a value that only one of them reads, or only the later ones, is not the others'."""
    s = make([12], [140], 1, 2, 64, 16, dtype, seed=6, K=4)
    s["sel"][:, 0] = torch.tensor([8, 1, -1, -1])
    s["sel"][5, 0] = torch.tensor([8, 3, 1, -1])
    s["V"][s["table"][0, 3].long(), 4, 0, 7] = bad          # row 5's alone
    s["V"][s["table"][0, 8].long(), 7, 0, 9] = -bad         # place 135: rows 7 and behind
    out, lse = check(s)
    assert bool(torch.isfinite(out[:5]).all()) and bool(torch.isfinite(out[6]).all()) and bool(torch.isfinite(lse).all())
    s["K"][s["table"][0, 8].long(), 9, 0, 3] = math.nan     # place 137
    out, lse = _comet().comet_block_attend(s["q"], s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"])
    assert bool(torch.isfinite(out[6]).all()) and bool(torch.isfinite(lse[:9]).all()) and bool(torch.isnan(lse[9:]).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_that_are_infinite(dtype):
    s = make([1, 17], [60, 60], 1, 2, 64, 16, dtype, seed=7, K=4)
    s["q"][:, :, 0] = 1
    s["K"][s["table"][:, 0].long(), 3, 0, 0] = -math.inf    # a place that weighs nothing
    check(s)
    s["K"][s["table"][:, :3].long(), :, 0, 0] = -math.inf
    s["sel"][:, 0] = torch.tensor([0, 1, -1, -1])           # none that weighs anything
    out, lse = check(s)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_rows_behind_the_last_sequence_and_lengths_that_are_too_small():
    comet = _comet()
    s = make([2, 3], [100, 90], 2, 2, 64, 16, torch.bfloat16, K=4)
    s["length"][1] = 2
    q, sel = torch.cat([s["q"], s["q"]]), torch.cat([s["sel"], s["sel"]])
    sel[2:5] = 0
    out, lse = torch.full((10, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((10, 4), 7.0, device="cuda")
    got = comet.comet_block_attend(q, s["K"], s["V"], s["table"], s["pos"], s["length"], sel, out=out, lse=lse)
    assert got[0] is out and got[1] is lse and bool((out[5:] == 7).all()) and bool((lse[5:] == 7).all())
    assert bool((out[2] == 0).all()) and bool((lse[2] == -math.inf).all()) and bool(torch.isfinite(lse[3:5]).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(dtype):
    """Heads outside of places, rows with room behind them, K and V in one memory."""
    s = make([2, 17], [300, 200], 3, 2, 64, 16, dtype, seed=9, K=5)
    want = check(s)
    P = s["K"].shape[0]
    both = torch.zeros((P, 3, 2, 16, 72), dtype=dtype, device="cuda")
    K, V = both[:, :, 0, :, :64].transpose(1, 2).copy_(s["K"]), both[:, :, 1, :, :64].transpose(1, 2).copy_(s["V"])
    q = torch.zeros((6, 19, 80), dtype=dtype, device="cuda").transpose(0, 1)[..., :64].copy_(s["q"])
    table = torch.zeros((2, 99), dtype=torch.int32, device="cuda")[:, :s["table"].shape[1]].copy_(s["table"])
    got = _comet().comet_block_attend(q, K, V, table, s["pos"], s["length"], s["sel"])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_cache_of_more_than_4_gib():
    comet = _comet()
    P, block, H, D = 70000, 64, 4, 128                      # 4.6 GB each
    K, V = (torch.zeros((P, block, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids = [P - 1, 3, P - 2, 40000]
    for p in ids:
        K[p].normal_(), V[p].normal_()
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    q = torch.randn((5, 8, D), device="cuda").bfloat16()
    pos, length = torch.tensor([0, 5], dtype=torch.int32, device="cuda"), torch.tensor([250], dtype=torch.int32, device="cuda")
    sel = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda").expand(5, H, 4).contiguous()
    got = comet.comet_block_attend(q, K, V, table, pos, length, sel)
    near = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    small = comet.comet_block_attend(q, K[ids].contiguous(), V[ids].contiguous(), near, pos, length, sel)
    assert torch.equal(got[0], small[0]) and torch.equal(got[1], small[1])
    check(dict(q=q, K=K[ids].contiguous(), V=V[ids].contiguous(), table=near, pos=pos, length=length, sel=sel))


def test_more_than_the_last_cache_holds():
    """From 256 MB of chosen keys and values on they are read past it; every token reads all of its request's 2560 places."""
    B, H, G, D, block, blocks = 16, 8, 4, 128, 64, 40
    L = block * blocks - 5
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    K, V = (torch.randn((B * blocks, block, H, D), device="cuda", generator=g).bfloat16() for _ in range(2))
    q = torch.randn((B, H * G, D), device="cuda", generator=g).bfloat16()
    table = torch.arange(B * blocks, dtype=torch.int32, device="cuda").view(B, blocks)
    pos, length = torch.arange(B + 1, dtype=torch.int32, device="cuda"), torch.full((B,), L, dtype=torch.int32, device="cuda")
    sel = torch.arange(blocks, dtype=torch.int32, device="cuda").expand(B, H, blocks).contiguous()
    out, lse = _comet().comet_block_attend(q, K, V, table, pos, length, sel)
    for b in range(B):
        k, v = (t[b * blocks:(b + 1) * blocks].flatten(0, 1)[:L].transpose(0, 1).double() for t in (K, V))          # H, L, D
        z = torch.matmul(q[b].view(H, G, D).double(), k.transpose(1, 2).contiguous()) * D ** -0.5
        w = torch.softmax(z, 2)
        want = torch.matmul(w, v.contiguous()).view(H * G, D)
        mass = torch.matmul(w, v.abs().contiguous()).view(H * G, D)
        # weights and the result are rounded to 8 bits; scores of 128 terms and sums of 2560 in 32 bits
        bound = (2.0 ** -8 + 2.0 ** -24 * 4096) * mass + 2.0 ** -8 * want.abs()
        assert bool(((out[b].double() - want).abs() <= bound).all())
        assert bool(((lse[b].double() - torch.logsumexp(z, 2).view(-1)).abs() <= 2.0 ** -24 * 4096).all())


def test_a_table_as_wide_as_it_may_be():
    """The list of chosen blocks takes the most room then, next to keys and values of the largest size."""
    for dtype, D in ((torch.float16, 256), (torch.float32, 256), (torch.bfloat16, 128)):
        s = make([1, 9], [300, 200], 1, 3, D, 16, dtype, seed=10, K=6)
        want = check(s)
        wide = torch.full((2, 262144), -1, dtype=torch.int32, device="cuda")
        wide[:, :s["table"].shape[1]] = s["table"]
        sel = torch.full((10, 1, 1000), -1, dtype=torch.int32, device="cuda")
        sel[:, :, 3:9] = s["sel"]
        got = _comet().comet_block_attend(s["q"], s["K"], s["V"], wide, s["pos"], s["length"], sel)
        unit = ref.UNIT[dtype]
        # the places are shared out in another way: weights rounded to the type, sums in another order
        assert bool(((got[0].double() - want[0].double()).abs() <= 8 * unit * (1 + want[0].double().abs())).all())


def test_in_inference_mode():
    comet = _comet()
    with torch.inference_mode():
        check(make([2, 9], [100, 200], 2, 2, 64, 16, torch.bfloat16, seed=11, K=4))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_captured_and_replayed_on_another_stream(D):
    comet = _comet()
    s = make([1] * 8 + [40], [200 + i for i in range(8)] + [600], 2, 2, D, 16, torch.bfloat16, seed=8, K=5)
    side = torch.cuda.Stream()
    call = lambda stream=None: comet.comet_block_attend(s["q"], s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"], stream=stream)
    want = call()
    side.wait_stream(torch.cuda.current_stream())
    other = call(side)
    torch.cuda.synchronize()
    assert torch.equal(want[0], other[0]) and torch.equal(want[1], other[1])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, call()))
    for step in range(3):
        s["q"].normal_()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        now = call()
        assert all(torch.equal(out, now[0]) and torch.equal(lse, now[1]) for _, (out, lse) in graphs)
        check(s)
