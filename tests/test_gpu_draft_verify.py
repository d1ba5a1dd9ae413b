"""Verified drafts against the plain implementation in 64 bits: equal, wherever a decision is not within 1e-11 of another one."""
import math

import pytest
import torch

import cache_reference as ref
from cache_util import host

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# probabilities and running sums in 64 bits: each term to about 2^-49 of its size, sums of 2^18 terms to 2^-35 at worst and 2^-44 as a rule
NEAR = 1e-11


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def make(counts, V, dtype, kept, seed=0, spread=2.0, near=0.5, draft_dtype=None):
    """kept: -1 the draft's logits, 0 nothing of it, else that many entries."""
    g = torch.Generator().manual_seed(seed)
    N, B = sum(counts), len(counts)
    Z = (torch.randn((N, V), generator=g) * spread).to(dtype)
    x = Z.float() + near * torch.randn((N, V), generator=g)
    s = dict(Z=Z, pos=torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32), u=torch.rand(N, generator=g), v=torch.rand(B, generator=g))
    if kept < 0:
        s["draft"] = x = x.to(draft_dtype or dtype)
    if kept > 0:
        k = min(kept, V)
        top = x.topk(k, dim=1)
        order = torch.randperm(k, generator=g)
        s["crd"], s["vals"] = top.indices[:, order].int().contiguous(), top.values[:, order].float().contiguous()
        x = torch.full_like(x, -math.inf).scatter_(1, top.indices, top.values)
    token = torch.zeros(N, dtype=torch.int32)
    if N > 1:
        token[1:] = torch.multinomial(torch.softmax(x.float(), 1), 1, generator=g)[:-1, 0].int()
    s["token"] = token
    return {n: t.cuda() for n, t in s.items()}


def check(s, scale=1.0, stream=None, length=None):
    comet = _comet()
    extra = {n: s[n] for n in ("draft", "crd", "vals") if n in s}
    accepted, follow = comet.comet_draft_verify(s["Z"], s["token"], s["pos"], s["u"], s["v"], scale=scale, stream=stream, length=length, **extra)
    torch.cuda.synchronize()
    B = s["pos"].numel() - 1
    scales = host(scale) if isinstance(scale, torch.Tensor) else [scale] * B
    given = {n: host(t) if t.is_floating_point() else t.cpu().numpy() for n, t in extra.items()}
    want = ref.draft_verify(host(s["Z"]), s["token"].tolist(), s["pos"].tolist(), host(s["u"]), host(s["v"]), scales, **given)
    for b, (a, t, margin) in enumerate(want):
        if margin > NEAR:
            assert (int(accepted[b]), int(follow[b])) == (a, t), (b, margin)
    return accepted, follow, want


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kept", [-1, 0, 1, 20])
@pytest.mark.parametrize("counts,V", [([1], 1), ([3], 2), ([4, 1, 2], 7), ([2, 0, 5, 3], 1001), ([8, 8], 5003), ([3, 2], 32000), ([2, 4], 70001)])
def test_sizes(counts, V, kept, dtype):
    check(make(counts, V, dtype, kept, seed=V + kept), scale=1.25)


@pytest.mark.parametrize("kept", [-1, 0, 30])
def test_many_requests(kept):
    g = torch.Generator().manual_seed(kept)
    counts = torch.randint(0, 7, (300,), generator=g).tolist()
    accepted, _, want = check(make(counts, 503, torch.bfloat16, kept, seed=3, near=0.3))
    assert sum(m > NEAR for _, _, m in want) > 290
    assert kept == 0 or int(accepted.max()) >= 3


@pytest.mark.parametrize("a", DTYPES)
@pytest.mark.parametrize("b", DTYPES)
def test_draft_of_another_type(a, b):
    check(make([4, 3, 1, 2], 20011, a, -1, draft_dtype=b, seed=5))


@pytest.mark.parametrize("kept", [-1, 0, 9])
def test_a_scale_for_each_request(kept):
    s = make([4] * 12, 3001, torch.float32, kept, seed=6)
    scale = torch.tensor([0.2, 1.0, 3.0, 50.0, math.inf, 1e-6, math.nan, 0.0, -1.0, math.inf, 1e4, 0.7]).cuda()
    accepted, follow, _ = check(s, scale)
    assert accepted[6:9].tolist() == [0, 0, 0] and follow[6:9].tolist() == [-1, -1, -1]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [3, 1000, 40001])
def test_the_largest(V, dtype):
    s = make([5, 4, 1], V, dtype, -1, seed=7)
    best = s["Z"].float().argmax(1).int()
    s["token"][1:] = best[:-1]
    s["token"][3] = (best[2] + 1) % V
    accepted, follow, _ = check(s, math.inf)
    assert accepted.tolist() == [2, 3, 0] and follow.tolist() == [int(best[2]), int(best[8]), int(best[9])]
    s["Z"][:] = 1.5                                                # all equal: any drafted token is taken, the lowest follows
    accepted, follow, _ = check(s, math.inf)
    assert accepted.tolist() == [4, 3, 0] and follow.tolist() == [0, 0, 0]


@pytest.mark.parametrize("kept", [-1, 0, 12])
def test_the_same_distribution_takes_all(kept):
    s = make([6, 3], 12, torch.float32, kept, near=0.0, seed=8)
    if kept == 0:
        s["Z"][:] = -math.inf
        for r in range(9):
            s["Z"][r, int(s["token"][(r + 1) % 9])] = 3.0
    accepted, _, _ = check(s)
    assert accepted.tolist() == [5, 2]


@pytest.mark.parametrize("kept", [-1, 0, 5])
def test_rows_without_probabilities(kept):
    s = make([3, 3, 3, 3, 3, 1], 2003, torch.float32, kept, seed=9)
    s["u"][:] = 0                                                  # whatever has a probability is taken
    s["Z"][1] = -math.inf
    s["Z"][4, 77] = math.nan
    s["Z"][7, 3] = math.inf
    s["Z"][11, 2000] = math.nan                                    # a last row
    s["Z"][15] = -math.inf
    s["token"][13] = 2003                                          # not a token
    accepted, follow, _ = check(s)
    assert accepted.tolist() == [1, 1, 1, 2, 0, 0]
    assert follow[:4].tolist() == [-1] * 4 and follow[5] == -1 and 0 <= int(follow[4]) < 2003
    if kept:
        name = "draft" if kept < 0 else "vals"
        s[name][12, 0] = math.nan
        s["token"][13] = 5
        s["u"][12] = 0.999
        assert int(check(s)[0][4]) >= 1                            # nothing is known of the draft: taken


def test_masked_places():
    for low in (-math.inf, -3e38, -65504.0):
        s = make([4, 2, 3], 1501, torch.float32, -1, seed=10)
        s["Z"][:, ::2] = low
        s["draft"][:, 1::3] = low
        _, follow, _ = check(s)
        assert bool((follow % 2 == 1).all())


def test_entries_that_are_none():
    s = make([4, 2, 3], 1501, torch.bfloat16, 8, seed=11)
    s["crd"][:, 3], s["crd"][:, 5] = -1, 1501
    s["vals"][:, 2] = -math.inf
    check(s)
    s["crd"][:] = -1                                               # q is 0: every drafted token is taken
    assert check(s)[0].tolist() == [3, 1, 2]


@pytest.mark.parametrize("V", [5, 999, 50021])
@pytest.mark.parametrize("v", [0.0, 1.0 - 2.0 ** -24, 1.0, -1.0, 0.5])
def test_ends_of_the_random_numbers(V, v):
    s = make([1, 3], V, torch.float16, 0, seed=12)
    s["v"][:] = v
    s["u"][:] = 1.0 - 2.0 ** -24
    if 0 <= v < 1:
        check(s)
    else:
        _, follow = _comet().comet_draft_verify(s["Z"], s["token"], s["pos"], s["u"], s["v"])
        assert bool(((follow >= 0) & (follow < V)).all())


def test_nothing_left_of_p():
    """p <= q throughout, as where both are one and rounding makes u q >= p: then p itself is drawn from."""
    s = make([2], 301, torch.float32, -1, near=0.0, seed=13)
    s["u"][:] = 1.5                                                # not taken, and nothing is left
    accepted, follow, _ = check(s)
    assert int(accepted[0]) == 0 and int(follow[0]) >= 0


def test_lengths_follow():
    s = make([4, 1, 0, 6], 703, torch.bfloat16, -1, seed=14)
    length = torch.tensor([40, 30, 20, 10], dtype=torch.int32, device="cuda")
    accepted, _, _ = check(s, length=length)
    assert length.tolist() == [40 - (3 - int(accepted[0])), 30, 20, 10 - (5 - int(accepted[3]))]


def test_rows_that_lie_apart():
    s = make([4, 3], 1501, torch.bfloat16, -1, seed=15)
    want = check(s)
    Z = torch.zeros((7, 1601), dtype=torch.bfloat16, device="cuda")[:, 3:1504].copy_(s["Z"])
    draft = torch.zeros((7, 1555), dtype=torch.bfloat16, device="cuda")[:, 1:1502].copy_(s["draft"])
    got = check({**s, "Z": Z, "draft": draft})
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_tokens_are_distributed_as_the_target():
    """200000 requests of one drafted token: what comes first, draft or not, has the target's distribution."""
    B, V = 200000, 6
    g = torch.Generator().manual_seed(16)
    z, x = torch.randn(V, generator=g), torch.randn(V, generator=g)
    drawn = torch.multinomial(torch.softmax(x, 0), B, replacement=True, generator=g).int()
    token = torch.stack([torch.zeros(B, dtype=torch.int32), drawn], 1).flatten().cuda()
    accepted, follow = _comet().comet_draft_verify(z.expand(2 * B, V).contiguous().cuda(), token, torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda"),
                                                   torch.rand(2 * B, generator=g).cuda(), torch.rand(B, generator=g).cuda(),
                                                   draft=x.expand(2 * B, V).contiguous().cuda())
    first = torch.where(accepted == 1, drawn.cuda(), follow)
    share = torch.bincount(first, minlength=V).double().cpu() / B
    p = torch.softmax(z.double(), 0)
    assert bool(((share - p).abs() < 6 * (p * (1 - p) / B).sqrt()).all())            # six standard deviations
    q = torch.softmax(x.double(), 0)
    taken = float(torch.minimum(p, q).sum())
    assert abs(float(accepted.double().mean()) - taken) < 6 * (taken * (1 - taken) / B) ** 0.5


def test_captured_and_replayed_on_another_stream():
    comet = _comet()
    s = make([5, 1, 3], 60013, torch.bfloat16, -1, seed=17)
    call = lambda stream=None: comet.comet_draft_verify(s["Z"], s["token"], s["pos"], s["u"], s["v"], draft=s["draft"], stream=stream)
    side = torch.cuda.Stream()
    want = call()
    side.wait_stream(torch.cuda.current_stream())
    other = call(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for step in range(4):
        s["u"].uniform_(), s["v"].uniform_(), s["Z"].normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, call()))
        check(s)
