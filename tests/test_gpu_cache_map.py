"""Block tables and slots against the plain implementation: whole numbers, equal throughout."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def state(B, M, block, S=None, seed=0, most=None, held_more=True):
    g = torch.Generator().manual_seed(seed)
    most = M * block if most is None else most
    length = torch.randint(0, most + 1, (B,), generator=g)
    held = (length + block - 1) // block
    if held_more:
        held = torch.minimum(held + torch.randint(0, 2, (B,), generator=g), torch.tensor(M))
    total = int(held.sum())
    S = total + B * 2 if S is None else max(S, 0)
    ids = torch.randperm(total + S, generator=g).int()
    table = torch.full((B, M), -7, dtype=torch.int32)
    table[torch.arange(M) < held[:, None]] = ids[:total]
    spare = torch.full((total + S,), -9, dtype=torch.int32)
    spare[:S] = ids[total:]
    return dict(length=length.int(), held=held.int(), table=table, spare=spare, count=torch.tensor([S], dtype=torch.int32))


def check(s, add, block, N, ended=None, stride=0, stream=None):
    comet = _comet()
    want = ref.cache_map(add, ended, s["length"].tolist(), s["held"].tolist(), s["table"].tolist(), s["spare"].tolist(), int(s["count"]), block, N)
    d = {name: t.cuda() for name, t in s.items()}
    if stride:
        wide = torch.full((s["table"].shape[0], s["table"].shape[1] + stride), -3, dtype=torch.int32, device="cuda")
        wide[:, :s["table"].shape[1]] = d["table"]
        d["table"] = wide[:, :s["table"].shape[1]]
    flags = None if ended is None else torch.tensor(ended, dtype=torch.bool).cuda()
    pos, slot, place = comet.comet_cache_map(torch.tensor(add, dtype=torch.int32).cuda(), d["length"], d["held"], d["table"], d["spare"], d["count"], block, N,
                                             ended=flags, stream=stream)
    torch.cuda.synchronize()
    got = (pos, slot, place, d["length"], d["held"], d["table"], d["spare"], d["count"])
    for name, x, y in zip(("pos", "slot", "place", "length", "held", "table", "spare"), got, want):
        assert x.tolist() == y, name
    assert int(d["count"]) == want[7]
    if stride:
        assert bool((wide[:, s["table"].shape[1]:] == -3).all())
    return {name: d[name].cpu().contiguous() for name in s}


@pytest.mark.parametrize("block", [1, 16, 48, 64, 1024])
@pytest.mark.parametrize("B,M", [(1, 1), (1, 5), (7, 9), (64, 30), (1025, 4), (2500, 3)])
def test_sizes(B, M, block):
    s = state(B, M, block, seed=B + M + block)
    g = torch.Generator().manual_seed(B)
    add = torch.randint(-1, min(2 * block, 40) + 1, (B,), generator=g).tolist()
    check(s, add, block, sum(max(a, 0) for a in add) + 5, stride=B % 2 * 3)


@pytest.mark.parametrize("B,M,N", [(5, 8, 200), (300, 20, 20000), (1500, 70, 60000)])
@pytest.mark.parametrize("ends", [0.3, 1.0, 0.0])
def test_ended_requests_make_room(B, M, N, ends):
    s = state(B, M, 16, seed=3, S=2)
    g = torch.Generator().manual_seed(B)
    ended = (torch.rand(B, generator=g) < ends).tolist()
    add = [int(x) if e else 1 for x, e in zip(torch.randint(0, M * 16 + 20, (B,), generator=g), ended)]
    check(s, add, 16, N, ended=ended)


def test_sums_that_pass_32_bits():
    """All places of all requests are more than 2^31: running sums are held in 64 bits."""
    s = state(1500, 2000, 1024, seed=4, most=3000, S=5000)
    g = torch.Generator().manual_seed(7)
    add = torch.randint(0, 1500, (1500,), generator=g).tolist()
    add[700] = add[701] = 2000 * 1024 - 3000
    ended = (torch.rand(1500, generator=g) < 0.1).tolist()
    check(s, add, 1024, 100000, ended=ended)


@pytest.mark.parametrize("S", [0, 1, 7, 40])
def test_too_few_spare_blocks(S):
    s = state(40, 9, 16, seed=S, S=S, held_more=False, most=100)
    add = [(i * 7) % 35 for i in range(40)]
    check(s, add, 16, 4000)
    check(s, [1] * 40, 16, 4000)                 # those that need no block get their token all the same


@pytest.mark.parametrize("N", [0, 1, 33, 100])
def test_too_few_rows(N):
    s = state(12, 9, 16, seed=N)
    check(s, [0, 5, 30, 0, 12, 3, 0, 9, 60, 1, 1, 0], 16, N)


def test_nothing_to_add_and_no_requests():
    check(state(6, 3, 16), [0] * 6, 16, 0)
    check(state(6, 3, 16), [0] * 6, 16, 9, ended=[True] * 6)
    s = dict(length=torch.zeros(0, dtype=torch.int32), held=torch.zeros(0, dtype=torch.int32), table=torch.zeros((0, 4), dtype=torch.int32),
             spare=torch.arange(3, dtype=torch.int32), count=torch.tensor([3], dtype=torch.int32))
    comet, d = _comet(), {name: t.cuda() for name, t in s.items()}
    pos, slot, place = comet.comet_cache_map(torch.zeros(0, dtype=torch.int32, device="cuda"), d["length"], d["held"], d["table"], d["spare"], d["count"], 16, 4)
    assert pos.tolist() == [0] and slot.tolist() == place.tolist() == [-1] * 4 and int(d["count"]) == 3


def test_numbers_that_cannot_be():
    s = state(6, 4, 16, seed=1)
    s["held"][:4] = torch.tensor([-3, 90, 2, 1])
    s["length"][:4] = torch.tensor([5, -8, 900, 2 ** 31 - 1])
    for count in (-4, 10 ** 6):
        s["count"][0] = count
        check(s, [1, 2, 3, 2 ** 31 - 1, 0, 4], 16, 100, ended=[False, True, False, False, True, False])


def test_steps_in_turn():
    """Blocks are neither lost nor given twice over many steps."""
    g = torch.Generator().manual_seed(5)
    s = state(20, 12, 16, seed=5, most=60)
    everything = sorted(s["spare"][:int(s["count"])].tolist() + s["table"][torch.arange(12) < s["held"][:, None]].tolist())
    for step in range(12):
        ended = (torch.rand(20, generator=g) < 0.2).tolist()
        add = torch.randint(0, 30, (20,), generator=g).tolist()
        s = check(s, add, 16, 400, ended=ended if step % 3 else None)
        s["length"] = (s["length"] - torch.randint(0, 4, (20,), generator=g).int()).clamp(min=0)      # drafts that were not taken
        now = s["spare"][:int(s["count"])].tolist() + s["table"][torch.arange(12) < s["held"][:, None]].tolist()
        assert sorted(now) == everything


def test_captured_and_replayed():
    comet = _comet()
    s = {name: t.cuda() for name, t in state(300, 64, 16, seed=9, most=200, S=4000).items()}
    add = torch.ones(300, dtype=torch.int32, device="cuda")
    ended = torch.zeros(300, dtype=torch.bool, device="cuda")
    ended[::50] = True
    eager = {name: t.clone() for name, t in s.items()}
    call = lambda d: comet.comet_cache_map(add, d["length"], d["held"], d["table"], d["spare"], d["count"], 16, 9000, ended=ended)
    call({name: t.clone() for name, t in s.items()})
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(s)
    for step in range(4):
        add.fill_(1 + 7 * step)
        graph.replay()
        torch.cuda.synchronize()
        want = call(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(torch.equal(s[n], eager[n]) for n in s)
