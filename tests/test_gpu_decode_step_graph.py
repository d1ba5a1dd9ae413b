"""A decoding step without prompts as one HIP graph: tables, writes, choice, attention and verification, replayed, against the same calls one by one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
H, G, D, BLOCK, M, V, DRAFTS = 2, 4, 64, 16, 40, 1003, 2


def _state(B, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    P = B * M // 2
    blank = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    return dict(length=blank(B), held=blank(B), table=blank(B, M), spare=torch.randperm(P, device="cuda", generator=g).int(), count=blank(1) + P,
                K=torch.zeros((P, BLOCK, H, D), dtype=dtype, device="cuda"), V=torch.zeros((P, BLOCK, H, D), dtype=dtype, device="cuda"),
                mean=torch.zeros((P, H, D), dtype=dtype, device="cuda"))


def _inputs(B, dtype, g):
    N = B * (1 + DRAFTS)
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=g)
    x = dict(k=rand(N, H, D).to(dtype), v=rand(N, H, D).to(dtype), q=rand(N, H * G, D).to(dtype), Z=2 * rand(N, V), draft=2 * rand(N, V),
             token=torch.randint(V, (N,), device="cuda", generator=g).int(), u=torch.rand(N, device="cuda", generator=g) * 0.3, v_=torch.rand(B, device="cuda", generator=g),
             add=torch.randint(0, 2 + DRAFTS, (B,), device="cuda", generator=g).int(), ended=torch.rand(B, device="cuda", generator=g) < 0.1)
    x["draft"] = x["Z"] + 0.3 * x["draft"]
    x["token"][1:] = x["draft"].argmax(1)[:-1].int()
    return x


def _step(s, x):
    import paper_2102_05187_amd as comet
    N = x["q"].shape[0]
    pos, slot, place = comet.comet_cache_map(x["add"], s["length"], s["held"], s["table"], s["spare"], s["count"], BLOCK, N, ended=x["ended"])
    comet.comet_cache_write(x["k"], x["v"], s["K"], s["V"], slot, s["mean"])
    # what is behind the last token is left as it was: fills instead of memory that nobody has written
    sel = comet.comet_block_select(x["q"], s["mean"], s["table"], pos, s["length"], BLOCK, 5, sel=torch.full((N, H, 5), -9, dtype=torch.int32, device="cuda"))
    out, lse = comet.comet_block_attend(x["q"], s["K"], s["V"], s["table"], pos, s["length"], sel, out=torch.full_like(x["q"], 7), lse=torch.full((N, H * G), 7.0, device="cuda"))
    accepted, follow = comet.comet_draft_verify(x["Z"], x["token"], pos, x["u"], x["v_"], draft=x["draft"], scale=1.25, length=s["length"])
    return [pos, slot, place, sel, out, lse, accepted, follow]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B", [1, 5, 70])
def test_a_step_is_one_graph(B, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    inputs = [_inputs(B, dtype, g) for _ in range(12)]
    mine, eager = _state(B, dtype, 1), _state(B, dtype, 1)
    given = {n: t.clone() for n, t in inputs[0].items()}
    _step(_state(B, dtype, 1), given)                              # what the library loads at its first call is loaded
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(mine, given)
    taken = 0
    for x in inputs:
        for n, t in x.items():
            given[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        want = _step(eager, x)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for n in mine:
            assert torch.equal(mine[n], eager[n]), n
        taken += int(want[6].sum())
    assert B == 1 or taken > 0
