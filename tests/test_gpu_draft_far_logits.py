"""Verified drafts where a row's logits lie far from 0: the answers are those of the plain implementation in 64 bits."""
import pytest
import torch

from test_gpu_draft_verify import DTYPES, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [301, 50021])
@pytest.mark.parametrize("far", [-3e38, -1e13, 1e13, 3e38])
@pytest.mark.parametrize("which", ["draft", "Z"])
def test_one_of_the_two_rows_lies_far_away(which, far, V):
    """All of a row's logits are `far`: its distribution is flat.  The other row's are ordinary."""
    s = make([2] * 24, V, torch.float32, -1, seed=20)
    s[which][:] = far
    s["u"][:] = 0.999                                              # some of the drafted tokens are not taken
    accepted, follow, _ = check(s, 0.7)
    assert bool((follow >= 0).all()) and int(accepted.sum()) < 24


@pytest.mark.parametrize("V", [301, 50021])
@pytest.mark.parametrize("far", [-1e9, -1e8, -2e7, 2e7, 1e8, 1e9])
@pytest.mark.parametrize("which", ["draft", "Z", "both"])
def test_rows_that_lie_away(which, far, V):
    s = make([2] * 24, V, torch.float32, -1, seed=23)
    for name in ("draft", "Z") if which == "both" else (which,):
        s[name][:] = far
    s["u"][:] = 0.999
    accepted, follow, _ = check(s, 0.7)
    assert bool((follow >= 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kept", [-1, 0, 5])
@pytest.mark.parametrize("top", [10.0, 40.0, 300.0])
@pytest.mark.parametrize("V", [301, 50021])
def test_temperatures_near_zero(V, top, kept, dtype):
    """The largest logit has all of p and, at the draft's rows, all of q."""
    B = 12
    g = torch.Generator().manual_seed(24)
    for scale in (1e6, 5e7, 1e8, 1e9, 1e10, 1e12, 1e30):
        s = make([3] * B, V, dtype, 0, seed=24)
        N = 3 * B
        best = torch.randint(V, (N,), generator=g).cuda()
        s["Z"] = (s["Z"].float() + top).to(dtype)
        s["Z"][torch.arange(N), best] = 1.25 * top + 10                # 2 and more above all others
        if kept < 0:
            s["draft"] = s["Z"].clone()
        if kept > 0:
            high = s["Z"].float().topk(kept, dim=1)
            s["crd"], s["vals"] = high.indices.int().contiguous(), high.values.contiguous()
        s["token"][1:] = best[:-1].int()
        s["token"][1:6:3] = (s["token"][1:6:3] + 1) % V                # a request's first drafted token
        s["token"][8:15:3] = (s["token"][8:15:3] + 7) % V              # its second one
        s["u"][:], s["v"][:] = 0.5, torch.rand(B, generator=g).cuda()
        for given in (scale, torch.full((B,), scale, device="cuda")):
            accepted, follow, _ = check(s, given)
            took = torch.tensor([0, 0, 1, 1, 1] + [2] * (B - 5), device="cuda")
            assert torch.equal(accepted, took.int()), scale
            assert torch.equal(follow.long(), best[torch.arange(0, N, 3, device="cuda") + took]), scale


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [301, 50021])
@pytest.mark.parametrize("kept", [-1, 0, 7])
def test_masks_of_whole_rows_and_pieces(kept, V, dtype):
    """Masks of -1e9 beside -2e9 or -inf, of all of a row or of long stretches of it, at ordinary temperatures."""
    seen = 0
    for scale in (20.0, 5.0, 2.0, 1.4, 1.25, 1.0, 0.9, 0.8, 0.7, 0.6, 0.5):
        s = make([2] * 20, V, dtype, kept, seed=25)
        for name in ("Z",) + (("draft",) if kept < 0 else ()):
            x = s[name]
            x[0:8] = -1e9
            x[0:4, ::2], x[4:8, 1::3] = -2e9, -float("inf")
            x[8:16, :V // 2] = -1e9
            x[8:12, :V // 4], x[12:16, V // 8:V // 3] = -2e9, -float("inf")
            x[16:24, V // 2:] = -1e9
            x[24:32, V // 3:V // 2] = 1e9
        s["u"][:] = 0.999
        s["token"][1:16:2] = V - 1 - (V - 1) % 3                       # not masked where every third place from 1 on is
        _, follow, want = check(s, scale)
        assert bool((follow >= 0).all()), scale
        seen += sum(margin > 1e-11 for _, _, margin in want)
    assert seen > 100
