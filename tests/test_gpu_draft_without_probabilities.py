"""Drafted tokens that are not taken, judged against a row of the draft that has no probabilities: what follows is drawn from p."""
import math

import pytest
import torch

from test_gpu_draft_verify import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kept", [-1, 5])
@pytest.mark.parametrize("bad", [math.inf, math.nan, -math.inf])
@pytest.mark.parametrize("V", [7, 40001])
def test_nothing_is_taken_off(V, bad, kept, dtype):
    B = 40
    s = make([2] * B, V, dtype, kept, seed=21)
    first = torch.arange(0, 2 * B, 2)
    d = s["token"][first + 1].long()
    s["Z"][first, d] = -math.inf                                   # p = 0 at the drafted token: it is not taken
    best = s["Z"][first].argmax(1)
    name = "draft" if kept < 0 else "vals"
    if bad == -math.inf:
        s[name][first] = bad                                       # a row of nothing else
    elif kept < 0:
        s[name][first, best] = bad                                 # at the token that is drawn most often
    else:
        s["crd"][first, 0], s[name][first, 0] = best.int(), bad
    if kept > 0:
        s["crd"][first, 1:] = torch.where(s["crd"][first, 1:] == best[:, None], -1, s["crd"][first, 1:])
    accepted, follow, _ = check(s)
    assert int(accepted.sum()) == 0
    if bad != -math.inf and V == 7:
        assert int((follow == best).sum()) > 0


def test_finite_logits_of_a_row_with_a_nan():
    """Logits around 710 over the scale are powers that 64 bits do not hold, where the row has no maximum to take off."""
    s = make([2] * 30, 501, torch.float32, -1, seed=22)
    first = torch.arange(0, 60, 2)
    s["Z"][first, s["token"][first + 1].long()] = -math.inf
    s["draft"][first] = torch.linspace(600, 900, 501, device="cuda")
    s["draft"][first, 3] = math.nan
    check(s)
