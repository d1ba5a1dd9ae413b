"""Beams with a score of +inf: all their candidates tie, thousands of them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W,V,n", [(4, 50, 6), (64, 300, 128), (16, 9001, 500)])
def test_lower_beams_then_lower_tokens(W, V, n):
    import paper_2102_05187_amd as comet
    Z = torch.zeros((2, W, V), device="cuda")
    c = torch.full((2, W), math.inf, device="cuda")
    c[1, 0] = 0.0
    score, parent, token = comet.comet_beam_select(Z, c, n)
    torch.cuda.synchronize()
    per = min(n, V)                        # a beam offers its n best
    want = torch.arange(n)
    assert bool((score == math.inf).all())
    for b in range(2):
        assert torch.equal(parent[b].cpu(), (want // per + b).int())
        assert torch.equal(token[b].cpu(), (want % per).int())
