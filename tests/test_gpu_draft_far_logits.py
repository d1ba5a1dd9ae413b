"""Verified drafts where a row's logits lie far from 0: the answers are those of the plain implementation in 64 bits."""
import pytest
import torch

from test_gpu_draft_verify import check, make

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
