"""Logits of large magnitude: places masked by a finite value, rows masked throughout, logits far above all others."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam import check_select
from test_gpu_distill import Problem
from test_gpu_rows_topk import check

pytestmark = pytest.mark.gpu
WIDE = [torch.float32, torch.bfloat16]
MASKS = [-1e8, -1e9, -1.6e9, -2e9, -1e10, -1e12, -1e20, -1e25, -1e29, -1e30]


def masked(V, mask, seed):
    """Rows of which some places hold `mask`: 11 kinds."""
    g = torch.Generator().manual_seed(seed)
    Z = torch.randn((11, V), generator=g) * 3
    Z[0, :V // 2] = mask                                         # the first half
    Z[1, V // 2:] = mask                                         # the last half
    at = V // 3 // 8 * 8
    Z[2, at:at + 8] = mask                                       # one vector of a thread
    Z[3, ::2] = mask                                             # every other place
    Z[4, :V - 1] = mask                                          # all but the last
    Z[5, 1:] = mask                                              # all but the first
    Z[6] = mask                                                  # the whole row
    Z[7] = mask * (1 + torch.rand(V, generator=g) * 2.0 ** -20)  # the whole row, not by one value
    Z[8, V // 2] = -mask                                         # one far above
    Z[9] = -mask                                                 # the whole row far above
    Z[10, torch.rand(V, generator=g) < 0.9] = mask               # nine tenths
    Z[10, 0] = 0.5
    return Z


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("V", [17, 2003, 40009, 140001])
def test_top(V, mask, dtype):
    check(masked(V, mask, V).to(dtype).cuda(), 12)


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("V", [17, 2003, 40009])
def test_distillation(V, mask, tail, dtype):
    p = Problem(13, V, 5, dtype, seed=V, tail=tail, weighted=False, scale=1.0)
    Z = torch.cat([masked(V, mask, V + 1), torch.tensor(p.host[11:]).float()])
    Z[11] = torch.where(torch.isin(torch.arange(V), torch.tensor(p.rows[11][0])), Z[11], mask)    # all outside of the entries
    Z[12, torch.tensor(p.rows[12][0])] = mask                                                     # the entries
    p.set(Z.to(dtype))
    p.check()


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("mask", [-1e10, -1e20])
def test_distillation_of_long_rows(mask, dtype):
    p = Problem(3, 140001, 9, dtype, seed=5, tail=True, weighted=False, scale=1.0)
    Z = torch.tensor(p.host)
    Z[0, :100000] = mask
    Z[1] = mask
    Z[2, 70000:] = mask
    p.set(Z.to(dtype))
    p.check()


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("V,n", [(40, 9), (2003, 6), (40009, 8)])
def test_selection(V, n, mask, dtype):
    Z = masked(V, mask, V + n)[[0, 2, 4, 6, 5, 8, 9, 10, 1, 3, 7, 6]].view(3, 4, V).to(dtype).cuda()
    c = -torch.rand((3, 4), generator=torch.Generator().manual_seed(V)).cuda()
    check_select(Z, c, n)


@pytest.mark.parametrize("dtype", WIDE)
def test_selection_among_fewer_tokens_than_wanted(dtype):
    Z = torch.full((2, 3, 32003), -1e10)
    Z[0, :, 5:8] = torch.tensor([1.0, 2.0, 0.5])
    Z[1, :, 9] = 3.0
    check_select(Z.to(dtype).cuda(), torch.tensor([[0.0, -0.5, -1.25], [0.0, -2.0, -math.inf]]).cuda(), 12)


@pytest.mark.parametrize("scale", [1e5, 1e6, 1e15])
def test_a_scale_that_makes_them_large(scale):
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        Z = masked(3001, -60000.0, 7).to(dtype)
        check(Z.cuda(), 6, scale=scale)
        p = Problem(11, 3001, 4, dtype, seed=3, tail=True, weighted=False, scale=scale)
        p.weight = np.full(11, 1 / scale, dtype=np.float32)      # the gradient stays in the type's range
        for r in range(11):                                      # teacher's logits of an ordinary size under that scale
            p.rows[r] = (p.rows[r][0], (p.rows[r][1] / scale).astype(np.float32))
            p.tlse[r] = 12.0
        p.set(Z)
        p.check()
