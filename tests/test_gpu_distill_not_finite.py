"""+inf and NaN in a row's tlse or weight: its loss and its gradient are NaN, and no other row's."""
import math

import numpy as np
import pytest
import torch

from test_gpu_distill import DTYPES, Problem

pytestmark = pytest.mark.gpu
INF = math.inf


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def check(p, bad):
    comet = _comet()
    loss, stat = comet.comet_distill_forward(p.Z, p.crd, p.tvals, **p.kw)
    g = comet.comet_distill_backward(p.Z, p.crd, p.tvals, stat, **p.kw)
    loss2, g2 = comet.comet_distill_step(p.Z, p.crd, p.tvals, **p.kw)
    torch.cuda.synchronize()
    for a, b in ((loss, g), (loss2, g2)):
        for r in bad:
            assert math.isnan(float(a[r])), r
            assert bool(torch.isnan(b[r]).all()), r
    p.N = min(bad)                                               # the rows before them
    p.compare(loss, g)
    p.compare(loss2, g2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [9, 3001, 40009, 140001])
def test_tlse(V, dtype):
    p = Problem(8, V, 6, dtype, seed=V, tail=True, weighted=False)
    p.rows[5] = (np.full(6, -1), p.rows[5][1])                   # no entry
    p.tlse[4] = p.tlse[5] = p.tlse[6] = np.float32(INF)
    p.rows[6] = (p.rows[6][0], np.full(6, -INF, dtype=np.float32))
    p.tlse[7] = np.float32(math.nan)
    p.args()
    check(p, (4, 5, 6, 7))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [9, 3001, 140001])
def test_weight(V, tail, dtype):
    p = Problem(8, V, 6, dtype, seed=V + 1, tail=tail, weighted=True)
    p.weight[:5] = 1.5, 0, 0.25, 1, 1
    p.weight[5], p.weight[6], p.weight[7] = INF, math.nan, -INF
    p.args()
    check(p, (5, 6, 7))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("value", [INF, math.nan])
@pytest.mark.parametrize("V", [9, 3001, 40009, 140001])
def test_a_logit_at_an_entry(V, value, tail, dtype):
    """... whatever the other places are."""
    p = Problem(8, V, 6, dtype, seed=V + 2, tail=tail, weighted=False)
    Z = torch.tensor(p.host)
    Z[4:7] = -INF                                                # nothing is left but that
    Z[5, torch.tensor(p.rows[5][0])] = 1.0                       # ... and the entries
    Z[6] = torch.finfo(dtype).min
    for r in range(4, 8):
        Z[r, int(p.rows[r][0][2])] = value
    p.set(Z.to(dtype))
    check(p, (4, 5, 6, 7))
