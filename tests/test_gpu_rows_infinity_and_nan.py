"""The log-sum-exp of a row with +inf, and of one with +inf and a NaN."""
import math

import pytest
import torch

from test_gpu_rows_topk import DTYPES, check

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [2, 9, 2000, 50021, 140001, 300007])
def test_both_in_a_row(V, dtype):
    Z = torch.randn((9, V), generator=torch.Generator().manual_seed(V))
    Z[0, 0], Z[0, V - 1] = INF, math.nan
    Z[1, 0], Z[1, V - 1] = math.nan, INF
    Z[2, V // 2 - 1], Z[2, V // 2] = INF, math.nan
    Z[3] = INF
    Z[4] = INF
    Z[4, V // 3] = math.nan
    Z[5, V - 1] = INF
    Z[6] = -INF
    Z[6, V // 2] = INF
    Z[7] = math.nan
    Z[7, V // 2] = INF
    Z[8, :2] = torch.tensor([INF, -INF])
    check(Z.to(dtype).cuda(), 3)
