"""Rows whose largest elements lie within subnormal distances of each other: none may get lost."""
import pytest
import torch

from test_gpu_beam import check_select
from test_gpu_rows_topk import check

pytestmark = pytest.mark.gpu
WIDE = [torch.float32, torch.bfloat16]


def rows(V, seed):
    g = torch.Generator().manual_seed(seed)
    Z = torch.zeros((9, V))
    Z[0, V // 2] = 1e-37
    Z[1, V // 3] = 1e-40                                         # a subnormal number
    Z[2] = torch.rand(V, generator=g) * 1e-37 + 1e-37
    Z[3] = torch.randn(V, generator=g) * 1e-37
    Z[4] = torch.randn(V, generator=g) * 1e-39
    Z[5, ::3] = -1e-38
    Z[6] = torch.randn(V, generator=g) * 1e-31
    Z[7] = torch.randn(V, generator=g) * 1e-29
    Z[8, :V // 2] = torch.randn(V // 2, generator=g) * 1e-36
    Z[8, V // 2:] = -torch.inf
    return Z


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("K", [1, 8, 100, 700])
@pytest.mark.parametrize("V", [30, 300, 5003, 40009, 140001])
def test_top(V, K, dtype):
    check(rows(V, V + K).to(dtype).cuda(), K)


@pytest.mark.parametrize("dtype", WIDE)
@pytest.mark.parametrize("V,n", [(300, 20), (5003, 8), (60013, 40)])
def test_selection(V, n, dtype):
    Z = rows(V, V + n)[:8].view(2, 4, V).to(dtype).cuda()
    check_select(Z, torch.zeros((2, 4), device="cuda"), n)
    check_select(Z, torch.tensor([[0.0, 1e-38, 0.0, 1e-40]] * 2).cuda(), n)
