"""The 64-bit definitions that the operators on dense rows are held against, held against torch and against differences (CPU)."""
import math

import numpy as np
import pytest
import torch

import rows_reference as ref


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V,count", [(1, 1), (7, 3), (40, 0), (40, 40), (101, 12)])
def test_distillation_gradient_is_the_derivative_of_its_loss(V, count, tail):
    rng = np.random.RandomState(V * 100 + count)
    z, scale, weight = rng.randn(V) * 2, 0.7, 1.3
    teacher = rng.randn(V) * 2
    crd = rng.permutation(V)[:count]
    tlse = ref.lse_row(teacher * scale) if tail else None
    t = teacher[crd]
    loss, g, _ = ref.distill_row(z, crd, t, tlse, scale, weight, 1.0)
    for j in range(V):
        h = 1e-5
        up, down = z.copy(), z.copy()
        up[j] += h
        down[j] -= h
        d = (ref.distill_row(up, crd, t, tlse, scale, weight)[0] - ref.distill_row(down, crd, t, tlse, scale, weight)[0]) / (2 * h)
        assert abs(d - g[j]) <= 1e-8          # h^2 / 6 of a third derivative of order 1, and 1e-16 / h of rounding


def test_distillation_with_all_places_kept_is_the_kl_divergence():
    rng = np.random.RandomState(0)
    z, t = rng.randn(50), rng.randn(50)
    want = torch.nn.functional.kl_div(torch.log_softmax(torch.tensor(z), 0), torch.log_softmax(torch.tensor(t), 0), log_target=True, reduction="sum")
    for tlse in (None, ref.lse_row(t)):
        assert abs(ref.distill_row(z, np.arange(50), t, tlse, 1.0, 1.0)[0] - float(want)) < 1e-12


def test_distillation_tail_is_one_more_outcome():
    """The same as the divergence of two distributions over the entries and everything else put together."""
    rng = np.random.RandomState(1)
    z, t, keep = rng.randn(30), rng.randn(30), np.arange(4, 12)
    p, q = np.exp(t - ref.lse_row(t)), np.exp(z - ref.lse_row(z))
    P, Q = np.append(p[keep], 1 - p[keep].sum()), np.append(q[keep], 1 - q[keep].sum())
    assert abs(ref.distill_row(z, keep, t[keep], ref.lse_row(t), 1.0, 1.0)[0] - (P * np.log(P / Q)).sum()) < 1e-12


def test_topk_order_and_missing_places():
    z = [1.0, 3.0, -math.inf, 3.0, math.nan, -0.0, 0.0]
    assert ref.topk_row(z, 4)[0] == [1, 3, 0, 5]
    assert ref.topk_row(z, 7) == ([1, 3, 0, 5, 6, -1, -1], [3.0, 3.0, 1.0, 0.0, 0.0, -math.inf, -math.inf])
    assert ref.topk_row(z, 3, True)[0] == [0, 1, 3]


def test_selection_is_torchs_where_nothing_ties():
    rng = np.random.RandomState(2)
    z, c = rng.randn(3, 40), rng.randn(3)
    s = torch.tensor(c)[:, None] + torch.log_softmax(torch.tensor(z), 1)
    v, at = s.flatten().topk(6)
    scores, parents, tokens, _ = ref.select_batch(z, c, 6)
    assert np.allclose(scores, v.numpy(), atol=1e-12)
    assert [p * 40 + t for p, t in zip(parents, tokens)] == at.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rounding_to_a_type_keeps_to_its_unit(dtype):
    x = torch.randn(20000, dtype=torch.float64, generator=torch.Generator().manual_seed(3)) + 3.0
    off = ((x.to(dtype).double() - x).abs() / x.abs()).max()
    assert 0.5 * ref.UNIT[dtype] < off <= ref.UNIT[dtype]
