"""Rows of 16-bit elements that start at odd multiples of 2 bytes, and rows around the longest that a workgroup holds."""
import numpy as np
import pytest
import torch

from test_gpu_distill import Problem
from test_gpu_rows_topk import check, matrix

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


def _comet():
    import paper_2102_05187_amd as comet
    return comet


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("V,ld", [(16383, 16383), (16384, 16385), (16384, 16387), (16385, 16385), (16390, 16391), (16391, 16391), (16392, 16399), (16393, 16395),
                                  (18432, 18433), (18440, 18441), (32768, 32769), (65535, 65535), (65536, 65539), (131071, 131071), (131072, 131073),
                                  (131081, 131081)])
def test_top_of_odd_rows(V, ld, start, dtype):
    check(matrix(4, V, dtype, seed=V + start, ld=ld, start=start), 33)


@pytest.mark.parametrize("dtype", HALVES)
def test_the_largest_are_at_the_ends_of_wavefronts(dtype):
    """Each element that a lane gets from somewhere else is one of those kept: last ones of vectors, of wavefronts, of the row."""
    V, ld = 16405, 16407
    Z = matrix(4, V, dtype, seed=3, ld=ld)
    places = torch.tensor([7, 8, 15, 504, 511, 512, 519, 2047, 2048, 2055, 16383, 16384, 16391, 16399, 16400, 16404], device="cuda")
    Z[:, places] = (torch.arange(places.numel(), device="cuda") + 30.0).to(dtype)
    check(Z, places.numel())
    crd, _, _ = _comet().comet_rows_topk(Z, places.numel(), by_coordinate=True)
    assert (crd.cpu() == places.cpu()).all()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("V,ld", [(16384, 16385), (16391, 16391), (16400, 16401), (20480, 20481), (33001, 33003), (65537, 65537), (70001, 70001), (131071, 131071)])
def test_gradient_of_odd_rows(V, ld, start, tail, dtype):
    Problem(5, V, 40, dtype, seed=V + start, tail=tail, ld=ld, start=start).check()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("tail", [False, True])
def test_entries_at_the_ends_of_wavefronts(tail, dtype):
    p = Problem(4, 16405, 16, dtype, seed=8, tail=tail, ld=16407)
    places = np.array([7, 8, 15, 504, 511, 512, 519, 2047, 2048, 2055, 16383, 16384, 16391, 16399, 16400, 16404])
    p.rows = [(places if r % 2 else places[::-1].copy(), t) for r, (_, t) in enumerate(p.rows)]
    p.set(torch.tensor(p.host).to(dtype))
    p.check()


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,dtype", [(64, 81921, torch.bfloat16), (64, 81920, torch.float16), (64, 131073, torch.bfloat16), (64, 163840, torch.float16),
                                       (64, 163841, torch.bfloat16), (64, 40961, torch.float32), (64, 40960, torch.float32), (64, 65537, torch.float32),
                                       (64, 81920, torch.float32), (64, 81921, torch.float32), (63, 81921, torch.bfloat16)])
def test_the_longest_rows_that_are_held(N, V, dtype, tail):
    Problem(N, V, 12, dtype, seed=V, tail=tail).check()


@pytest.mark.parametrize("dtype", HALVES)
def test_alike_at_every_address(dtype):
    """A row's results do not depend on where it starts."""
    comet = _comet()
    V, K = 40003, 24
    one = matrix(1, V, dtype, seed=9)
    Z = torch.empty(6 * (V + 8), dtype=dtype, device="cuda")
    rows = Z[:6 * V].view(6, V)
    rows.copy_(one.expand(6, V))
    crd, vals, lse = comet.comet_rows_topk(rows, K)
    loss, stat = comet.comet_distill_forward(rows, crd, vals, tlse=lse + 0.1)
    g = comet.comet_distill_backward(rows, crd, vals, stat, tlse=lse + 0.1)
    loss2, g2 = comet.comet_distill_step(rows, crd, vals, tlse=lse + 0.1)
    for x in (crd, vals, lse, loss, stat, g, loss2, g2):
        bits = x.view(torch.int16) if x.dtype in HALVES else x
        assert (bits == bits[:1]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pieces", [3, 5, 15, 17])
def test_rows_of_many_pieces(pieces, dtype):
    per = 32768 if dtype == torch.float32 else 65536
    check(matrix(1, pieces * per, dtype, seed=pieces), min(1024, 2 ** 29 // (pieces * per)))
    check(matrix(2, (pieces - 1) * per + 1, dtype, seed=pieces), 1)
