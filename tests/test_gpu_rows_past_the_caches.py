"""Calls on so many rows that they are read past the caches: the same bits as for a part of the rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V,dtype", [(2100, 65537, torch.bfloat16), (1100, 65536, torch.float32), (4200, 32768, torch.float16), (8400, 16391, torch.bfloat16),
                                       (33000, 4099, torch.float16), (1400, 100003, torch.bfloat16)])
def test_the_same_as_of_a_part(N, V, dtype):
    import paper_2102_05187_amd as comet
    assert N * V * torch.empty(0, dtype=dtype).element_size() >= 256 << 20
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    Z = (torch.randn((N, V), device="cuda", generator=g) * 3).to(dtype)
    crd, vals, lse = comet.comet_rows_topk(Z, 20)
    loss = comet.comet_distill_forward(Z, crd, vals + 0.5, tlse=lse + 0.75)[0]
    only = comet.comet_distill_forward(Z, crd, vals + 0.5)[0]
    part = 300                                                   # less than 256 MB, and of odd rows less than are shifted
    for r in (0, N // 2 + 1, N - part):
        rows = slice(r, r + part)
        some = comet.comet_rows_topk(Z[rows], 20)
        assert all(torch.equal(a, b[rows]) for a, b in zip(some, (crd, vals, lse)))
        args = Z[rows], crd[rows], (vals + 0.5)[rows]
        assert torch.equal(comet.comet_distill_forward(*args, tlse=(lse + 0.75)[rows])[0], loss[rows])
        assert torch.equal(comet.comet_distill_forward(*args)[0], only[rows])
