"""As many rows as there may be, each of two pieces: the gradient's grid passes what one launch takes."""
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu


def test_the_last_rows_get_their_gradient():
    import paper_2102_05187_amd as comet
    N, V = 1 << 23, 8193                   # 137 GB: two pieces of 1024 vectors and less a row
    free, _ = torch.cuda.mem_get_info()
    if free < 150 << 30:
        pytest.skip("needs 150 GB of free device memory")
    torch.cuda.empty_cache()
    Z = torch.empty((N, V), dtype=torch.bfloat16, device="cuda")
    some = [0, 1, (1 << 22) - 1, 1 << 22, N - 2, N - 1]
    g = torch.Generator().manual_seed(1)
    rows = torch.randn((len(some), V), generator=g).bfloat16()
    for r, row in zip(some, rows):
        Z[r].copy_(row)
    Z[5, :] = 7.0                          # a row of weight 0
    Z[N - 3, V - 1] = 7.0
    weight = torch.zeros(N, device="cuda")
    weight[some] = 1.5
    crd = torch.full((N, 1), -1, dtype=torch.int32, device="cuda")
    crd[some, 0] = torch.tensor([0, 8192, 8191, 100, 8192, 5], dtype=torch.int32, device="cuda")
    tvals = torch.zeros((N, 1), device="cuda")
    loss, stat = comet.comet_distill_forward(Z, crd, tvals, weight=weight)
    comet.comet_distill_backward(Z, crd, tvals, stat, weight=weight, dZ=Z)
    torch.cuda.synchronize()
    assert bool((Z[5] == 0).all()) and float(Z[N - 3, V - 1]) == 0
    for i, r in enumerate(some):
        z = rows[i].double().numpy()
        want, grad, size = ref.distill_row(z, [int(crd[r, 0])], [0.0], None, 1.0, 1.5)
        bl, bg = ref.distill_bounds(z, want, grad, size, V, 1.0, 1.5, torch.bfloat16)
        assert abs(float(loss[r]) - want) <= bl
        assert (abs(Z[r].double().cpu().numpy() - grad) <= bg).all(), r
    del Z
    torch.cuda.empty_cache()
