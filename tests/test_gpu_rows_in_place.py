"""Tensors that a call overwrites are marked as changed, so that automatic differentiation notices."""
import pytest
import torch

from test_gpu_beam import parents, state
from test_gpu_distill import Problem

pytestmark = pytest.mark.gpu


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def test_versions():
    comet = _comet()
    p = Problem(4, 301, 5, torch.float32, weighted=False)

    def changed(call, *tensors):
        before = [t._version for t in tensors]
        call()
        assert all(t._version > b for t, b in zip(tensors, before))

    dev = dict(device="cuda")
    crd, vals, lse = torch.empty((4, 5), dtype=torch.int32, **dev), torch.empty((4, 5), **dev), torch.empty(4, **dev)
    loss, stat, dZ = torch.empty(4, **dev), torch.empty((4, 7), dtype=torch.float64, **dev), torch.empty((4, 301), **dev)
    changed(lambda: comet.comet_rows_topk(p.Z, 5, crd=crd, vals=vals, lse=lse), crd, vals, lse)
    changed(lambda: comet.comet_distill_forward(p.Z, p.crd, p.tvals, loss=loss, stat=stat, **p.kw), loss, stat)
    changed(lambda: comet.comet_distill_backward(p.Z, p.crd, p.tvals, stat, dZ=dZ, **p.kw), dZ)
    changed(lambda: comet.comet_distill_step(p.Z, p.crd, p.tvals, loss=loss, dZ=p.Z, **p.kw), loss, p.Z)
    states = [state((2, 3, 8), torch.float32, 0), state((2, 3, 5), torch.bfloat16, 1)]
    changed(lambda: comet.comet_beam_reorder(states, parents(2, 3, 0)), *states)
    unread = p.Z._version
    comet.comet_distill_forward(p.Z, p.crd, p.tvals, **p.kw)
    assert p.Z._version == unread


def test_a_saved_tensor_that_was_overwritten_is_refused():
    comet = _comet()
    p = Problem(4, 301, 5, torch.float32, weighted=False)
    a = torch.ones(4, 1, device="cuda", requires_grad=True)
    y = (a * p.Z).sum()                                          # keeps Z for its gradient
    comet.comet_distill_step(p.Z, p.crd, p.tvals, dZ=p.Z, **p.kw)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    x = state((2, 3, 8), torch.float32, 2)
    b = torch.ones(2, 3, 1, device="cuda", requires_grad=True)
    y = (b * x).sum()
    comet.comet_beam_reorder([x[:, :, :5]], parents(2, 3, 1))    # a part of it
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()


def test_tensors_of_inference_mode():
    """They have no version to raise."""
    comet = _comet()
    with torch.inference_mode():
        x = state((2, 3, 8), torch.float32, 3)
        par = parents(2, 3, 2)
        want = x[torch.arange(2, device="cuda")[:, None], par.long()]
        comet.comet_beam_reorder([x], par)
        crd, vals, lse = comet.comet_rows_topk(x.view(6, 8), 3)
        comet.comet_rows_topk(x.view(6, 8), 3, crd=crd, vals=vals, lse=lse)
    comet.comet_beam_reorder([x], torch.arange(3, dtype=torch.int32, device="cuda").repeat(2, 1))
    torch.cuda.synchronize()
    assert torch.equal(x, want)
