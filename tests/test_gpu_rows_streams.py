"""Results and scratch of a call on another stream: memory that the current stream still uses is not theirs."""
import pytest
import torch

from test_gpu_rows_topk import matrix

pytestmark = pytest.mark.gpu
CYCLES = 20_000_000                        # a wait on the device of 10 to 200 ms


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def test_results_do_not_take_memory_that_is_still_read():
    """A freed tensor's memory goes back to its stream at once, while work on that stream may still be about to read it."""
    comet = _comet()
    Z = matrix(4096, 1500, torch.float32, seed=1)
    side = torch.cuda.Stream()
    comet.comet_rows_topk(Z, 1024)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    x = torch.full((4096, 1024), 3.0, device="cuda")
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    torch.cuda._sleep(CYCLES)
    y.copy_(x)
    del x
    out = comet.comet_rows_topk(Z, 1024, stream=side)
    torch.cuda.synchronize()
    assert bool((y == 3).all())
    assert all(torch.equal(a, b) for a, b in zip(out, comet.comet_rows_topk(Z, 1024)))


def test_scratch_does_not_take_memory_that_is_still_read():
    comet = _comet()
    from paper_2102_05187_amd import binding
    Z = matrix(300, 140001, torch.bfloat16, seed=2)
    want = comet.comet_rows_topk(Z, 1024)
    out = [torch.empty_like(t) for t in want]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    x = torch.full((binding._work_bytes("comet_rows_topk", comet.COMET_BF16, 300, 140001, 1024),), 3, dtype=torch.uint8, device="cuda")
    assert x.numel() > 1 << 20
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    torch.cuda._sleep(CYCLES)
    y.copy_(x)
    del x
    comet.comet_rows_topk(Z, 1024, crd=out[0], vals=out[1], lse=out[2], stream=side)
    torch.cuda.synchronize()
    assert bool((y == 3).all())
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_results_that_the_current_stream_reads_are_not_given_away():
    comet = _comet()
    Z = matrix(4096, 1500, torch.float32, seed=3)
    want = comet.comet_rows_topk(Z, 1024)[1]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    vals = comet.comet_rows_topk(Z, 1024, stream=side)[1]
    torch.cuda.current_stream().wait_stream(side)
    y = torch.empty_like(vals)
    torch.cuda._sleep(CYCLES)
    y.copy_(vals)
    del vals
    with torch.cuda.stream(side):
        again = [torch.zeros((4096, 1024), device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert len(again) == 3 and torch.equal(y, want)


def test_every_call_on_another_stream():
    comet = _comet()
    Z = matrix(6, 140001, torch.bfloat16, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, torch.cuda.current_stream(), side):
        crd, vals, lse = comet.comet_rows_topk(Z, 40, stream=stream)
        loss, stat = comet.comet_distill_forward(Z, crd, vals, tlse=lse, stream=stream)
        g = comet.comet_distill_backward(Z, crd, vals, stat, tlse=lse, stream=stream)
        both = comet.comet_distill_step(Z, crd, vals, tlse=lse, stream=stream)
        chosen = comet.comet_beam_select(Z.view(2, 3, -1), lse.view(2, 3), 4, stream=stream)
        torch.cuda.synchronize()
        got = [crd, vals, lse, loss, stat, g, *both, *chosen]
        if stream is None:
            want = got
        assert all(torch.equal(a, b) for a, b in zip(got, want))
