"""Layouts that the operators over a cache in blocks do not take: elements that lie at one place, or apart."""
import pytest
import torch

gpu = pytest.mark.gpu


def test_the_last_dimension_is_read_as_it_lies():
    from paper_2102_05187_amd import binding
    lines = lambda t: binding._lines(t.shape, t.stride(), t.itemsize)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    assert lines(x)[0] == (128, 64)
    assert lines(x[:, :, :8])[0] == (128, 64) and lines(x[:1])[0] == (0, 64) and lines(x.transpose(0, 1))[0] == (64, 128)
    assert lines(x[:, :1].expand(4, 2, 64))[0] == (128, 0)
    assert lines(torch.zeros((1, 1, 1)))[0] == (0, 0) and lines(torch.zeros((0, 2, 64)))[0] == (0, 64)
    assert lines(torch.zeros(1, dtype=torch.bfloat16).expand(4, 2, 128)) is None
    assert lines(torch.zeros((4, 8))[:, :1, None].expand(4, 1, 64)) is None
    assert lines(torch.zeros((4, 2, 64)).transpose(1, 2)) is None and lines(x[:, :, ::2]) is None


@gpu
@pytest.mark.parametrize("which", ["q", "K", "V", "mean", "k", "v"])
def test_expanded_vectors_are_refused(which):
    import paper_2102_05187_amd as comet
    from cache_util import make
    s = make([2, 3], [100, 90], 2, 2, 64, 16, torch.bfloat16, K=4)
    s["slot"] = torch.arange(5, device="cuda")
    s["k"], s["v"] = (torch.zeros((5, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s[which] = torch.zeros(1, dtype=torch.bfloat16, device="cuda").expand(s[which].shape)
    calls = []
    if which in ("q", "mean"):
        calls.append(lambda: comet.comet_block_select(s["q"], s["mean"], s["table"], s["pos"], s["length"], 16, 4))
    if which in ("q", "K", "V"):
        calls.append(lambda: comet.comet_block_attend(s["q"], s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"]))
    if which != "q":
        calls.append(lambda: comet.comet_cache_write(s["k"], s["v"], s["K"], s["V"], s["slot"], s["mean"]))
    for call in calls:
        with pytest.raises(ValueError):
            call()


@gpu
def test_queries_that_share_memory_are_read():
    """A head that all heads of the queries are: a stride of 0 in front of the last dimension is a layout as any other."""
    import paper_2102_05187_amd as comet
    from cache_util import make
    s = make([2, 3], [100, 90], 2, 2, 64, 16, torch.bfloat16, K=4)
    q = s["q"][:, :1].expand(5, 4, 64)
    for a, b in zip(comet.comet_block_attend(q, s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"]),
                    comet.comet_block_attend(q.contiguous(), s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"])):
        assert torch.equal(a, b)


def test_a_cache_that_is_written_lies_apart():
    import ctypes
    from paper_2102_05187_amd import binding, build
    build.build_if_missing()
    two, p, invalid = ctypes.c_int64 * 2, ctypes.c_void_p(4096), 1

    def write(ks=(2048, 128, 64), vs=(2048, 128, 64), ms=(128, 64), mean=4096, blocks=10, block=16, heads=2, N=3):
        c = binding._Cache(4096, 4096, mean, 1, blocks, block, heads, 64)
        c.key_stride[:], c.value_stride[:], c.mean_stride[:] = ks, vs, ms
        return binding._lib().comet_cache_write(ctypes.byref(c), N, p, two(128, 64), p, two(128, 64), p, None)

    for kw in (dict(ks=(0, 128, 64)), dict(ks=(2048, 0, 64)), dict(ks=(2048, 128, 0)), dict(ks=(2048, 128, 56)), dict(vs=(0, 128, 64)), dict(vs=(2048, 8, 64)),
               dict(vs=(2048, 128, 0)), dict(ms=(0, 64)), dict(ms=(128, 0)), dict(ms=(128, 32))):
        assert write(**kw) == invalid, kw
    # of one element, or without means: nothing to lie apart
    assert write(ks=(0, 64, 0), vs=(0, 64, 0), ms=(0, 0), blocks=1, heads=1, N=0) == 0
    assert write(ms=(0, 0), mean=None, N=0) == 0
    apart = lambda t: binding._apart(t.shape, t.stride())
    x = torch.zeros((4, 16, 2, 64))
    assert apart(x) and apart(x.transpose(1, 2)) and apart(x[..., :8]) and apart(x[:1].expand(1, 16, 2, 64)) and apart(x[:0])
    assert not apart(x[:1].expand(4, 16, 2, 64)) and not apart(x[:, :1].expand(4, 16, 2, 64)) and not apart(x[:, :, :1].expand(4, 16, 2, 64))


@gpu
@pytest.mark.parametrize("which", ["K", "V", "mean"])
def test_a_cache_of_one_block_many_times_is_not_written(which):
    import paper_2102_05187_amd as comet
    from cache_util import make
    s = make([2, 3], [100, 90], 2, 2, 64, 16, torch.bfloat16)
    s["slot"] = torch.arange(5, device="cuda")
    k, v = (torch.zeros((5, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s[which] = s[which][:1].expand(s[which].shape)
    with pytest.raises(ValueError):
        comet.comet_cache_write(k, v, s["K"], s["V"], s["slot"], s["mean"])
