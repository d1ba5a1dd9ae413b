"""The operators over a cache in blocks together, as a decoding loop calls them."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("decode_with_drafts", os.path.join(ROOT, "examples", "decode_with_drafts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("temperature", [0.7, 0.0])
def test_the_example_runs(temperature):
    example = _example()
    model, cache, history, taken, finished = example.main(["--requests", "5", "--steps", "20", "--prompt", "40", "--answer", "16", "--temperature", str(temperature)])
    # a step gives a token at least, so that every request has ended once by then
    assert finished >= 5 and all(0 <= n <= 3 for n in taken) and all(0 <= t < 501 for h in history for t in h)
    # no block is lost or had twice: those held and those spare are all there are
    held = [cache.table[b, :int(cache.held[b])].tolist() for b in range(5)]
    assert sorted(sum(held, cache.spare[:int(cache.count)].tolist())) == list(range(cache.K.shape[0]))
    # what the cache holds of a request is what its tokens give, drafted or not
    for b, tokens in enumerate(history):
        n = int(cache.length[b])
        _, _, k, v = model.read(torch.tensor(tokens[:n]).cuda(), torch.arange(n, dtype=torch.int32, device="cuda"))
        at = [held[b][p // example.BLOCK] * example.BLOCK + p % example.BLOCK for p in range(n)]
        for mine, cached in ((k, cache.K), (v, cache.V)):
            # products of 128 terms, added up in one order or another
            assert bool(((cached.flatten(0, 1)[at] - mine).abs() <= 2.0 ** -24 * 256 * (1 + mine.abs().max())).all())
        whole = n // example.BLOCK
        mean = cache.K[held[b][:whole]].double().mean(1)
        assert bool(((cache.mean[held[b][:whole]].double() - mean).abs() <= 2.0 ** -24 * 20 * (1 + cache.K.abs().max())).all())


def test_tokens_read_one_by_one_or_together():
    """Attention over all blocks, whatever the tokens arrive in: a whole prompt, parts of it, single tokens; against plain attention in 64 bits."""
    example = _example()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    model = example.Model(101, 128, g, torch.float32)
    B, most = 3, 8
    length = [70, 33, 100]
    tokens = [torch.randint(101, (n,), device="cuda", generator=g).int() for n in length]
    want = []
    for t in tokens:
        n = len(t)
        x, q, k, v = (y.double() for y in model.read(t, torch.arange(n, dtype=torch.int32, device="cuda")))
        k, v = k.repeat_interleave(example.GROUP, 1), v.repeat_interleave(example.GROUP, 1)
        z = torch.einsum("qhd,khd->hqk", q, k) * example.SIZE ** -0.5
        z = z.masked_fill(torch.arange(n, device="cuda") > torch.arange(n, device="cuda")[:, None], -math.inf)
        o = torch.einsum("hqk,khd->qhd", torch.softmax(z, 2), v)
        want.append(o.reshape(n, -1) @ model.out.double() + x @ model.own.double())
    size = max(float(w.abs().max()) for w in want)
    for parts in ([[70], [33], [100]], [[1] * 3 + [67], [30, 1, 1, 1], [5, 40, 50, 5]], [[20, 0, 49, 1], [0, 33, 0, 0], [64, 16, 16, 4]]):
        cache = example.Cache(B, B * most, most, torch.float32)
        read = [0] * B
        for i in range(max(len(p) for p in parts)):
            add = [p[i] if i < len(p) else 0 for p in parts]
            packed = torch.cat([tokens[b][read[b]:read[b] + add[b]] for b in range(B)])
            pos, place, logits = example.step(model, cache, packed, torch.tensor(add, dtype=torch.int32).cuda(), None, 4, whole=True)
            assert pos.tolist() == [sum(add[:b]) for b in range(B + 1)]
            for b in range(B):
                mine = logits[sum(add[:b]):sum(add[:b + 1])].double()
                # three products of a hundred terms in a row in 32 bits
                assert bool(((mine - want[b][read[b]:read[b] + add[b]]).abs() <= 2.0 ** -24 * 1024 * size).all())
                read[b] += add[b]
        assert read == length and cache.length.tolist() == length


def test_a_step_in_inference_mode():
    example = _example()
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    with torch.inference_mode():
        model = example.Model(101, 128, g, torch.float32)
        cache = example.Cache(2, 16, 8, torch.float32)
        for add in ([40, 3], [1, 1]):
            tokens = torch.zeros(sum(add), dtype=torch.int32, device="cuda")
            pos, _, logits = example.step(model, cache, tokens, torch.tensor(add, dtype=torch.int32).cuda(), None, 4)
        comet = example.comet
        u = torch.rand(2, device="cuda")
        accepted, follow = comet.comet_draft_verify(logits, tokens, pos, u, u, length=cache.length)
    assert cache.length.tolist() == [41, 4] and accepted.tolist() == [0, 0] and bool(((follow >= 0) & (follow < 101)).all())
