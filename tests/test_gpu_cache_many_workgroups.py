"""Calls over a cache in blocks that take more workgroups than a launch may have (2^32 threads), at sizes that their limits allow."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def _int(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("with_mean", [False, True])
def test_cache_write(with_mean):
    """2^26 rows and more, four a workgroup; with means, which run over the end of a launch's rows."""
    N, block = (1 << 26) + 1003, 16
    P = N // block + 2
    k = torch.arange(N, device="cuda", dtype=torch.int32).view(N, 1, 1).expand(N, 1, 4).contiguous().view(torch.bfloat16)       # 8 elements: i, four times
    k = (k.view(torch.int16) & 0x3fff).view(torch.bfloat16)                       # below 2, none of them infinite
    v = k.flip(0).contiguous()
    K, V = (torch.zeros((P, block, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mean = torch.full((P, 1, 8), -1, dtype=torch.bfloat16, device="cuda") if with_mean else None
    slot = torch.arange(9, N + 9, device="cuda")
    _comet().comet_cache_write(k, v, K, V, slot, mean)
    assert torch.equal(K.view(-1, 1, 8)[9:N + 9], k) and torch.equal(V.view(-1, 1, 8)[9:N + 9], v)
    if with_mean:
        whole = (N + 9) // block
        assert bool((mean[whole:] == -1).all())
        for lo in range(0, whole, 1 << 20):
            x = K[lo:min(lo + (1 << 20), whole)].float()
            # sixteen terms in 32 bits in one order or another, then half a step
            assert bool(((mean[lo:lo + (1 << 20)][:x.shape[0]].float() - x.mean(1)).abs() <= 2.0 ** -8 * x.mean(1) * 1.001 + 2.0 ** -120).all())


def test_block_select():
    """2^23 tokens of two heads, one a workgroup as the table has more than 1024 columns; all but the last 16000 lie before their request."""
    comet = _comet()
    N, few, M, K = 1 << 23, 16000, 1040, 4
    q = torch.randn((N, 2, 8), device="cuda").bfloat16()
    mean = torch.randn((M, 2, 8), device="cuda").bfloat16()
    table = torch.randperm(M, device="cuda").int()[None]
    sel = comet.comet_block_select(q, mean, table, _int(0, N), _int(few), 16, K)
    want = comet.comet_block_select(q[-few:], mean, table, _int(0, few), _int(few), 16, K)
    assert torch.equal(sel[-few:], want) and bool((sel[:-few] == -1).all())


def test_block_attend():
    """2^23 tokens of two heads of the cache with 33 heads each, which take two workgroups of a token."""
    comet = _comet()
    N, few = 1 << 23, 2000
    q = torch.randn((1, 66, 8), device="cuda").bfloat16().expand(N, 66, 8)
    K, V = (torch.randn((125, 16, 2, 8), device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(125, device="cuda").int()[None]
    sel = (torch.arange(N, device="cuda") % 125).int().view(N, 1, 1).expand(N, 2, 1).contiguous()
    out, lse = comet.comet_block_attend(q, K, V, table, _int(0, N), _int(few), sel)
    want = comet.comet_block_attend(q[-few:], K, V, table, _int(0, few), _int(few), sel[-few:].contiguous())
    assert torch.equal(out[-few:], want[0]) and torch.equal(lse[-few:], want[1])          # shared out in the same way
    assert bool((lse[:-few] == -math.inf).all())
    assert all(not bool(out[lo:lo + (1 << 20)][:max(0, N - few - lo)].any()) for lo in range(0, N, 1 << 20))


def test_draft_verify_of_many_rows():
    """2^23 rows, a workgroup for each of the target's and each of the draft's."""
    comet = _comet()
    N = 1 << 23
    Z, draft = (torch.randn((N, 9), device="cuda").bfloat16() for _ in range(2))
    token = torch.randint(9, (N,), device="cuda").int()
    u, v = torch.rand(N, device="cuda"), torch.rand(4, device="cuda")
    u[0] = u[7] = 2.0                                              # the first tokens of the long requests are not taken
    pos = _int(0, 7, N - 5, N - 5, N)
    accepted, follow = comet.comet_draft_verify(Z, token, pos, u, v, draft=draft)
    want = comet.comet_draft_verify(Z[-5:], token[-5:], _int(0, 5), u[-5:], v[3:], draft=draft[-5:])
    first = comet.comet_draft_verify(Z[:7], token[:7], _int(0, 7), u[:7], v[:1], draft=draft[:7])
    assert int(accepted[3]) == int(want[0]) and int(follow[3]) == int(want[1])
    assert accepted[:3].tolist() == [0, 0, 0] and int(follow[0]) == int(first[1]) and int(follow[2]) == -1 and 0 <= int(follow[1]) < 9


def test_draft_verify_of_many_requests():
    """2^23 requests, all without rows but two; rows of two pieces."""
    comet = _comet()
    B, V = 1 << 23, 3000
    Z = torch.randn((5, V), device="cuda")
    token = torch.randint(V, (5,), device="cuda").int()
    u, v = torch.rand(5, device="cuda"), torch.rand(B, device="cuda")
    pos = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    pos[B // 2 + 1:], pos[B:] = 2, 5
    accepted, follow = comet.comet_draft_verify(Z, token, pos, u, v)
    want = comet.comet_draft_verify(Z, token, _int(0, 2, 5), u, torch.stack([v[B // 2], v[B - 1]]))
    at = torch.tensor([B // 2, B - 1], device="cuda")
    assert torch.equal(accepted[at], want[0]) and torch.equal(follow[at], want[1])
    accepted[at], follow[at] = 0, -1
    assert not bool(accepted.any()) and bool((follow == -1).all())
