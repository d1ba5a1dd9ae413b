"""Keys and values into their slots, bit for bit, and the means of whole blocks."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _comet():
    import paper_2102_05187_amd as comet
    return comet


def check(slot, P, block, H, D, dtype, seed=0, mean=True, arrange=lambda t: t, stream=None):
    comet = _comet()
    g = torch.Generator().manual_seed(seed)
    N = len(slot)
    make = lambda *shape: arrange(torch.randn(shape, generator=g).to(dtype).cuda())
    K, V, k, v = make(P, block, H, D), make(P, block, H, D), make(N, H, D), make(N, H, D)
    m = torch.full((P, H, D), 7.0, dtype=dtype, device="cuda") if mean else None
    want = [K.clone(), V.clone()]
    whole = []
    for i, s in enumerate(slot):
        if 0 <= s < P * block:
            want[0][s // block, s % block], want[1][s // block, s % block] = k[i], v[i]
            if s % block == block - 1:
                whole.append(s // block)
    comet.comet_cache_write(k, v, K, V, torch.tensor(slot, dtype=torch.int64).cuda(), mean=m, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])
    if not mean:
        return
    rest = torch.ones(P, dtype=torch.bool, device="cuda")
    rest[whole] = False
    assert bool((m[rest] == 7).all())
    exact = want[0][whole].double()
    # sums of `block` terms in 32 bits, the quotient and the result rounded once each
    off = ref.UNIT[dtype] * exact.mean(1).abs() + 2.0 ** -24 * (block + 1) * exact.abs().mean(1) * 1.01 + 2.0 ** -25 * (dtype == torch.float16)
    assert bool(((m[whole].double() - exact.mean(1)).abs() <= off).all())


def run_of(table, first, n, block):
    return [table[p // block] * block + p % block for p in range(first, first + n)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block,H,D", [(16, 1, 8), (16, 3, 64), (48, 2, 72), (64, 8, 128), (128, 5, 256), (1024, 1, 16)])
def test_sizes(block, H, D, dtype):
    table = [3, 0, 5, 1]
    for first, n in ((0, 1), (block - 1, 1), (block - 2, 3), (0, block), (5, 2 * block + 3), (0, 4 * block)):
        check(run_of(table, first, n, block), 7, block, H, D, dtype, seed=n)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_requests_and_rows(dtype):
    slot = []
    for r in range(40):
        slot += run_of([r * 5 + i for i in (4, 0, 3, 1)], (r * 13) % 50, 1 + (r * 29) % 75, 32)
    check(slot, 200, 32, 2, 64, dtype)
    slot = run_of([i ^ 5 for i in range(320)], 3, 5000, 16)
    check(slot, 320, 16, 2, 80, dtype, seed=2)


def test_slots_that_are_none():
    check([-1, 5, 16 * 4, 6, -1, 2 ** 40, 7, -2 ** 60], 4, 16, 2, 64, torch.bfloat16)
    check([], 4, 16, 2, 64, torch.bfloat16)
    check([31, -1, 15], 4, 16, 2, 64, torch.bfloat16)


def test_without_means():
    check(run_of([2, 0, 1], 0, 40, 16), 3, 16, 2, 64, torch.float16, mean=False)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(dtype):
    def arrange(t):                              # heads outermost, and room behind each vector
        order = (len(t.shape) - 2, *range(len(t.shape) - 2), len(t.shape) - 1)
        back = [order.index(i) for i in range(len(order))]
        wide = torch.zeros((*[t.shape[i] for i in order[:-1]], t.shape[-1] + 8), dtype=t.dtype, device=t.device)
        wide = wide[..., :t.shape[-1]].permute(back)
        wide.copy_(t)
        return wide
    check(run_of([2, 0, 1, 4], 3, 50, 16), 5, 16, 3, 64, dtype, arrange=arrange)


def test_a_cache_of_more_than_4_gib():
    comet = _comet()
    P, block, H, D = 140000, 64, 2, 128              # 4.6 GB each
    K, V = (torch.zeros((P, block, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m = torch.zeros((P, H, D), dtype=torch.bfloat16, device="cuda")
    slot = torch.tensor(run_of([0, P - 1], 0, 128, block)).cuda()
    k, v = (torch.randn((128, H, D), device="cuda").bfloat16() for _ in range(2))
    comet.comet_cache_write(k, v, K, V, slot, mean=m)
    torch.cuda.synchronize()
    assert torch.equal(K[P - 1], k[64:]) and torch.equal(V[P - 1], v[64:]) and torch.equal(K[0], k[:64])
    assert int((K != 0).any(3).any(2).sum()) == 128
    # 64 terms of size 1 in 32 bits, one rounding to 16
    assert bool(((m[P - 1].double() - k[64:].double().mean(0)).abs() <= 2.0 ** -8 * k[64:].double().mean(0).abs() + 2.0 ** -17).all())
