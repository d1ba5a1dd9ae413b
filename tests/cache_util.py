"""Inputs for the tests of the operators over a cache in blocks."""
import torch


def make(news, lengths, H, G, D, block, dtype, seed=0, K=None, spread=1.0, spare=3):
    """A cache whose unused places hold NaN, packed queries, and a choice of blocks: news[b] new tokens of lengths[b] in all."""
    g = torch.Generator().manual_seed(seed)
    B, N = len(news), sum(news)
    blocks = [-(-n // block) for n in lengths]
    M, P = max([1] + blocks), sum(blocks) + spare
    ids = torch.randperm(P, generator=g).tolist()
    table = torch.full((B, M), -5, dtype=torch.int32)
    keys, values = (torch.full((P, block, H, D), float("nan")) for _ in range(2))
    for b in range(B):
        for j in range(blocks[b]):
            p = ids.pop()
            table[b, j] = p
            n = min(block, lengths[b] - j * block)
            for t in (keys, values):
                t[p, :n] = torch.randn((n, H, D), generator=g)
    q = torch.randn((N, H * G, D), generator=g) * spread
    pos = torch.tensor([0] + torch.tensor(news).cumsum(0).tolist() if B else [0], dtype=torch.int32)
    s = dict(q=q.to(dtype), K=keys.to(dtype), V=values.to(dtype), table=table, pos=pos, length=torch.tensor(lengths, dtype=torch.int32))
    mean = torch.randn((P, H, D), generator=g)
    s["mean"] = mean.to(dtype)
    if K is not None:
        sel = torch.full((N, H, K), -1, dtype=torch.int32)
        for b in range(B):
            for r in range(int(pos[b]), int(pos[b + 1])):
                p = lengths[b] - int(pos[b + 1]) + r
                for h in range(H):
                    seen = torch.randperm(p // block + 1, generator=g)[:K].sort().values
                    if K > 1 and p // block not in seen.tolist():
                        seen[-1] = p // block
                    sel[r, h, :len(seen)] = seen.int()
        s["sel"] = sel
    return {name: t.cuda() for name, t in s.items()}


def host(t):
    return t.double().cpu().numpy()
