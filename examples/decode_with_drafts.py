"""Requests are answered token by token from a cache in blocks, with drafted tokens that are verified.

A small model (one layer of attention over what each request has read, random weights) and a smaller one that drafts for it.  A step is
    comet_cache_map      tables, slots and places for the tokens that every request adds: a prompt, or its last token and the drafted ones
    comet_cache_write    their keys and values into the cache, and the mean keys of the blocks that become whole
    comet_block_select   which blocks each query reads
    comet_block_attend   attention over them
    comet_draft_verify   how many of the drafted tokens stand, what follows them, and how long the requests are now
and nothing of it is known on the host but how many tokens there are at most.  Requests that have answered enough end, and others take
their rows and blocks.

    python examples/decode_with_drafts.py [--requests 12] [--drafts 3] [--temperature 0.7]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2102_05187_amd as comet  # noqa: E402

HEADS, GROUP, SIZE, BLOCK = 2, 4, 64, 16


class Model:
    """Token and place give a vector; queries, keys and values are linear in it; logits are linear in the attention's output and the vector."""

    def __init__(self, vocabulary, width, generator, dtype):
        def weight(*shape):
            return (torch.randn(shape, device="cuda", generator=generator) * shape[0] ** -0.5).to(dtype)
        self.token = weight(vocabulary, width) * vocabulary ** 0.5
        self.turn = torch.rand(width, device="cuda", generator=generator) * 0.004
        self.q, self.k, self.v = weight(width, HEADS * GROUP * SIZE), weight(width, HEADS * SIZE), weight(width, HEADS * SIZE)
        self.out, self.own = weight(HEADS * GROUP * SIZE, vocabulary) * 0.2, weight(width, vocabulary)

    def read(self, token, place):
        """(vector, q, k, v) of packed tokens."""
        x = self.token[token.long()] * torch.cos(place[:, None] * self.turn).to(self.token.dtype)
        return x, (x @ self.q).view(-1, HEADS * GROUP, SIZE), (x @ self.k).view(-1, HEADS, SIZE), (x @ self.v).view(-1, HEADS, SIZE)

    def logits(self, x, attended):
        return attended.reshape(len(x), -1) @ self.out + x @ self.own


class Cache:
    """Blocks of keys and values, and who has them."""

    def __init__(self, requests, blocks, most, dtype):
        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device="cuda")
        self.K, self.V = (torch.zeros((blocks, BLOCK, HEADS, SIZE), dtype=dtype, device="cuda") for _ in range(2))
        self.mean = torch.zeros((blocks, HEADS, SIZE), dtype=dtype, device="cuda")
        self.table, self.length, self.held = ints(requests, most), ints(requests), ints(requests)
        self.spare, self.count = torch.arange(blocks, dtype=torch.int32, device="cuda"), ints(1) + blocks


def step(model, cache, tokens, add, ended, chosen, whole=False):
    """Reads the requests' packed tokens, add[b] of each, and returns (pos, place, logits).  whole: every block is read."""
    N = len(tokens)
    pos, slot, place = comet.comet_cache_map(add, cache.length, cache.held, cache.table, cache.spare, cache.count, BLOCK, N, ended=ended)
    x, q, k, v = model.read(tokens, place)
    comet.comet_cache_write(k, v, cache.K, cache.V, slot, mean=cache.mean)
    K = cache.table.shape[1] if whole else chosen
    sel = comet.comet_block_select(q, cache.mean, cache.table, pos, cache.length, BLOCK, K, first=1, last=min(2, K - 1))
    attended, _ = comet.comet_block_attend(q, cache.K, cache.V, cache.table, pos, cache.length, sel)
    return pos, place, model.logits(x, attended)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--drafts", type=int, default=3)
    ap.add_argument("--vocabulary", type=int, default=501)
    ap.add_argument("--prompt", type=int, default=100, help="tokens of a prompt, at most")
    ap.add_argument("--answer", type=int, default=40, help="tokens after which a request ends")
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--chosen", type=int, default=6, help="blocks that a query reads")
    ap.add_argument("--temperature", type=float, default=0.7)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    B, T, V = a.requests, a.drafts, a.vocabulary
    model = Model(V, 128, g, torch.float32)
    # the draft knows the tokens alone: the target's logits without attention, and some noise
    draft = model.token.float() @ model.own.float()
    draft += 0.1 * torch.randn(draft.shape, device="cuda", generator=g)
    most = -(-(a.prompt + a.answer + 2 * (T + 1)) // BLOCK)
    cache = Cache(B, B * most, most, torch.float32)
    scale = 1.0 / a.temperature if a.temperature > 0 else float("inf")

    def prompts(which):
        n = torch.randint(1, a.prompt + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
        return torch.where(which, n, 0).int()

    history = [[] for _ in range(B)]
    answered = torch.zeros(B, dtype=torch.int32, device="cuda")
    last = torch.zeros(B, dtype=torch.int32, device="cuda")
    fresh = torch.ones(B, dtype=torch.bool, device="cuda")
    taken, finished = [], 0
    for number in range(a.steps):
        # new requests read their prompt, the others their last token and what is drafted behind it
        add = torch.where(fresh, prompts(fresh), T + 1).int()
        first = torch.cumsum(add, 0) - add
        N = int(add.sum())
        tokens = torch.randint(V, (N,), device="cuda", generator=g).int()
        q = torch.zeros((N, V), device="cuda")
        where = torch.nonzero(~fresh).flatten()
        token = last[where]
        for t in range(T + 1):
            tokens[first[where] + t] = token
            q[first[where] + t] = draft[token.long()]
            noise = torch.rand((len(where), V), device="cuda", generator=g).log_().neg_().log_().neg_() if a.temperature > 0 else 0.0
            token = (q[first[where] + t] * min(scale, 1e6) + noise).argmax(1).int()
        pos, place, logits = step(model, cache, tokens, add, fresh if number else None, a.chosen)
        # a prompt has no drafted tokens: its last row alone is drawn from, as a request of one row
        row = torch.arange(N, device="cuda")
        owner = torch.repeat_interleave(torch.arange(B, device="cuda"), add.long())
        keep = ~fresh[owner] | (row == (first + add - 1)[owner])
        some = torch.where(fresh, 1, T + 1)
        start = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        start[1:] = torch.cumsum(some, 0)
        u, v = torch.rand(int(some.sum()), device="cuda", generator=g), torch.rand(B, device="cuda", generator=g)
        accepted, follow = comet.comet_draft_verify(logits[keep].contiguous(), tokens[keep].contiguous(), start, u, v, draft=q[keep].contiguous(), scale=scale, length=cache.length)
        for b in range(B):
            if bool(fresh[b]):
                history[b] = tokens[int(first[b]):int(first[b] + add[b])].tolist()
            else:
                history[b] += tokens[int(first[b]) + 1:int(first[b] + accepted[b]) + 1].tolist()
            history[b].append(int(follow[b]))
        taken += accepted[~fresh].tolist()
        answered = torch.where(fresh, 1, answered + accepted + 1).int()
        last = follow
        # what the cache holds: everything but the token that was drawn last
        assert cache.length.tolist() == [len(h) - 1 for h in history]
        fresh = answered >= a.answer
        finished += int(fresh.sum())
    print("%d steps, %d requests answered, %.2f of %d drafted tokens taken, %d of %d blocks in use" % (
        a.steps, finished, sum(taken) / max(1, len(taken)), T, cache.K.shape[0] - int(cache.count), cache.K.shape[0]))
    return model, cache, history, taken, finished


if __name__ == "__main__":
    main()
