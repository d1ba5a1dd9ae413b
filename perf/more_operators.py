"""Performance cases of a decoding step over a cache that is kept in blocks.

A cache holds keys and values in blocks of a few dozen places; a request's blocks lie anywhere, and its table says where.
`cache_map` builds tables and slots on the device from the requests' lengths, `cache_write` puts new keys and values in their
slots and keeps the mean key of every whole block, `block_select` chooses blocks for each query by those means, `block_attend` is
attention over the chosen blocks, and `draft_verify` takes drafted tokens against the target's logits.  The sizes are generic:
vocabularies of 5 thousand to 131072, contexts of one place to 32768, one token to a few thousand.

A case is a dict of plain values:
  op       cache_map, cache_write, block_select, block_attend, draft_verify
  dtype    bf16, f16, f32: the type of cache, queries or logits
  B        requests;  N tokens of all of them together (block_select, block_attend: not evenly, where N > B);  context: the longest one
  H, G, D  heads of the cache, queries' heads of each, size of a head
  block, K places of a block, chosen blocks of a query
  M        cache_map: blocks that a request may have;  prompts: requests that end and make room for a new prompt, of up to
           `longest` tokens;  the others add up to `step` tokens
  T, V     draft_verify: drafted tokens of a request at most, vocabulary;  kept: what is known of the draft's distribution: all
           of its logits (-1), that many of them, or the token alone (0)
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
TEMPERATURE = 0.8


# ---- cases ---------------------------------------------------------------------------------------------------------
def _map(B, M, block, prompts, longest, step, **kw):
    return dict(kw, op="cache_map", B=B, M=M, block=block, prompts=prompts, longest=longest, step=step)


def _write(B, N, H, D, block, dtype, **kw):
    return dict(kw, op="cache_write", B=B, N=N, H=H, D=D, block=block, dtype=dtype)


def _sparse(op, B, N, context, H, G, D, block, K, dtype, **kw):
    return dict(kw, op=op, B=B, N=N, context=context, H=H, G=G, D=D, block=block, K=K, dtype=dtype)


def _verify(B, T, V, kept, dtype, **kw):
    return dict(kw, op="draft_verify", B=B, T=T, V=V, kept=kept, dtype=dtype)


def listed():
    return [
        # a few requests that decode token by token: latency is all
        _map(8, 8192, 16, 0, 0, 1, name="cache_map_8"),
        # a serving step that mixes decoding with drafts and new prompts: about 130 thousand tokens, and room for twice as many
        _map(512, 2048, 64, 128, 2048, 5, name="cache_map_512"),
        # one new token for each of 64 requests
        _write(64, 64, 8, 128, 64, "bf16", name="cache_write_64"),
        # the prompts of three requests, which end inside of blocks
        _write(3, 8191, 8, 128, 64, "f16", name="cache_write_8191"),
        # decoding: the blocks of 16 queries in contexts of up to 32768 places
        _sparse("block_select", 16, 16, 32768, 8, 4, 128, 64, 32, "bf16", name="block_select_16"),
        # a part of three long prompts
        _sparse("block_select", 3, 4093, 16384, 4, 8, 128, 64, 16, "f16", name="block_select_4093"),
        # one token of one request, an odd number of heads: the smallest call
        _sparse("block_attend", 1, 1, 777, 2, 7, 64, 16, 16, "f16", name="block_attend_1"),
        # decoding a serving batch
        _sparse("block_attend", 64, 64, 32768, 8, 4, 128, 64, 32, "bf16", name="block_attend_64"),
        # a few drafted tokens of each request, 32 bits, odd sizes throughout
        _sparse("block_attend", 24, 71, 5000, 3, 5, 80, 32, 20, "f32", name="block_attend_71"),
        # a part of three long prompts: the most operations
        _sparse("block_attend", 3, 4093, 16384, 4, 8, 128, 64, 16, "bf16", name="block_attend_4093"),
        # two requests with three drafted tokens, of whose distribution the top is known
        _verify(2, 3, 32000, 50, "f32", name="draft_verify_2x3"),
        # a serving batch, four drafted tokens each, the draft's logits whole
        _verify(64, 4, 131072, -1, "bf16", name="draft_verify_64x4"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("cache_map", "cache_write", "block_select", "block_attend", "block_attend", "draft_verify"))
    dtype = rng.choice(("bf16", "f16", "f32"))
    block = rng.choice((16, 32, 64, 128))
    if op == "cache_map":
        B = _log(rng, 1, 512)
        prompts = rng.choice((0, B // 8, B // 4))
        return _map(B, 131072 // block, block, prompts, _log(rng, 1, 2048), rng.randint(1, 8))
    H, D = rng.choice((1, 2, 3, 4, 8)), rng.choice((64, 72, 80, 96, 128))
    B = _log(rng, 1, 64)
    if op == "cache_write":
        return _write(B, max(B, _log(rng, 1, 8191)), H, D, block, dtype)
    if op == "draft_verify":
        T, V = rng.randint(1, 7), _log(rng, 5003, 131072) if rng.random() < 0.6 else 8 * _log(rng, 625, 16384)
        B = min(B, max(1, (64 * 5 * 131072 * 2) // ((T + 1) * V * SIZE[dtype])))
        return _verify(B, T, V, rng.choice((-1, 0, 1, _log(rng, 2, 200))), dtype)
    G, K = rng.choice((1, 2, 4, 5, 7, 8, 12)), _log(rng, 3, 48)
    kind = rng.choice(("token", "drafts", "prompt"))
    if kind == "prompt":                            # at most a third of the largest case's operations
        B = rng.randint(1, 4)
        most = 4093 * 32 * 128 * 1024 // 3 // (H * G * D * min(K * block, 16384))
        N = max(B, _log(rng, 8, max(9, min(4093, most))))
        context = N + _log(rng, 1, 16384 - 4093)
    else:
        N = B if kind == "token" else B * rng.randint(2, 6) + rng.randint(0, B - 1)
        context = _log(rng, max(8, N // B + 1), 32768)
    while op == "block_attend" and N * H * min(K * block, context) * D * SIZE[dtype] > 64 * 8 * 2048 * 128 * 2 * (2 if kind == "prompt" else 1) and K > 3:
        K = max(3, K * 2 // 3)
    return _sparse(op, B, N, context, H, G, D, block, K, dtype)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _parts(total, parts, rng):
    """`total` as that many numbers of 1 and more, uneven."""
    cut = torch.rand(parts, generator=rng) + 0.2
    n = 1 + torch.floor(cut / cut.sum() * (total - parts)).long()
    n[0] += total - int(n.sum())
    return n


def _start(n):
    pos = torch.zeros(n.numel() + 1, dtype=torch.int32)
    pos[1:] = torch.cumsum(n, 0)
    return pos


def _blocks_of(n, block):
    return (n + block - 1) // block


def _tables(length, block, P, g):
    """The table: the blocks of all requests in no order, anywhere among the cache's P."""
    held = _blocks_of(length, block)
    total = int(held.sum())
    ids = torch.randperm(P, device="cuda", generator=g).int()
    table = torch.zeros((length.numel(), max(1, int(held.max()))), dtype=torch.int32, device="cuda")
    at = torch.arange(table.shape[1], device="cuda") < held.cuda()[:, None]
    table[at] = ids[:total]
    return table


def _prepare_map(c, g, host):
    B, M, block = c["B"], c["M"], c["block"]
    most = M * block
    prompt = torch.arange(B) < c["prompts"]
    prompt = prompt[torch.randperm(B, generator=host)]
    add = torch.where(prompt, torch.randint(1, max(1, c["longest"]) + 1, (B,), generator=host), torch.randint(1, c["step"] + 1, (B,), generator=host))
    length = torch.floor((most // 8) ** torch.rand(B, generator=host)).long()
    held = _blocks_of(length, block)
    total = int(held.sum())
    ids = torch.randperm(B * M, device="cuda", generator=g).int()
    table = torch.full((B, M), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(M, device="cuda") < held.cuda()[:, None]] = ids[:total]
    spare = torch.full((B * M,), -1, dtype=torch.int32, device="cuda")
    spare[:B * M - total] = ids[total:]
    return {"add": add.int().cuda(), "ended": prompt.cuda() if c["prompts"] else None, "length": length.int().cuda(), "held": held.int().cuda(), "table": table,
            "spare": spare, "count": torch.tensor([B * M - total], dtype=torch.int32, device="cuda"), "N": c["prompts"] * c["longest"] + (B - c["prompts"]) * c["step"]}


def _prepare_write(c, g, host):
    B, N, H, D, block, kind = c["B"], c["N"], c["H"], c["D"], c["block"], TYPES[c["dtype"]]
    n = _parts(N, B, host)
    length = n + torch.randint(0, 4 * block, (B,), generator=host)
    P = N // block + 6 * B
    table = _tables(length, block, P, g)
    b = torch.arange(B).repeat_interleave(n).cuda()
    place = torch.arange(N, device="cuda") - _start(n).cuda().long()[b] + (length - n).cuda()[b]
    s = {"slot": table[b, place // block].long() * block + place % block}
    for name in ("K", "V"):
        s[name] = torch.randn((P, block, H, D), device="cuda", generator=g).to(kind)
        s[name.lower()] = torch.randn((N, H, D), device="cuda", generator=g).to(kind)
    s["mean"] = s["K"].float().mean(1).to(kind)
    return s


def _prepare_sparse(c, g, host):
    """Keys that lean to their block's topic and queries that lean to their neighbours': what trained models give."""
    B, N, H, G, D, block, kind = c["B"], c["N"], c["H"], c["G"], c["D"], c["block"], TYPES[c["dtype"]]
    n = _parts(N, B, host)
    room = (c["context"] - n).clamp(min=0).float()
    length = n + torch.floor(room * (0.25 + 0.75 * torch.rand(B, generator=host))).long()
    P = int(_blocks_of(length, block).sum()) + 5
    table = _tables(length, block, P, g)
    topic = torch.randn((P, 1, H, D), device="cuda", generator=g)
    span = torch.randn((N // 32 + 1, H * G, D), device="cuda", generator=g).repeat_interleave(32, 0)[:N]
    s = {"q": (span + torch.randn((N, H * G, D), device="cuda", generator=g)).to(kind), "table": table, "pos": _start(n).cuda(), "length": length.int().cuda()}
    if c["op"] == "block_select":
        s["mean"] = topic.squeeze(1).add_(torch.randn((P, H, D), device="cuda", generator=g), alpha=block ** -0.5).to(kind)
        return s
    s["mean"] = topic.squeeze(1).to(kind)
    s["sel"] = _plain_select(dict(s, case=c))
    del s["mean"]
    # part by part: the largest cache is gigabytes
    for name, lean in (("K", 1.0), ("V", 0.0)):
        s[name] = torch.empty((P, block, H, D), dtype=kind, device="cuda")
        for p in range(0, P, 4096):
            x = torch.randn(s[name][p:p + 4096].shape, device="cuda", generator=g)
            s[name][p:p + 4096] = x.add_(topic[p:p + 4096], alpha=lean)
    return s


def _prepare_verify(c, g, host):
    B, T, V, kind = c["B"], c["T"], c["V"], TYPES[c["dtype"]]
    n = torch.randint(1, T + 2, (B,), generator=host)
    n[0] = T + 1
    N = int(n.sum())
    # most of a vocabulary near its mean, two dozen places of a row well above: what trained models give
    z = torch.randn((N, V), device="cuda", generator=g).mul_(1.5).sub_(11.0)
    part = V // 24
    hot = torch.arange(24, device="cuda") * part + torch.randint(part, (N, 24), device="cuda", generator=g)
    z.scatter_(1, hot, torch.rand(hot.shape, device="cuda", generator=g).mul_(10.0).sub_(5.0))
    x = z + torch.randn((N, V), device="cuda", generator=g).mul_(0.5)
    s = {"Z": z.to(kind), "draft": None, "crd": None, "vals": None, "pos": _start(n).cuda(), "length": (n + 100).int().cuda(),
         "u": torch.rand(N, device="cuda", generator=g), "v": torch.rand(B, device="cuda", generator=g)}
    del z
    if c["kept"] < 0:
        s["draft"] = x = x.to(kind)
    elif c["kept"] > 0:
        vals, crd = x.topk(c["kept"], dim=1)
        s["vals"], s["crd"] = vals, crd.int()
        x = torch.full_like(x, -math.inf).scatter_(1, crd, vals)
    # the drafted tokens are drawn from the draft's distribution (of which nothing is told where kept is 0)
    noise = torch.rand(x.shape, device="cuda", generator=g).clamp_(min=1e-30).log_().neg_().log_().neg_()
    token = torch.zeros(N, dtype=torch.int32, device="cuda")
    token[1:] = (x.float() / TEMPERATURE + noise).argmax(1)[:-1].int()
    s["token"] = token
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    make = {"cache_map": _prepare_map, "cache_write": _prepare_write, "draft_verify": _prepare_verify}.get(case["op"], _prepare_sparse)
    return dict(make(case, g, host), case=case)


# ---- the operators in their plain form -----------------------------------------------------------------------------
def _plain_map(s):
    c = s["case"]
    B, M, block, N = c["B"], c["M"], c["block"], s["N"]
    length, held, table, spare, count = s["length"], s["held"], s["table"], s["spare"], s["count"]
    at = torch.arange(M, device="cuda")
    if s["ended"] is not None:
        back = (at < held[:, None]) & s["ended"][:, None]
        rank = torch.cumsum(back.flatten(), 0) - 1
        longer = torch.cat([spare, spare[:1]])
        longer[torch.where(back.flatten(), count + rank, spare.numel())] = table.flatten()
        spare.copy_(longer[:-1])
        count += back.sum().int()
        length.masked_fill_(s["ended"], 0)
        held.masked_fill_(s["ended"], 0)
    add = s["add"].clamp(min=0).long()
    fits = length + add <= M * block
    want = torch.where(fits, (_blocks_of(length + add, block) - held).clamp(min=0), 0)
    blocks, tokens = torch.cumsum(want, 0), torch.cumsum(torch.where(fits, add, 0), 0)
    granted = fits & (tokens <= N) & ((want == 0) | (blocks <= count))
    want, add = torch.where(granted, want, 0), torch.where(granted, add, 0)
    first = torch.cumsum(want, 0) - want
    new = at - held[:, None]
    source = (count - 1 - first[:, None] - new).clamp(min=0, max=spare.numel() - 1)
    table.copy_(torch.where((new >= 0) & (new < want[:, None]), spare[source], table))
    count -= want.sum().int()
    held += want.int()
    pos = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    pos[1:] = torch.cumsum(add, 0)
    i = torch.arange(N, device="cuda")
    b = torch.searchsorted(pos[1:].long(), i, right=True).clamp(max=B - 1)
    place = length[b] + i - pos[b]
    there = i < pos[B]
    slot = table[b, torch.where(there, place // block, 0).long()].long() * block + place % block
    length += add.int()
    return {"pos": pos, "slot": torch.where(there, slot, -1), "place": torch.where(there, place, -1).int()}


def _plain_write(s):
    K, V, slot, block = s["K"], s["V"], s["slot"], s["case"]["block"]
    K.view(-1, *K.shape[2:])[slot] = s["k"]
    V.view(-1, *V.shape[2:])[slot] = s["v"]
    whole = torch.div(slot[slot % block == block - 1], block, rounding_mode="floor")
    s["mean"][whole] = (K[whole].float().sum(1) / block).to(K.dtype)


def _requests(s):
    """Request and place of every query."""
    i = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(s["pos"][1:].long(), i, right=True)
    return b, s["length"][b].long() - s["pos"][b + 1].long() + i


def _plain_select(s, first=1, last=1):
    c = s["case"]
    H, G, K, block, table = c["H"], c["G"], c["K"], c["block"], s["table"]
    q = s["q"].double().view(-1, H, G, c["D"]).sum(2)
    request, place = _requests(s)
    mine = torch.div(place, block, rounding_mode="floor")[:, None, None]
    j = torch.arange(table.shape[1], device="cuda")
    sel = torch.empty((q.shape[0], H, K), dtype=torch.int32, device="cuda")
    start = s["pos"].tolist()
    for b in range(c["B"]):
        mean = s["mean"][table[b].long()].double()
        for r in range(start[b], start[b + 1], 256):
            rows = slice(r, min(r + 256, start[b + 1]))
            own_block = mine[rows]
            score = torch.matmul(q[rows].transpose(0, 1).contiguous(), mean.permute(1, 2, 0).contiguous()).transpose(0, 1)
            score = torch.where((j < first) | (j > own_block - last), math.inf, score)
            score = torch.where(j > own_block, -math.inf, score)
            at = score.sort(dim=2, descending=True, stable=True).indices[:, :, :K]
            at = torch.where(at > own_block, table.shape[1], at).sort(dim=2).values
            if at.shape[2] < K:
                at = torch.nn.functional.pad(at, (0, K - at.shape[2]), value=table.shape[1])
            sel[rows] = torch.where(at == table.shape[1], -1, at).int()
    return sel


def _plain_attend(s):
    c = s["case"]
    H, G, D, block = c["H"], c["G"], c["D"], c["block"]
    q, sel = s["q"], s["sel"]
    N = q.shape[0]
    request, place = _requests(s)
    out, lse = torch.empty_like(q), torch.empty((N, H * G), device="cuda")
    head = torch.arange(H, device="cuda")[:, None]
    rows = max(1, (1 << 28) // (H * sel.shape[2] * block * D))
    for r in range(0, N, rows):
        x = sel[r:r + rows].long()                                  # n, H, K
        n = x.shape[0]
        keys = x[..., None] * block + torch.arange(block, device="cuda")
        ok = ((x >= 0)[..., None] & (keys <= place[r:r + rows, None, None, None])).view(n, H, 1, -1)
        at = s["table"][request[r:r + rows, None, None], x.clamp(min=0)].long()
        k = s["K"][at, :, head].view(n * H, -1, D).float()          # n H, K block, D
        z = torch.bmm(q[r:r + rows].reshape(n * H, G, D).float(), k.transpose(1, 2)).view(n, H, G, -1) * D ** -0.5
        z = torch.where(ok, z, -math.inf)
        m = z.amax(3, keepdim=True)
        p = torch.exp(z - m)
        total = p.sum(3, keepdim=True)
        v = s["V"][at, :, head].view(n * H, -1, D).float()
        o = torch.bmm((p / total).view(n * H, G, -1), v)
        out[r:r + rows] = o.view(n, H * G, D).to(q.dtype)
        lse[r:r + rows] = (m + torch.log(total)).view(n, H * G)
    return {"out": out, "lse": lse}


def _plain_verify(s):
    c = s["case"]
    Z, pos, token, B, T, V = s["Z"], s["pos"].long(), s["token"].long(), c["B"], c["T"], c["V"]
    N = Z.shape[0]
    row = torch.arange(N, device="cuda")

    def softmax(x):
        e = torch.exp((x - x.amax(1, keepdim=True)) / TEMPERATURE)
        return e / e.sum(1, keepdim=True)

    p = softmax(Z.double())
    d = torch.cat([token[1:], token[:1]])
    if c["kept"] < 0:
        q = softmax(s["draft"].double())
    elif c["kept"] > 0:
        q = torch.zeros_like(p).scatter_(1, s["crd"].long(), softmax(s["vals"].double()))
    else:
        q = torch.zeros_like(p).scatter_(1, d[:, None], 1.0)
    took = s["u"] * q[row, d] < p[row, d]
    drafted = pos[1:] - pos[:-1] - 1
    t = torch.arange(T, device="cuda")
    judged = t < drafted[:, None]
    run = torch.cumprod((took[(pos[:-1, None] + t).clamp(max=N - 1)] & judged).int(), 1)
    accepted = run.sum(1)
    at = pos[:-1] + accepted
    weight = torch.where((accepted < drafted)[:, None], (p[at] - q[at]).clamp(min=0), p[at])
    weight = torch.where(weight.sum(1, keepdim=True) > 0, weight, p[at])
    up_to = torch.cumsum(weight, 1)
    over = up_to > s["v"].double()[:, None] * up_to[:, -1:]
    # the first place behind which the sum is beyond the drawn part of it
    follow = over.int().argmax(1)
    return {"accepted": accepted.int(), "next": follow.int()}


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    c, op = s["case"], s["case"]["op"]
    if op == "cache_map":
        if own:
            import paper_2102_05187_amd as comet
            pos, slot, place = comet.comet_cache_map(s["add"], s["length"], s["held"], s["table"], s["spare"], s["count"], c["block"], s["N"], ended=s["ended"])
            made = {"pos": pos, "slot": slot, "place": place}
        else:
            made = _plain_map(s)
        return dict(made, **{name: s[name] for name in ("length", "held", "table", "spare", "count")})
    if op == "cache_write":
        if own:
            import paper_2102_05187_amd as comet
            comet.comet_cache_write(s["k"], s["v"], s["K"], s["V"], s["slot"], mean=s["mean"])
        else:
            _plain_write(s)
        return {name: s[name] for name in ("K", "V", "mean")}
    if not own:
        if op == "block_select":
            return {"sel": _plain_select(s)}
        return _plain_attend(s) if op == "block_attend" else _plain_verify(s)
    import paper_2102_05187_amd as comet
    if op == "block_select":
        return {"sel": comet.comet_block_select(s["q"], s["mean"], s["table"], s["pos"], s["length"], c["block"], c["K"])}
    if op == "block_attend":
        out, lse = comet.comet_block_attend(s["q"], s["K"], s["V"], s["table"], s["pos"], s["length"], s["sel"])
        return {"out": out, "lse": lse}
    accepted, follow = comet.comet_draft_verify(s["Z"], s["token"], s["pos"], s["u"], s["v"], draft=s["draft"], crd=s["crd"], vals=s["vals"],
                                                scale=1.0 / TEMPERATURE)
    return {"accepted": accepted, "next": follow}


def work(case):
    """Lengths are drawn from the seed; these are their means."""
    if case["op"] == "cache_map":
        N = case["prompts"] * (case["longest"] + 1) / 2 + (case["B"] - case["prompts"]) * (case["step"] + 1) / 2
        return {"bytes": int(12 * N + case["B"] * 24 + 8 * N / case["block"]), "flops": 0}
    size = SIZE[case["dtype"]] if "dtype" in case else 0
    if case["op"] == "cache_write":
        place = case["H"] * case["D"] * size
        return {"bytes": int(case["N"] * (4 * place + 8 + place / case["block"])), "flops": case["N"] * case["H"] * case["D"]}
    if case["op"] == "draft_verify":
        rows = case["B"] * (case["T"] + 2) / 2
        read = rows * (case["V"] * size + 8) + (rows - case["B"]) * (case["V"] * size if case["kept"] < 0 else 8 * case["kept"])
        return {"bytes": int(read), "flops": int(rows * case["V"] * (8 if case["kept"] < 0 else 4))}
    B, N, H, G, D, block, K = (case[k] for k in ("B", "N", "H", "G", "D", "block", "K"))
    length = N / B + max(0, case["context"] - N / B) * 0.625
    asked = N * H * G * D * size
    if case["op"] == "block_select":
        blocks = length / block
        return {"bytes": int(asked + B * H * blocks * D * size + N * H * K * 4), "flops": int(2 * N * H * blocks * D)}
    seen = min(K * block, length)
    # every query reads what it chose, but no more than there is
    return {"bytes": int(2 * asked + 2 * min(N * seen, B * length) * H * D * size), "flops": int(4 * N * H * G * seen * D)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] not in ("cache_write", "block_attend"):
        return None                                 # whole numbers
    s = prepare(case, seed)
    if case["op"] == "cache_write":
        mean = s["mean"].double()
        block = case["block"]
        key = s["K"].flatten(0, 1)
        key.index_copy_(0, s["slot"], s["k"])
        for slot in s["slot"].tolist():
            if slot % block == block - 1:
                mean[slot // block] = key[slot - block + 1:slot + 1].double().mean(0)
        return {"K": None, "V": None, "mean": mean}
    H, G, D, block = case["H"], case["G"], case["D"], case["block"]
    N = s["q"].shape[0]
    out = torch.empty((N, H * G, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((N, H * G), dtype=torch.float64, device="cuda")
    start, length, table = s["pos"].tolist(), s["length"].tolist(), s["table"]
    for b in range(case["B"]):
        n = start[b + 1] - start[b]
        used = -(-length[b] // block)
        for h in range(H):
            # the request's places in a row, and which of them each query sees
            key = s["K"][table[b, :used].long(), :, h].reshape(used * block, D).double()
            value = s["V"][table[b, :used].long(), :, h].reshape(used * block, D).double()
            for i in range(0, n, 512):
                m = min(512, n - i)
                rows = slice(start[b] + i, start[b] + i + m)
                chosen = torch.zeros((m, used + 1), dtype=torch.bool, device="cuda")
                at = s["sel"][rows, h].long()
                chosen.scatter_(1, torch.where(at < 0, used, at), True)
                place = length[b] - n + i + torch.arange(m, device="cuda")
                seen = chosen[:, :used].repeat_interleave(block, 1) & (torch.arange(used * block, device="cuda") <= place[:, None])
                for g in range(h * G, h * G + G):
                    z = (s["q"][rows, g].double() @ key.t() / math.sqrt(D)).masked_fill(~seen, -math.inf)
                    out[rows, g] = torch.softmax(z, 1) @ value
                    lse[rows, g] = torch.logsumexp(z, 1)
    return {"out": out, "lse": lse}
