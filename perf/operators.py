"""Performance cases of the operators between a model's dense logits and their sparse top part.

The rows are tokens and the columns a vocabulary: `rows_topk` keeps the K largest logits of every row as a compressed
level (coordinates and values) with the row's log-sum-exp, `distill` is the loss of dense student logits against such
sparse teacher rows and its gradient, `beam_select` picks the best continuations over beams and vocabulary, and
`beam_reorder` lets the states of the beams follow.  The sizes are generic: vocabularies of 5 thousand to 131072,
one row to a few thousand.

A case is a dict of plain values:
  op       distill_step      the loss and its gradient, known row weights: what a training step calls
           distill_autograd  the loss, then the gradient for given derivatives of the losses: two calls, as automatic
                             differentiation makes them
           distill_loss      the loss alone: evaluation
           rows_topk, beam_select, beam_reorder
  dtype    bf16, f16, f32: the logits' or the states' type
  N, V     rows and vocabulary;  for the beams: B batches of W beams, V the vocabulary
  K        kept logits of a row (ragged: 0 to K of them, listed through a pos array)
  tail     the teacher's mass outside of what it kept counts as one more outcome
  ignored  rows of weight zero (prompt and padding tokens)
  n        continuations selected in each batch;  finished: beams of a batch that have ended
  states, heads, length, capacity, dim   beam_reorder: number of [B, W, heads, capacity, dim] tensors, of which the
           first `length` places are in use;  moved, sources: beams of a batch that get another one's state, and the
           number of different beams that they get it from
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
TEMPERATURE = 1.25
EOS = 1
NO_TAIL_BELOW = 2.0 ** -20     # a tail that 32-bit inputs do not resolve is none


# ---- cases ---------------------------------------------------------------------------------------------------------
def _distill(op, N, V, K, dtype, ragged=False, tail=False, ignored=0, **kw):
    return dict(kw, op=op, N=N, V=V, K=K, dtype=dtype, ragged=ragged, tail=tail, ignored=ignored)


def _topk(N, V, K, dtype, by_coordinate=False, **kw):
    return dict(kw, op="rows_topk", N=N, V=V, K=K, dtype=dtype, by_coordinate=by_coordinate)


def _select(B, W, V, n, dtype, finished=0, **kw):
    return dict(kw, op="beam_select", B=B, W=W, V=V, n=n, dtype=dtype, finished=finished)


def _reorder(B, W, states, heads, length, capacity, dim, moved, sources, dtype, **kw):
    return dict(kw, op="beam_reorder", B=B, W=W, states=states, heads=heads, length=length, capacity=capacity, dim=dim,
                moved=moved, sources=sources, dtype=dtype)


def listed():
    return [
        # a training step's loss on a micro-batch of 4096 tokens, a quarter of them prompt or padding
        _distill("distill_step", 4096, 131072, 64, "bf16", tail=True, ignored=1024, name="distill_step_4096x131072"),
        # the smallest step: a handful of tokens of a small vocabulary, where latency is all
        _distill("distill_step", 6, 5003, 8, "f32", name="distill_step_6x5003"),
        # evaluation on rows whose teacher kept what its mass asked for (ragged rows), an odd vocabulary
        _distill("distill_loss", 2048, 50021, 48, "f16", ragged=True, name="distill_loss_2048x50021"),
        # the same loss under automatic differentiation, logits kept in 32 bits
        _distill("distill_autograd", 1000, 32003, 100, "f32", ragged=True, tail=True, ignored=100,
                 name="distill_autograd_1000x32003"),
        # writing a teacher's top logits to disk: rows in the order of their coordinates
        _topk(2048, 131072, 64, "bf16", by_coordinate=True, name="rows_topk_2048x131072_k64"),
        # the candidates for sampling one token
        _topk(1, 32000, 50, "f32", name="rows_topk_1x32000_k50"),
        # a wide selection from a middling number of rows
        _topk(300, 60013, 500, "f16", name="rows_topk_300x60013_k500"),
        # one request decoded with four beams, twice as many continuations as beams
        _select(1, 4, 32000, 8, "bf16", name="beam_select_1x4x32000"),
        # a serving batch with some beams at their end
        _select(16, 8, 131072, 16, "bf16", finished=1, name="beam_select_16x8x131072"),
        # more and narrower beams, odd sizes, logits in 32 bits
        _select(24, 5, 50021, 10, "f32", finished=1, name="beam_select_24x5x50021"),
        # the caches of one request, short so far
        _reorder(1, 4, 16, 8, 333, 512, 64, 3, 1, "bf16", name="beam_reorder_1x4"),
        # the caches of a serving batch, long: the most bytes of all
        _reorder(8, 8, 16, 8, 2000, 2048, 128, 5, 2, "bf16", name="beam_reorder_8x8"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _vocabulary(rng):
    """An odd size or one that a vector width divides."""
    return _log(rng, 5003, 131072) if rng.random() < 0.6 else 8 * _log(rng, 625, 16384)


def draw(rng):
    op = rng.choice(("distill_step", "distill_autograd", "distill_loss", "rows_topk", "beam_select", "beam_reorder"))
    dtype = rng.choice(("bf16", "f16", "f32"))
    V = _vocabulary(rng)
    most = 4096 * 131072 // SIZE[dtype]            # elements: at most half of the largest case's bytes
    if op.startswith("distill"):
        N = _log(rng, 1, min(4096, most // V))
        return _distill(op, N, V, _log(rng, 1, 256), dtype, ragged=rng.random() < 0.5, tail=rng.random() < 0.5,
                        ignored=rng.choice((0, N // 8, N // 3)))
    if op == "rows_topk":
        return _topk(_log(rng, 1, min(4096, most // V)), V, _log(rng, 1, 512), dtype, by_coordinate=rng.random() < 0.5)
    W = rng.randint(2, 16)
    if op == "beam_select":
        return _select(_log(rng, 1, max(2, min(48, most // (V * W)))), W, V, rng.choice((W, 2 * W)), dtype, finished=rng.choice((0, 1, W // 4)))
    moved = rng.randint(2, W) if W > 2 else 2
    sources = rng.randint(1, W - moved) if moved < W else 0
    if moved > 2 and sources == 0:
        moved, sources = W - 1, 1
    B, heads, dim = _log(rng, 1, 16), rng.choice((1, 2, 4, 8, 12)), rng.choice((64, 80, 96, 128))
    states, length = 2 * rng.randint(1, 12), _log(rng, 1, 4000)
    while B * W * states * heads * length * dim * SIZE[dtype] > 2 << 30:
        length = max(1, length * 2 // 3)
        B = max(1, B * 2 // 3)
    return _reorder(B, W, states, heads, length, length + rng.randint(0, 100), dim, moved, sources, dtype)


# ---- inputs --------------------------------------------------------------------------------------------------------
def _logits(shape, dtype, g):
    """Most of a vocabulary near its mean, two dozen places of a row well above: what trained models give."""
    z = torch.randn(shape, device="cuda", generator=g).mul_(1.5).sub_(11.0)
    part = shape[-1] // 24
    hot = torch.arange(24, device="cuda") * part + torch.randint(part, (*shape[:-1], 24), device="cuda", generator=g)
    z.scatter_(-1, hot, torch.rand(hot.shape, device="cuda", generator=g).mul_(10.0).sub_(5.0))
    return z.to(TYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "rows_topk":
        s["Z"] = _logits((case["N"], case["V"]), case["dtype"], g)
    elif case["op"].startswith("distill"):
        N, V, K = case["N"], case["V"], min(case["K"], case["V"])
        Z = _logits((N, V), case["dtype"], g)
        crd = torch.empty((N, K), dtype=torch.int32, device="cuda")
        tvals = torch.empty((N, K), device="cuda")
        tlse = torch.empty(N, device="cuda")
        for r in range(0, N, 512):                  # the teacher agrees with the student up to some noise
            t = Z[r:r + 512].float()
            t = t.add_(torch.randn(t.shape, device="cuda", generator=g))
            tvals[r:r + 512], at = t.topk(K, dim=1)
            crd[r:r + 512] = at.int()
            tlse[r:r + 512] = torch.logsumexp(t.div_(TEMPERATURE), 1)
        s.update(Z=Z, crd=crd, tvals=tvals, pos=None, tlse=tlse if case["tail"] else None)
        if case["ragged"]:
            count = torch.randint(K + 1, (N,), device="cuda", generator=g)
            keep = torch.arange(K, device="cuda") < count[:, None]
            pos = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
            pos[1:] = torch.cumsum(count, 0)
            s.update(crd=crd[keep], tvals=tvals[keep], pos=pos)
        weight = torch.rand(N, device="cuda", generator=g) + 0.5
        weight[torch.randperm(N, device="cuda", generator=g)[:case["ignored"]]] = 0
        if case["dtype"] != "f16":                  # in 16 bits with a small exponent the loss is scaled up instead
            weight /= N
        s["weight"] = weight
        if case["op"] == "distill_autograd":
            s["dloss"] = torch.rand(N, device="cuda", generator=g) + 0.5
    elif case["op"] == "beam_select":
        B, W, V = case["B"], case["W"], case["V"]
        s["Z"] = _logits((B, W, V), case["dtype"], g)
        s["Z"][..., 0] = -math.inf                  # the padding token is never chosen
        s["score"] = torch.rand((B, W), device="cuda", generator=g).mul_(-6.0)
        ended = torch.rand((B, W), device="cuda", generator=g).argsort(1) < case["finished"]
        s["finished"] = ended if case["finished"] else None
    else:
        B, W = case["B"], case["W"]
        shape = (B, W, case["heads"], case["capacity"], case["dim"])
        s["whole"] = [torch.randn(shape, dtype=TYPES[case["dtype"]], device="cuda", generator=g) for _ in range(case["states"])]
        s["states"] = [x[:, :, :, :case["length"]] for x in s["whole"]]
        # two beams swap; the other moved ones take the state of `sources` beams that stay
        place = torch.rand((B, W), device="cuda", generator=g).argsort(1)
        moved, sources = case["moved"], case["sources"]
        parent = torch.arange(W, device="cuda").repeat(B, 1)
        parent.scatter_(1, place[:, 0:1], place[:, 1:2])
        parent.scatter_(1, place[:, 1:2], place[:, 0:1])
        if moved > 2:
            take = W - 1 - torch.arange(moved - 2, device="cuda") % sources
            parent.scatter_(1, place[:, 2:moved], place[:, take])
        s["parent"] = parent.int()
    return s


# ---- the operators in their plain form -----------------------------------------------------------------------------
def _order_key(x):
    """int64 whose order is that of x, equal values by the place along the last axis, lowest first; -inf and NaN last."""
    x = torch.where(torch.isnan(x), -math.inf, x) + 0.0
    bits = x.view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits + 2 ** 31), bits)
    return bits * 2 ** 32 - torch.arange(x.shape[-1], device=x.device)


def _lse(z):
    m = z.amax(-1, keepdim=True)
    return (m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))).squeeze(-1)


def _plain_topk(s):
    z, K = s["Z"].float(), s["case"]["K"]
    crd = _order_key(z).topk(K, dim=1).indices
    if s["case"]["by_coordinate"]:
        crd = crd.sort(dim=1).values
    vals = z.gather(1, crd)
    return {"crd": crd.int(), "vals": vals, "lse": _lse(z)}


def _plain_distill(s, gradient, dloss=None):
    c = s["case"]
    N, V, scale, w = c["N"], c["V"], 1.0 / TEMPERATURE, s["weight"]
    col = s["crd"].long().reshape(-1)
    if s["pos"] is None:
        row = torch.arange(N, device="cuda").repeat_interleave(col.numel() // N)
    else:
        row = torch.searchsorted(s["pos"].long(), torch.arange(col.numel(), device="cuda"), right=True) - 1
    t = s["tvals"].reshape(-1) * scale
    zero = torch.zeros(N, device="cuda")
    if c["tail"]:
        logp = t - s["tlse"][row]
    else:
        m = torch.full_like(zero, -math.inf).scatter_reduce(0, row, t, "amax")
        logp = t - m[row] - torch.log(zero.index_add(0, row, torch.exp(t - m[row])))[row]
    p = torch.exp(logp)
    mass = zero.index_add(0, row, p)
    z = s["Z"].float() * scale
    logq = z - _lse(z)[:, None]
    loss = zero.index_add(0, row, p * (logp - logq[row, col]))
    if gradient or c["tail"]:
        q = torch.exp(logq)
        del z, logq
    if c["tail"]:
        rest = 1.0 - mass
        rest = torch.where(rest < NO_TAIL_BELOW, 0.0, rest)
        outside = torch.ones((N, V), dtype=torch.bool, device="cuda")
        outside[row, col] = False
        qrest = torch.where(outside, q, 0.0).sum(1)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(qrest)), 0.0)
        mass = mass + rest
    loss = torch.where(w > 0, w * loss, 0.0)
    if not gradient:
        return {"loss": loss}
    up = w * scale if dloss is None else w * scale * dloss
    d = q * mass[:, None]
    if c["tail"]:
        d = torch.where(outside, d - q * (rest / qrest)[:, None], d)
    d[row, col] -= p
    d = torch.where((w > 0)[:, None], d * up[:, None], 0.0)
    return {"loss": loss, "dZ": d.to(s["Z"].dtype)}


def _plain_select(s):
    c = s["case"]
    z = s["Z"].float()
    scores = s["score"][..., None] + (z - _lse(z)[..., None])
    if s["finished"] is not None:
        only = torch.where(torch.arange(c["V"], device="cuda") == EOS, s["score"][..., None], -math.inf)
        scores = torch.where(s["finished"][..., None], only, scores)
    scores = scores.reshape(c["B"], -1)
    at = _order_key(scores).topk(c["n"], dim=1).indices
    best = scores.gather(1, at)
    none = best == -math.inf
    parent = torch.where(none, -1, torch.div(at, c["V"], rounding_mode="floor"))
    return {"score": best, "parent": parent.int(), "token": torch.where(none, -1, at % c["V"]).int()}


def _plain_reorder(s):
    batch, parent = torch.arange(s["case"]["B"], device="cuda")[:, None], s["parent"].long()
    for x in s["states"]:
        x.copy_(x[batch, parent])
    return {"states": s["whole"]}


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(s):
    c, op = s["case"], s["case"]["op"]
    if not own:
        if op == "rows_topk":
            return _plain_topk(s)
        if op == "beam_select":
            return _plain_select(s)
        if op == "beam_reorder":
            return _plain_reorder(s)
        return _plain_distill(s, op != "distill_loss", s.get("dloss"))
    import paper_2102_05187_amd as comet
    if op == "rows_topk":
        crd, vals, lse = comet.comet_rows_topk(s["Z"], c["K"], by_coordinate=c["by_coordinate"])
        return {"crd": crd, "vals": vals, "lse": lse}
    if op == "beam_select":
        score, parent, token = comet.comet_beam_select(s["Z"], s["score"], c["n"], finished=s["finished"], eos=EOS)
        return {"score": score, "parent": parent, "token": token}
    if op == "beam_reorder":
        comet.comet_beam_reorder(s["states"], s["parent"])
        return {"states": s["whole"]}
    rows = dict(pos=s["pos"], tlse=s["tlse"], scale=1.0 / TEMPERATURE, weight=s["weight"])
    if op == "distill_loss":
        return {"loss": comet.comet_distill_forward(s["Z"], s["crd"], s["tvals"], **rows)[0]}
    if op == "distill_step":
        loss, dZ = comet.comet_distill_step(s["Z"], s["crd"], s["tvals"], **rows)
        return {"loss": loss, "dZ": dZ}
    loss, stat = comet.comet_distill_forward(s["Z"], s["crd"], s["tvals"], **rows)
    dZ = comet.comet_distill_backward(s["Z"], s["crd"], s["tvals"], stat, dloss=s["dloss"], **rows)
    return {"loss": loss, "dZ": dZ}


def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] == "rows_topk":
        N, V, K = case["N"], case["V"], min(case["K"], case["V"])
        return {"bytes": N * (V * size + K * 8 + 4), "flops": N * V * 4}
    if case["op"] == "beam_select":
        B, W, V = case["B"], case["W"], case["V"]
        return {"bytes": B * ((W - case["finished"]) * V * size + W * 5 + case["n"] * 12), "flops": B * W * V * 4}
    if case["op"] == "beam_reorder":
        place = case["heads"] * case["length"] * case["dim"] * size * case["states"]
        sources = 2 + (case["sources"] if case["moved"] > 2 else 0)
        return {"bytes": case["B"] * ((sources + case["moved"]) * place + case["W"] * 4), "flops": 0}
    N, V, K = case["N"], case["V"], min(case["K"], case["V"])
    read = (N - case["ignored"]) * (V * size + (K / 2 if case["ragged"] else K) * 8) + N * 8
    if case["op"] == "distill_loss":
        return {"bytes": read, "flops": (N - case["ignored"]) * V * 4}
    return {"bytes": read + N * V * size, "flops": (N - case["ignored"]) * V * 8}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "beam_reorder":
        return None                                 # nothing is computed: the states are moved as they are
    s = prepare(case, seed)
    if case["op"] == "rows_topk":
        crd, vals, lse = [], [], []
        for z in s["Z"].split(256):
            v, at = torch.sort(z.double(), dim=1, descending=True, stable=True)
            v, at = v[:, :case["K"]], at[:, :case["K"]]
            if case["by_coordinate"]:
                at, by = at.sort(dim=1)
                v = v.gather(1, by)
            crd.append(at.int())
            vals.append(v)
            lse.append(torch.logsumexp(z.double(), 1))
        return {"crd": torch.cat(crd), "vals": torch.cat(vals), "lse": torch.cat(lse)}
    if case["op"] == "beam_select":
        score, parent, token = [], [], []
        for b in range(case["B"]):
            x = s["score"][b].double()[:, None] + torch.log_softmax(s["Z"][b].double(), 1)
            if s["finished"] is not None:
                x[s["finished"][b]] = -math.inf
                x[s["finished"][b], EOS] = s["score"][b].double()[s["finished"][b]]
            v, at = torch.sort(x.flatten(), descending=True, stable=True)
            score.append(v[:case["n"]])
            parent.append((at[:case["n"]] // case["V"]).int())
            token.append((at[:case["n"]] % case["V"]).int())
        return {"score": torch.stack(score), "parent": torch.stack(parent), "token": torch.stack(token)}
    N, V, K = case["N"], case["V"], min(case["K"], case["V"])
    if s["pos"] is None:
        begin = torch.arange(N, device="cuda") * K
        count = torch.full((N,), K, device="cuda")
    else:
        begin, count = s["pos"][:-1].long(), s["pos"][1:].long() - s["pos"][:-1].long()
    crd, tvals = s["crd"].reshape(-1), s["tvals"].reshape(-1).double()
    out = {"loss": torch.zeros(N, dtype=torch.float64, device="cuda")}
    if case["op"] != "distill_loss":
        out["dZ"] = torch.zeros((N, V), dtype=torch.float64, device="cuda")
    for r0 in range(0, N, 256):
        rows = slice(r0, min(N, r0 + 256))
        z = s["Z"][rows].double().requires_grad_()
        # teacher rows padded to K places; a place that is none has no probability
        at = (begin[rows, None] + torch.arange(K, device="cuda")).clamp(max=max(0, crd.numel() - 1))
        there = torch.arange(K, device="cuda") < count[rows, None]
        t = torch.where(there, tvals[at] / TEMPERATURE, -math.inf) if crd.numel() else torch.full(at.shape, -math.inf, device="cuda").double()
        col = torch.where(there, crd[at].long(), 0) if crd.numel() else at * 0
        if case["tail"]:
            p = torch.exp(t - s["tlse"][rows].double()[:, None])
        else:
            p = torch.where(there.any(1, keepdim=True), torch.softmax(t, 1), 0.0)
        x = z / TEMPERATURE
        logq = x.gather(1, col) - torch.logsumexp(x, 1, keepdim=True)
        terms = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, 1.0)) - logq), 0.0)
        loss = terms.sum(1)
        if case["tail"]:
            rest = 1.0 - p.sum(1)
            rest = torch.where(rest < NO_TAIL_BELOW, 0.0, rest)
            spare = torch.zeros((z.shape[0], V + 1), dtype=torch.bool, device="cuda")
            spare.scatter_(1, torch.where(there, col, V), True)
            logrest = torch.logsumexp(x.masked_fill(spare[:, :V], -math.inf), 1) - torch.logsumexp(x, 1)
            loss = loss + torch.where(rest > 0, rest * (torch.log(torch.where(rest > 0, rest, 1.0)) - logrest), 0.0)
        w = s["weight"][rows].double()
        out["loss"][rows] = (w * loss).detach()
        if "dZ" in out:
            up = w if "dloss" not in s else w * s["dloss"][rows].double()
            out["dZ"][rows] = torch.autograd.grad((up * loss).sum(), z)[0]
    return out
