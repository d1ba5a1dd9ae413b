"""Plain 64-bit implementations of the operators on dense rows, on the host, from their definitions (row by row)."""
import math

import numpy as np
import torch

NO_TAIL_BELOW = 2.0 ** -20
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # 2^-p for p significant bits
TINY = {torch.float32: 2.0 ** -125, torch.bfloat16: 2.0 ** -125, torch.float16: 2.0 ** -25}   # what underflows

INF = math.inf


def sum_error(V):
    """Relative error that a 32-bit sum of exp over V places may have: every term's argument and exp round a few times
    (64 half units cover arguments of 20 and the joins of partial sums), and a thread adds up V / 64 terms at most in a row."""
    return 2.0 ** -24 * (64 + V / 64)


def lse_row(x):
    x = np.asarray(x, dtype=np.float64)
    if x.size == 0 or np.all(x == -INF):
        return -INF
    if np.any(np.isnan(x)):
        return math.nan
    m = x.max()
    if m == INF:
        return INF
    return m + math.log(np.exp(x - m).sum())


def log_softmax(x):
    """x - log sum exp(x), also where x is so large throughout that the logarithm would be lost in it."""
    with np.errstate(all="ignore"):
        m = x.max()
        return np.where(x == -INF, -INF, (x - m) - math.log(np.exp(x - m).sum())) if m > -INF else np.full(x.shape, -INF)


def topk_row(z, K, by_coordinate=False):
    """(coordinates, values) of the K largest; -1 and -inf where there are fewer."""
    z = np.asarray(z, dtype=np.float64)
    at = [int(i) for i in np.argsort(-z, kind="stable") if z[i] > -INF][:K]
    if by_coordinate:
        at.sort()
    return at + [-1] * (K - len(at)), [float(z[i]) for i in at] + [-INF] * (K - len(at))


def distill_row(z, crd, t, tlse, scale, weight, dloss=1.0):
    """(loss, gradient, sizes) of one row: the sizes are the sums of the magnitudes of each gradient's terms; tlse None: no tail."""
    z = np.asarray(z, dtype=np.float64)
    V = z.size
    if weight == 0:
        return 0.0, np.zeros(V), np.zeros(V)
    crd, t = np.asarray(crd, dtype=np.int64), np.asarray(t, dtype=np.float64)
    there = (crd >= 0) & (crd < V)
    crd, a = crd[there], t[there] * scale
    x = z * scale
    lse = lse_row(x)
    with np.errstate(all="ignore"):
        norm = lse_row(a) if tlse is None else float(tlse)
        logp = np.full(a.shape, -INF) if a.size == 0 else log_softmax(a) if tlse is None else a - norm
        p = np.where(a == -INF, 0.0, np.exp(logp))
        if math.isnan(lse) or lse == INF or np.any(np.isnan(p)) or math.isnan(norm):
            return math.nan, np.full(V, math.nan), np.full(V, math.nan)
        logq = log_softmax(x)
        q = np.exp(logq)
        loss = sum(pi * (lp - logq[c]) for pi, lp, c in zip(p, logp, crd) if pi > 0)
        outside = np.ones(V, dtype=bool)
        outside[crd] = False
        rest, ratio = 0.0, 0.0
        mass = math.fsum(p)
        if tlse is not None:
            rest = 1.0 - mass
            if rest < NO_TAIL_BELOW:
                rest = 0.0
            if rest > 0:
                loss += rest * (math.log(rest) - lse_row(logq[outside]))
            ratio = rest
        P = mass + rest
        g = P * q
        size = g.copy()
        if ratio:
            r = ratio * np.exp(log_softmax(x[outside])) if outside.any() else 0.0
            g[outside] -= r
            size[outside] += r
        g[crd] -= p
        size[crd] += p
    return weight * loss, weight * scale * dloss * g, abs(weight * scale * dloss) * size


def distill_bounds(z, loss, g, size, V, scale, weight, dtype):
    """How far a loss and a gradient computed with 32-bit sums and exponentials may be off: the sums' error in every log and
    quotient, an exponential's growing with its argument, and one rounding to the type."""
    z = np.asarray(z, dtype=np.float64)
    eps = sum_error(V)
    top = np.max(z[np.isfinite(z)], initial=0.0)
    arg = np.where(np.isfinite(z), np.abs(top - z), 0.0) * scale
    arg = np.minimum(arg, 200.0)             # beyond that everything is 0
    return (2.0 ** -23 * abs(loss) + 3 * eps * abs(weight),
            1.01 * UNIT[dtype] * np.abs(g) + size * (2 * eps + 2.0 ** -22 * (1 + arg)) + TINY[dtype])


def select_batch(z, score, n, finished=None, eos=0):
    """(scores, parents, tokens), and all candidates' scores in order."""
    z = np.asarray(z, dtype=np.float64)
    W, V = z.shape
    found = []
    for w in range(W):
        c = float(score[w])
        if finished is not None and finished[w]:
            found.append((-c, w, 0.0, eos) if c > -INF else None)
            continue
        with np.errstate(all="ignore"):
            s = c + (log_softmax(z[w]) if math.isfinite(lse_row(z[w])) else z[w] * math.nan)
        best = [int(v) for v in np.argsort(-z[w], kind="stable")[:n]]
        found += [(-s[v], w, -z[w][v], v) if s[v] > -INF else None for v in best]
    found = sorted(f for f in found if f is not None)
    every = [-f[0] for f in found]
    found = found[:n]
    pad = n - len(found)
    return ([-f[0] for f in found] + [-INF] * pad, [f[1] for f in found] + [-1] * pad, [f[3] for f in found] + [-1] * pad, every)
