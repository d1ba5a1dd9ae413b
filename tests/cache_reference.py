"""Plain implementations of the operators over a cache in blocks and of the drafts' verification, on the host, from their definitions."""
import math

import numpy as np
import torch

INF = math.inf
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # half a step, relative


def cache_map(add, ended, length, held, table, spare, count, block, N):
    """(pos, slot, place, length, held, table, spare, count) afterwards, request by request; lists in, lists out."""
    length, held, table, spare, count = list(length), list(held), [list(r) for r in table], list(spare), int(count)
    B, M, S = len(add), len(table[0]) if table else 0, len(spare)
    held = [min(max(h, 0), M) for h in held]
    length = [min(max(n, 0), h * block) for n, h in zip(length, held)]
    count = min(max(count, 0), S)
    for b in range(B):
        if ended is not None and ended[b]:
            for j in range(held[b]):
                if count < S:
                    spare[count] = table[b][j]
                    count += 1
            held[b] = length[b] = 0
    blocks = tokens = 0
    top, taken = count, 0
    pos, slot, place = [0], [], []
    for b in range(B):
        n = max(add[b], 0)
        if length[b] + n > M * block:
            pos.append(pos[-1])
            continue
        want = max(0, -(-(length[b] + n) // block) - held[b])
        blocks += want
        tokens += n
        if tokens > N or (want and blocks > top):
            pos.append(pos[-1])
            continue
        for _ in range(want):
            table[b][held[b]] = spare[top - 1 - taken]
            held[b] += 1
            taken += 1
        for p in range(length[b], length[b] + n):
            slot.append(table[b][p // block] * block + p % block)
            place.append(p)
        length[b] += n
        pos.append(pos[-1] + n)
    slot += [-1] * (N - len(slot))
    place += [-1] * (N - len(place))
    return pos, slot, place, length, held, table, spare, count - taken


def rows_of(pos, length):
    """(row, request, place) of every packed row."""
    return [(r, b, length[b] - pos[b + 1] + r) for b in range(len(length)) for r in range(pos[b], pos[b + 1])]


def block_select(q, mean, table, pos, length, block, K, first=1, last=1):
    """{row: [heads, K]}; q [N, Q, D], mean [P, H, D] as 64-bit arrays."""
    H = mean.shape[1]
    out = {}
    for r, b, p in rows_of(pos, length):
        C = min(p // block + 1 if p >= 0 else 0, len(table[b]))
        rows = []
        for h in range(H):
            x = q[r].reshape(H, -1, q.shape[2])[h].sum(0)
            if C <= K:
                rows.append(list(range(C)) + [-1] * (K - C))
                continue
            score = []
            for j in range(C):
                t = table[b][j]
                s = float(np.dot(x, mean[t, h])) if 0 <= t < mean.shape[0] else math.nan
                forced = j < first or j >= C - last
                score.append(((0, 0.0) if forced else (2, 0.0) if math.isnan(s) else (1, -s)) + (j,))
            rows.append(sorted(j for _, _, j in sorted(score)[:K]))
        out[r] = rows
    return out


def block_attend(q, K, V, table, pos, length, sel, scale):
    """{row: (out [Q, D], lse [Q], scores' size)}, arrays of 64 bits."""
    block, H = K.shape[1], K.shape[2]
    G = q.shape[1] // H
    out = {}
    for r, b, p in rows_of(pos, length):
        o, lse = np.zeros(q.shape[1:]), np.full(q.shape[1], -INF)
        mass = np.zeros(q.shape[1:])
        for h in range(H):
            named = sorted({int(j) for j in sel[r][h] if 0 <= j < len(table[b]) and j * block <= p})
            named = [j for j in named if 0 <= table[b][j] < K.shape[0]]
            if not named:
                continue
            at = [(table[b][j], i) for j in named for i in range(block) if j * block + i <= p]
            k = np.stack([K[t, i, h] for t, i in at])
            v = np.stack([V[t, i, h] for t, i in at])
            with np.errstate(all="ignore"):
                z = scale * (k @ q[r, h * G:h * G + G].T)             # places x G
                m = z.max(0)
                w = np.exp(z - np.where(m == -INF, 0, m))
                total = w.sum(0)
                lse[h * G:h * G + G] = np.where(total == 0, -INF, m + np.log(total))
                w = np.where(total == 0, 0, w / total)
                o[h * G:h * G + G] = w.T @ v
                mass[h * G:h * G + G] = w.T @ np.abs(v)
        out[r] = (o, lse, mass)
    return out


def softmax(x, scale):
    """None where it has no probabilities."""
    x = np.asarray(x, dtype=np.float64)
    if x.size == 0 or np.isnan(x).any() or not x.max() < INF or x.max() == -INF or not scale > 0:
        return None
    if scale == INF:
        e = (np.arange(x.size) == int(np.argmax(x))).astype(np.float64)
    else:
        e = np.exp((x - x.max()) * scale)
    return e / e.sum()


def draft_verify(Z, token, pos, u, v, scale, draft=None, crd=None, vals=None):
    """[(accepted, next, margin)] of the requests; margin: how far the nearest decision was from being another one."""
    V, out = Z.shape[1], []
    for b in range(len(pos) - 1):
        rows = range(pos[b], pos[b + 1])
        if len(rows) == 0:
            out.append((0, -1, INF))
            continue
        took, margin, q = 0, INF, None
        for r in rows[:-1]:
            d, p = int(token[r + 1]), softmax(Z[r], scale[b])
            if draft is not None:
                q = softmax(draft[r], scale[b])
                q = np.zeros(V) if q is None else q
            elif crd is not None:
                inside = [k for k in range(crd.shape[1]) if 0 <= crd[r, k] < V]
                q, e = np.zeros(V), softmax([vals[r, k] for k in inside], scale[b])
                if e is not None:
                    for k, x in zip(inside, e):
                        q[crd[r, k]] += x
            else:
                q = np.zeros(V)
                if 0 <= d < V:
                    q[d] = 1.0
            if p is None or not 0 <= d < V:
                break
            if scale[b] == INF:
                if Z[r, d] != Z[r].max():
                    break
            else:
                margin = min(margin, abs(u[r] * q[d] - p[d]))
                if not u[r] * q[d] < p[d]:
                    break
            took += 1
        r = pos[b] + took
        p = softmax(Z[r], scale[b])
        if p is None:
            out.append((took, -1, margin))
            continue
        w = p
        if took < len(rows) - 1 and scale[b] != INF:
            w = np.maximum(p - q, 0)
            if not w.sum() > 0:
                w = p
        run = np.cumsum(w)
        goal = v[b] * run[-1] if scale[b] != INF else 0
        over = np.nonzero(run > goal)[0]
        at = int(over[0]) if len(over) else int(np.nonzero(w)[0][-1])
        if scale[b] != INF:
            margin = min(margin, np.min(np.abs(run - goal)) / run[-1])
        out.append((took, at, margin))
    return out
