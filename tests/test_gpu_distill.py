"""Distillation from a teacher's top logits: loss and gradient against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
INF = math.inf


def _comet():
    import paper_2102_05187_amd as comet
    return comet


class Problem:
    """Student logits, teacher rows and weights on the device; `counts` None: K entries in each row, else ragged rows."""

    def __init__(self, N, V, K, dtype, seed=0, tail=False, ragged=False, weighted=True, scale=0.8, ld=None, start=0, spread=2.0):
        rng = np.random.RandomState(seed)
        ld = ld or V
        self.N, self.V, self.dtype, self.scale, self.ld, self.start = N, V, dtype, scale, ld, start
        Z = torch.from_numpy(rng.randn(N, V).astype(np.float32) * spread).to(dtype)
        teacher = Z.double().numpy() + rng.randn(N, V)
        self.rows = []
        for r in range(N):
            n = rng.randint(0, K + 1) if ragged else K
            c = rng.permutation(V)[:n]
            c = np.append(c, np.full(n - c.size, -1))
            self.rows.append((c, np.where(c >= 0, teacher[r][c], -INF).astype(np.float32)))
        self.tlse = [np.float32(ref.lse_row(teacher[r] * scale)) for r in range(N)] if tail else None
        self.weight = (rng.rand(N).astype(np.float32) + 0.5) * (rng.rand(N) < 0.8) if weighted else None
        self.dloss = rng.randn(N).astype(np.float32)
        self.ragged = ragged
        self.set(Z)

    def set(self, Z):
        """Takes over student logits and the teacher's rows as they are now."""
        self.host = Z.double().numpy()
        flat = torch.zeros(self.start + max(1, self.N) * self.ld, dtype=self.dtype, device="cuda")
        self.Z = flat[self.start:].view(max(1, self.N), self.ld)[:self.N, :self.V]
        self.Z.copy_(Z.cuda())
        self.args()

    def args(self):
        cuda = lambda x, t: None if x is None else torch.tensor(np.asarray(x), dtype=t, device="cuda")  # noqa: E731
        c = np.concatenate([r[0] for r in self.rows]) if self.rows else np.zeros(0)
        t = np.concatenate([r[1] for r in self.rows]) if self.rows else np.zeros(0)
        self.crd, self.tvals, self.pos = cuda(c, torch.int32), cuda(t, torch.float32), None
        if self.ragged:
            self.pos = cuda(np.concatenate([[0], np.cumsum([r[0].size for r in self.rows])]), torch.int32)
        else:
            K = self.rows[0][0].size if self.rows else 0
            self.crd, self.tvals = self.crd.view(self.N, K), self.tvals.view(self.N, K)
        self.kw = dict(pos=self.pos, tlse=cuda(self.tlse, torch.float32), scale=self.scale, weight=cuda(self.weight, torch.float32))

    def reference(self, r, dloss):
        w = 1.0 if self.weight is None else float(self.weight[r])
        return ref.distill_row(self.host[r], *self.rows[r], None if self.tlse is None else self.tlse[r], self.scale, w, dloss), w

    def compare(self, loss, dZ, dloss=None):
        loss, dZ = loss.double().cpu().numpy(), None if dZ is None else dZ.double().cpu().numpy()
        for r in range(self.N):
            up = 1.0 if dloss is None else float(dloss[r])
            (want, g, size), w = self.reference(r, up)
            bl, bg = ref.distill_bounds(self.host[r], want if math.isfinite(want) else 0.0, g, size, self.V, self.scale, w, self.dtype)
            if math.isfinite(want):
                assert abs(loss[r] - want) <= bl, ("loss", r, loss[r], want, bl)
            else:
                assert loss[r] == want or (math.isnan(want) and math.isnan(loss[r])), ("loss", r, loss[r], want)
            if dZ is not None and not math.isnan(want):
                off = np.abs(dZ[r] - g) - bg
                assert off.max(initial=-1) <= 0, ("gradient", r, int(off.argmax()), dZ[r][off.argmax()], g[off.argmax()], bg[off.argmax()])
            elif dZ is not None:
                assert np.isnan(dZ[r]).all(), ("gradient", r)

    def check(self):
        comet = _comet()
        dl = torch.tensor(self.dloss, device="cuda")
        loss, stat = comet.comet_distill_forward(self.Z, self.crd, self.tvals, **self.kw)
        g1 = comet.comet_distill_backward(self.Z, self.crd, self.tvals, stat, **self.kw)
        g2 = comet.comet_distill_backward(self.Z, self.crd, self.tvals, stat, dloss=dl, **self.kw)
        loss2, g3 = comet.comet_distill_step(self.Z, self.crd, self.tvals, **self.kw)
        torch.cuda.synchronize()
        self.compare(loss, g1)
        self.compare(loss, g2, self.dloss)
        self.compare(loss2, g3)
        # in place
        keep = self.Z.clone()
        out = comet.comet_distill_backward(self.Z, self.crd, self.tvals, stat, dZ=self.Z, dloss=dl, **self.kw)
        assert out is self.Z
        torch.cuda.synchronize()
        self.compare(loss, self.Z, self.dloss)
        self.Z.copy_(keep)
        loss3, _ = comet.comet_distill_step(self.Z, self.crd, self.tvals, dZ=self.Z, **self.kw)
        torch.cuda.synchronize()
        self.compare(loss3, self.Z)
        self.Z.copy_(keep)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (2, 2, 1), (3, 7, 7), (2, 8, 3), (3, 9, 0), (3, 63, 5), (4, 64, 64), (2, 65, 1), (5, 1000, 40), (3, 2049, 300),
                                   (9, 4099, 17), (2, 5003, 1500), (1, 32003, 50), (2, 32769, 8), (1, 70001, 100), (2, 131072, 64), (1, 140001, 64)])
def test_sizes(N, V, K, tail, dtype):
    Problem(N, V, K, dtype, seed=N + V + K, tail=tail, weighted=N > 2).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,V", [(2, 1024), (2, 4097), (2, 8193), (2, 16384), (2, 16391), (70, 16400), (3, 32768), (3, 65536), (2, 65543), (66, 65537), (2, 131079),
                                 (3, 300007)])
def test_around_the_sizes_of_pieces(N, V, dtype):
    Problem(N, V, 9, dtype, seed=V, tail=True, weighted=N > 60).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
def test_ragged_rows(tail, dtype):
    Problem(12, 3001, 40, dtype, seed=1, tail=tail, ragged=True).check()
    Problem(40, 50, 6, dtype, seed=2, tail=tail, ragged=True).check()
    Problem(3, 40009, 3000, dtype, seed=3, tail=tail, ragged=True).check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("start", [0, 1, 3, 6])
@pytest.mark.parametrize("ld", [1001, 1003, 1008, 1500])
def test_rows_anywhere(ld, start, dtype):
    Problem(5, 1001, 20, dtype, seed=ld + start, tail=True, ld=ld, start=start).check()


def test_gradient_of_another_row_distance_leaves_the_gaps_alone():
    comet = _comet()
    for dtype in DTYPES:
        p = Problem(4, 1001, 20, dtype, seed=5, tail=True)
        wide = torch.full((4, 1100), 7.0, dtype=dtype, device="cuda")
        loss, g = comet.comet_distill_step(p.Z, p.crd, p.tvals, dZ=wide[:, 3:1004], **p.kw)
        torch.cuda.synchronize()
        p.compare(loss, wide[:, 3:1004])
        assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 1004:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("V", [11, 3001, 40009])
def test_rows_of_every_kind(V, tail, dtype):
    """Masked places, rows of the lowest value, rows without a place or an entry, entries without a probability."""
    low = torch.finfo(dtype).min
    p = Problem(14, V, 5, dtype, seed=V, tail=tail, weighted=False, scale=1.0)
    Z = torch.tensor(p.host)
    Z[0] = -INF                                                  # no place is left: loss +inf
    Z[1, :] = low                                                # all equal, by the lowest value
    Z[2, 1:] = low                                               # one place
    Z[3, torch.arange(V) % 2 == 0] = -INF                        # half masked, entries maybe among them
    Z[4, torch.tensor(p.rows[4][0])] = -INF                      # the entries' places masked: loss +inf
    outside = torch.ones(V, dtype=torch.bool)
    outside[torch.tensor(p.rows[5][0])] = False
    Z[5, outside] = -INF                                         # everything else masked
    Z[6, outside] = -300.0                                       # (other places than row 6's entries) far below
    Z[7, torch.tensor(p.rows[7][0])] += 200.0                    # the entries far above all others
    Z[8, torch.tensor(p.rows[8][0])] -= 200.0                    # ... and far below
    p.rows[9] = (np.full(5, -1), p.rows[9][1])                   # no entry
    p.rows[10] = (np.array([V, -5, 2 ** 31 - 1, -2 ** 31, 0]), p.rows[10][1])    # one entry
    p.rows[11] = (p.rows[11][0], np.full(5, -INF, dtype=np.float32))             # entries without a probability
    p.rows[12] = (p.rows[12][0], np.where(np.arange(5) < 2, -INF, p.rows[12][1]).astype(np.float32))
    p.rows[13] = (p.rows[13][0], np.full(5, -3e38, dtype=np.float32))
    if tail:
        p.tlse[11] = np.float32(0.0)
        p.tlse[13] = np.float32(0.0)
    p.set(Z.to(dtype))
    p.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", [False, True])
def test_infinities_and_nan_stay_in_their_rows(tail, dtype):
    p = Problem(8, 2003, 6, dtype, seed=4, tail=tail, weighted=False)
    Z = torch.tensor(p.host)
    Z[0, 100] = INF
    Z[1, 1999] = math.nan
    Z[2] = math.nan
    p.rows[3] = (p.rows[3][0], np.where(np.arange(6) == 2, math.nan, p.rows[3][1]).astype(np.float32))
    if tail:
        p.tlse[4] = np.float32(math.nan)
    p.set(Z.to(dtype))
    p.check()


def test_ignored_rows_may_hold_anything():
    comet = _comet()
    p = Problem(6, 1501, 4, torch.bfloat16, seed=6, tail=True, weighted=False)
    p.weight = np.array([0, 1, 0, 0.5, 2, 0], dtype=np.float32)
    Z = torch.tensor(p.host)
    Z[0], Z[2, 5], Z[5] = math.nan, INF, -INF
    p.tlse[0] = np.float32(math.nan)
    p.set(Z.to(torch.bfloat16))
    dZ = torch.full_like(p.Z, math.nan)
    loss, dZ = comet.comet_distill_step(p.Z, p.crd, p.tvals, dZ=dZ, **p.kw)
    torch.cuda.synchronize()
    for r in (0, 2, 5):
        assert float(loss[r]) == 0 and bool((dZ[r] == 0).all())
        p.host[r] = 0
    p.compare(loss, dZ)


def test_many_rows():
    Problem(700, 300, 12, torch.bfloat16, seed=7, tail=True).check()
    Problem(1500, 20, 3, torch.float32, seed=8, ragged=True).check()


def test_differences_of_the_loss():
    """The gradient against differences of the loss itself, along random directions."""
    comet = _comet()
    p = Problem(4, 501, 10, torch.float32, seed=9, tail=True, weighted=False, scale=0.5)
    loss, g = comet.comet_distill_step(p.Z, p.crd, p.tvals, **p.kw)
    gen = torch.Generator().manual_seed(1)
    for _ in range(3):
        d = torch.randn(p.Z.shape, generator=gen).cuda()
        h = 2.0 ** -5
        up = comet.comet_distill_forward(p.Z + h * d, p.crd, p.tvals, **p.kw)[0].double()
        down = comet.comet_distill_forward(p.Z - h * d, p.crd, p.tvals, **p.kw)[0].double()
        slope, want = (up - down) / (2 * h), (g.double() * d.double()).sum(1)
        # third derivatives of a log-sum-exp along d are below max|scale d|^3 = 2^3: h^2 / 6 * 8; and the losses' rounding over 2 h
        assert bool((slope - want).abs().max() <= h * h * 8 / 6 + (2.0 ** -22 * 4 + 6 * ref.sum_error(501)) / (2 * h))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_beyond_four_gib(dtype):
    comet = _comet()
    p = Problem(2, 5003, 20, dtype, seed=10, tail=True, weighted=False)
    ld = (5 << 30) // p.Z.element_size()
    flat = torch.empty(ld + 5003, dtype=dtype, device="cuda")
    Z = flat.as_strided((2, 5003), (ld, 1))
    Z.copy_(p.Z)
    loss, _ = comet.comet_distill_step(Z, p.crd, p.tvals, dZ=Z, **p.kw)
    torch.cuda.synchronize()
    p.compare(loss, Z)


def test_another_stream():
    comet = _comet()
    p = Problem(6, 20011, 30, torch.bfloat16, seed=11, tail=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, dZ = comet.comet_distill_step(p.Z, p.crd, p.tvals, stream=side, **p.kw)
    loss2, stat = comet.comet_distill_forward(p.Z, p.crd, p.tvals, stream=side, **p.kw)
    g = comet.comet_distill_backward(p.Z, p.crd, p.tvals, stat, stream=side, **p.kw)
    torch.cuda.synchronize()
    p.compare(loss, dZ)
    p.compare(loss2, g)


def test_same_bits_twice():
    comet = _comet()
    for N, V in ((3, 50021), (300, 5003)):
        p = Problem(N, V, 60, torch.bfloat16, seed=12, tail=True)
        a = comet.comet_distill_step(p.Z, p.crd, p.tvals, **p.kw)
        b = comet.comet_distill_step(p.Z, p.crd, p.tvals, **p.kw)
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_graph_replays():
    comet = _comet()
    p = Problem(5, 40009, 30, torch.bfloat16, seed=13, tail=True)
    loss, dZ = torch.empty(5, device="cuda"), torch.empty_like(p.Z)
    comet.comet_distill_step(p.Z, p.crd, p.tvals, loss=loss, dZ=dZ, **p.kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        comet.comet_distill_step(p.Z, p.crd, p.tvals, loss=loss, dZ=dZ, **p.kw)
    for seed in range(4):
        p.Z.copy_(Problem(5, 40009, 30, torch.bfloat16, seed=20 + seed).Z)
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), dZ.clone()
        eager = comet.comet_distill_step(p.Z, p.crd, p.tvals, **p.kw)
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])


def test_teacher_rows_from_the_top_logits():
    """What rows_topk writes is what the loss reads, places that are missing included."""
    comet = _comet()
    g = torch.Generator().manual_seed(14)
    teacher, student = (torch.randn((5, 37), generator=g).cuda() for _ in range(2))
    teacher[2, 3:] = -INF
    for K in (10, 37, 60):
        crd, vals, lse = comet.comet_rows_topk(teacher, K, scale=0.5)
        loss, _ = comet.comet_distill_forward(student, crd, vals, tlse=lse, scale=0.5)
        want = [ref.distill_row(student[r].double().cpu().numpy(), *ref.topk_row(teacher[r].cpu().numpy(), K),
                                ref.lse_row(teacher[r].double().cpu().numpy() * 0.5), 0.5, 1.0)[0] for r in range(5)]
        # tlse in 32 bits moves every log p by half a unit of about 4
        assert np.abs(loss.cpu().numpy() - want).max() <= 2.0 ** -20 + 3 * ref.sum_error(37)


def test_no_rows_and_no_columns():
    comet = _comet()
    loss, dZ = comet.comet_distill_step(torch.empty((0, 10), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"),
                                        torch.empty((0, 3), device="cuda"))
    assert loss.shape == (0,) and dZ.shape == (0, 10)
    loss, dZ = comet.comet_distill_step(torch.empty((2, 0), device="cuda"), torch.full((2, 3), -1, dtype=torch.int32, device="cuda"),
                                        torch.zeros((2, 3), device="cuda"))
    torch.cuda.synchronize()
    assert loss.tolist() == [0.0, 0.0] and dZ.shape == (2, 0)


def test_refusals():
    comet = _comet()
    p = Problem(4, 100, 3, torch.float32)
    Z, c, t, kw = p.Z, p.crd, p.tvals, p.kw
    ones = torch.ones(4, device="cuda")
    for bad, error in ((lambda: comet.comet_distill_step(Z, c, t, scale=-1.0), comet.CometError),
                       (lambda: comet.comet_distill_step(Z, c, t, scale=math.inf), comet.CometError),
                       (lambda: comet.comet_distill_step(Z.double(), c, t), TypeError), (lambda: comet.comet_distill_step(Z.t(), c, t), ValueError),
                       (lambda: comet.comet_distill_step(Z, c.long(), t), TypeError), (lambda: comet.comet_distill_step(Z, c, t[:, :2]), ValueError),
                       (lambda: comet.comet_distill_step(Z, c.reshape(-1), t.reshape(-1)), ValueError),
                       (lambda: comet.comet_distill_step(Z, c, t, pos=torch.zeros(5, dtype=torch.int32, device="cuda")), ValueError),
                       (lambda: comet.comet_distill_step(Z, c, t, weight=ones[:3]), ValueError), (lambda: comet.comet_distill_step(Z, c, t, tlse=ones.double()), TypeError),
                       (lambda: comet.comet_distill_step(Z, c, t, dZ=torch.empty((4, 99), device="cuda")), ValueError),
                       (lambda: comet.comet_distill_step(Z, c, t, dZ=torch.empty((4, 100), dtype=torch.bfloat16, device="cuda")), ValueError),
                       (lambda: comet.comet_distill_backward(Z, c, t, torch.zeros((4, 4), dtype=torch.float64, device="cuda")), ValueError)):
        with pytest.raises(error):
            bad()
