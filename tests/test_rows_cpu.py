"""What the entry points of the operators on dense rows refuse, before they touch a device (CPU only)."""
import ctypes
import math

import pytest

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 3, 4
P = ctypes.c_void_p(4096)                 # a pointer that no refused call reads


@pytest.fixture(scope="module")
def lib():
    from paper_2102_05187_amd import binding, build
    build.build_if_missing()
    return binding._lib()


def topk(lib, Z=P, kind=1, N=4, V=100, ld=100, scale=1.0, K=5, flags=0, crd=P, vals=P, lse=P, work=P, size=1 << 40):
    return lib.comet_rows_topk(Z, kind, N, V, ld, scale, K, flags, crd, vals, lse, work, size, None)


def test_topk(lib):
    for kw, status in ((dict(Z=None), INVALID), (dict(kind=3), INVALID), (dict(N=-1), INVALID), (dict(V=-1), INVALID), (dict(ld=99), SHAPE),
                       (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID),
                       (dict(scale=1e-60), INVALID), (dict(scale=1e39), INVALID), (dict(K=0), INVALID), (dict(K=1025), UNSUPPORTED), (dict(flags=2), INVALID),
                       (dict(crd=None), INVALID), (dict(vals=None), INVALID), (dict(V=1 << 31, ld=1 << 31), UNSUPPORTED), (dict(N=(1 << 23) + 1), UNSUPPORTED),
                       (dict(ld=1 << 41), UNSUPPORTED), (dict(Z=ctypes.c_void_p(4097)), INVALID), (dict(kind=0, Z=ctypes.c_void_p(4098)), INVALID),
                       (dict(crd=ctypes.c_void_p(4098)), INVALID), (dict(lse=ctypes.c_void_p(4097)), INVALID), (dict(N=0), OK)):
        assert topk(lib, **kw) == status, kw
    need = ctypes.c_int64(-1)
    assert lib.comet_rows_topk_work(1, 4, 100, 5, None) == INVALID
    assert lib.comet_rows_topk_work(7, 4, 100, 5, ctypes.byref(need)) == INVALID
    assert lib.comet_rows_topk_work(1, 4, 100, 2000, ctypes.byref(need)) == UNSUPPORTED
    assert lib.comet_rows_topk_work(1, 4, 100, 5, ctypes.byref(need)) == OK and need.value >= 0


def distill(lib, which, Z=P, kind=1, N=4, V=100, ld=100, pos=None, K=5, crd=P, tvals=P, tlse=None, scale=1.0, weight=None, loss=P, stat=P, dloss=None,
            dZ=P, ldd=100, work=P, size=1 << 40):
    args = (Z, kind, N, V, ld, pos, K, crd, tvals, tlse, scale, weight)
    if which == "forward":
        return lib.comet_distill_forward(*args, loss, stat, work, size, None)
    if which == "backward":
        return lib.comet_distill_backward(*args, stat, dloss, dZ, ldd, None)
    return lib.comet_distill_step(*args, loss, dZ, ldd, work, size, None)


@pytest.mark.parametrize("which", ["forward", "backward", "step"])
def test_distill(lib, which):
    cases = [(dict(Z=None), INVALID), (dict(kind=9), INVALID), (dict(N=-1), INVALID), (dict(V=-2), INVALID), (dict(ld=99), SHAPE), (dict(scale=0.0), INVALID),
             (dict(scale=math.nan), INVALID), (dict(K=-1), INVALID), (dict(crd=None), INVALID), (dict(tvals=None), INVALID),
             (dict(tvals=ctypes.c_void_p(4098)), INVALID), (dict(pos=ctypes.c_void_p(4098)), INVALID), (dict(weight=ctypes.c_void_p(4097)), INVALID),
             (dict(V=1 << 31, ld=1 << 31, ldd=1 << 31), UNSUPPORTED), (dict(N=0), OK)]
    if which != "backward":
        cases += [(dict(loss=None), INVALID)]
    if which != "step":
        cases += [(dict(stat=None), INVALID), (dict(stat=ctypes.c_void_p(4100)), INVALID)]
    if which != "forward":
        cases += [(dict(dZ=None), INVALID), (dict(ldd=99), SHAPE), (dict(dZ=ctypes.c_void_p(4097)), INVALID), (dict(dZ=P, ldd=120), INVALID)]
    if which == "step":
        need = ctypes.c_int64(-1)
        long = dict(V=1 << 20, ld=1 << 20, ldd=1 << 20)          # rows that no workgroup holds
        assert lib.comet_distill_work(1, 4, 1 << 20, ctypes.byref(need)) == OK and need.value > 0
        cases += [(dict(long, work=None), INVALID), (dict(long, size=need.value - 1), INVALID), (dict(long, work=ctypes.c_void_p(4104)), INVALID)]
    for kw, status in cases:
        assert distill(lib, which, **kw) == status, kw


def select(lib, Z=P, kind=1, B=2, W=3, V=100, ld=100, score=P, finished=None, eos=0, n=6, a=P, b=P, c=P, work=P, size=1 << 40):
    return lib.comet_beam_select(Z, kind, B, W, V, ld, score, finished, eos, n, a, b, c, work, size, None)


def test_select(lib):
    need = ctypes.c_int64(-1)
    assert lib.comet_beam_select_work(1, 2, 3, 100, 6, ctypes.byref(need)) == OK and need.value > 0
    for kw, status in ((dict(Z=None), INVALID), (dict(kind=-1), INVALID), (dict(B=-1), INVALID), (dict(W=0), INVALID), (dict(n=0), INVALID),
                       (dict(W=257), UNSUPPORTED), (dict(n=1025), UNSUPPORTED), (dict(W=16, n=513), UNSUPPORTED), (dict(V=1 << 24, ld=1 << 24), UNSUPPORTED),
                       (dict(ld=99), SHAPE), (dict(score=None), INVALID), (dict(a=None), INVALID), (dict(b=None), INVALID), (dict(c=None), INVALID),
                       (dict(finished=P, eos=100), INVALID), (dict(finished=P, eos=-1), INVALID), (dict(work=None), INVALID),
                       (dict(size=need.value - 1), INVALID), (dict(score=ctypes.c_void_p(4098)), INVALID), (dict(B=0), OK)):
        assert select(lib, **kw) == status, kw


def reorder(lib, states=(4096, 8192), B=2, W=3, batch=300, beam=100, outer=1, ostride=0, inner=100, parent=P, n=None):
    ptrs = None if states is None else (ctypes.c_void_p * len(states))(*states)
    return lib.comet_beam_reorder(ptrs, (0 if states is None else len(states)) if n is None else n, B, W, batch, beam, outer, ostride, inner, parent, None)


def test_reorder(lib):
    for kw, status in ((dict(states=None, n=1), INVALID), (dict(states=(4096, None)), INVALID), (dict(B=-1), INVALID), (dict(W=0), INVALID),
                       (dict(W=257), UNSUPPORTED), (dict(outer=-1), INVALID), (dict(inner=-1), INVALID), (dict(parent=None), INVALID),
                       (dict(parent=ctypes.c_void_p(4098)), INVALID), (dict(beam=99), INVALID), (dict(beam=0), INVALID), (dict(batch=299), INVALID),
                       (dict(batch=-300), INVALID), (dict(outer=2, ostride=49, inner=50), INVALID), (dict(outer=3, ostride=50, beam=150, batch=600), INVALID),
                       (dict(outer=1 << 40, ostride=1 << 40), INVALID), (dict(states=()), OK), (dict(B=0), OK), (dict(inner=0), OK), (dict(outer=0), OK)):
        assert reorder(lib, **kw) == status, kw
