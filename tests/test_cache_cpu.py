"""What the entry points of the operators over a cache in blocks refuse, before they touch a device (CPU only)."""
import ctypes
import math

import pytest
import torch

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 3, 4
P = ctypes.c_void_p(4096)                 # a pointer that no refused call reads
ODD4, ODD2 = ctypes.c_void_p(4098), ctypes.c_void_p(4097)


@pytest.fixture(scope="module")
def lib():
    from paper_2102_05187_amd import binding, build
    build.build_if_missing()
    return binding._lib()


def cache(keys=4096, values=4096, mean=4096, type=1, blocks=10, block=16, heads=2, size=64, ks=(2048, 128, 64), vs=(2048, 128, 64), ms=(128, 64)):
    from paper_2102_05187_amd import binding
    c = binding._Cache(keys, values, mean, type, blocks, block, heads, size)
    c.key_stride[:], c.value_stride[:], c.mean_stride[:] = ks, vs, ms
    return ctypes.byref(c)


def two(a, b):
    return (ctypes.c_int64 * 2)(a, b)


def cache_map(lib, B=2, M=4, block=16, add=P, ended=None, length=P, held=P, table=P, ldt=4, spare=P, S=8, count=P, N=5, pos=P, slot=P, place=P, work=P, size=1 << 40):
    return lib.comet_cache_map(B, M, block, add, ended, length, held, table, ldt, spare, S, count, N, pos, slot, place, work, size, None)


def test_map(lib):
    need = ctypes.c_int64(-1)
    assert lib.comet_cache_map_work(2, 4, 5000, ctypes.byref(need)) == OK and need.value > 0
    assert lib.comet_cache_map_work(2, 4, 5, None) == INVALID
    for kw, status in ((dict(B=-1), INVALID), (dict(M=-1), INVALID), (dict(N=-1), INVALID), (dict(S=-1), INVALID), (dict(block=0), INVALID), (dict(block=1025), UNSUPPORTED),
                       (dict(ldt=3), SHAPE), (dict(ldt=1 << 41), UNSUPPORTED), (dict(B=(1 << 20) + 1), UNSUPPORTED), (dict(M=1 << 31, ldt=1 << 31), UNSUPPORTED),
                       (dict(M=1 << 27, ldt=1 << 27), UNSUPPORTED), (dict(S=1 << 31), UNSUPPORTED), (dict(N=1 << 31), UNSUPPORTED),
                       (dict(B=1 << 20, M=1 << 20, ldt=1 << 20), UNSUPPORTED), (dict(add=None), INVALID), (dict(length=None), INVALID), (dict(held=None), INVALID),
                       (dict(table=None), INVALID), (dict(spare=None), INVALID), (dict(count=None), INVALID), (dict(pos=None), INVALID), (dict(slot=None), INVALID),
                       (dict(place=None), INVALID), (dict(add=ODD4), INVALID), (dict(slot=ctypes.c_void_p(4100)), INVALID), (dict(table=ODD4), INVALID),
                       (dict(N=5000, work=None), INVALID), (dict(N=5000, size=need.value - 1), INVALID), (dict(N=5000, work=ctypes.c_void_p(4104)), INVALID)):
        assert cache_map(lib, **kw) == status, kw


CACHES = [(dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(blocks=-1), INVALID), (dict(block=0), INVALID), (dict(block=8), UNSUPPORTED), (dict(block=24), UNSUPPORTED),
          (dict(block=1040), UNSUPPORTED), (dict(heads=0), INVALID), (dict(heads=65537), UNSUPPORTED), (dict(size=0), INVALID), (dict(size=60), UNSUPPORTED),
          (dict(size=264), UNSUPPORTED), (dict(blocks=1 << 31), UNSUPPORTED)]
DATA = [(dict(keys=None), INVALID), (dict(values=None), INVALID), (dict(keys=4104), INVALID), (dict(values=4097), INVALID), (dict(ks=(2048, 128, 60)), INVALID),
        (dict(vs=(-2048, 128, 64)), INVALID), (dict(type=0, vs=(2048, 126, 64)), INVALID), (dict(ks=(1 << 41, 128, 64)), UNSUPPORTED)]
MEAN = [(dict(mean=4104), INVALID), (dict(ms=(128, 60)), INVALID), (dict(ms=(1 << 41, 64)), UNSUPPORTED)]


def write(lib, c=None, N=3, k=P, ks=(128, 64), v=P, vs=(128, 64), slot=P):
    return lib.comet_cache_write(c or cache(), N, k, two(*ks), v, two(*vs), slot, None)


def test_write(lib):
    for kw, status in CACHES + DATA + MEAN:
        assert write(lib, c=cache(**kw)) == status, kw
    assert lib.comet_cache_write(None, 3, P, two(128, 64), P, two(128, 64), P, None) == INVALID
    for kw, status in ((dict(N=-1), INVALID), (dict(N=1 << 31), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slot=None), INVALID),
                       (dict(k=ctypes.c_void_p(4104)), INVALID), (dict(slot=ctypes.c_void_p(4100)), INVALID), (dict(ks=(129, 64)), INVALID), (dict(N=0), OK)):
        assert write(lib, **kw) == status, kw


def select(lib, c=None, N=3, Q=4, q=P, qs=(256, 64), B=2, pos=P, length=P, table=P, M=9, ldt=9, K=5, first=1, last=1, sel=P, work=P, size=1 << 40):
    return lib.comet_block_select(c or cache(), N, Q, q, two(*qs), B, pos, length, table, M, ldt, K, first, last, sel, work, size, None)


QUERIES = [(dict(N=-1), INVALID), (dict(Q=0), INVALID), (dict(Q=3), SHAPE), (dict(B=-1), INVALID), (dict(M=-1), INVALID), (dict(K=0), INVALID), (dict(K=1025), UNSUPPORTED),
           (dict(N=(1 << 23) + 1), UNSUPPORTED), (dict(Q=65538), UNSUPPORTED), (dict(N=1 << 22, Q=512), UNSUPPORTED), (dict(ldt=8), SHAPE), (dict(ldt=1 << 41), UNSUPPORTED),
           (dict(q=None), INVALID), (dict(q=ctypes.c_void_p(4104)), INVALID), (dict(qs=(250, 64)), INVALID), (dict(qs=(-256, 64)), INVALID), (dict(pos=None), INVALID),
           (dict(length=None), INVALID), (dict(table=None), INVALID), (dict(pos=ODD4), INVALID), (dict(sel=None), INVALID), (dict(sel=ODD4), INVALID), (dict(N=0), OK)]


def test_select(lib):
    for kw, status in CACHES + MEAN + [(dict(mean=None), INVALID)]:
        assert select(lib, c=cache(**kw)) == status, kw
    for kw, status in QUERIES + [(dict(first=-1), INVALID), (dict(last=0), INVALID), (dict(first=3, last=3), INVALID), (dict(M=16385, ldt=16385), UNSUPPORTED), (dict(B=0), OK)]:
        assert select(lib, **kw) == status, kw
    need = ctypes.c_int64(-1)
    assert lib.comet_block_select_work(cache(), 3, 4, 2, 9, 5, None) == INVALID
    assert lib.comet_block_select_work(cache(), 3, 4, 2, 9, 5, ctypes.byref(need)) == OK and need.value >= 0
    assert lib.comet_block_select_work(cache(), 3, 4, 2, 16385, 5, ctypes.byref(need)) == UNSUPPORTED


def attend(lib, c=None, N=3, Q=4, q=P, qs=(256, 64), B=2, pos=P, length=P, table=P, M=9, ldt=9, sel=P, K=5, scale=0.125, out=P, lse=P, work=P, size=1 << 40):
    return lib.comet_block_attend(c or cache(), N, Q, q, two(*qs), B, pos, length, table, M, ldt, sel, K, scale, out, lse, work, size, None)


def test_attend(lib):
    for kw, status in CACHES + DATA:
        assert attend(lib, c=cache(**kw)) == status, kw
    for kw, status in QUERIES + [(dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
                                 (dict(scale=1e-60), INVALID), (dict(scale=1e39), INVALID), (dict(out=None), INVALID), (dict(out=ctypes.c_void_p(4104)), INVALID),
                                 (dict(lse=ODD4), INVALID), (dict(M=262145, ldt=262145), UNSUPPORTED), (dict(B=0), OK)]:
        assert attend(lib, **kw) == status, kw
    need = ctypes.c_int64(-1)
    assert lib.comet_block_attend_work(cache(), 3, 4, 2, 9, 5, None) == INVALID
    assert lib.comet_block_attend_work(cache(), 3, 4, 2, 9, 5, ctypes.byref(need)) == OK and need.value >= 0


def verify(lib, Z=P, kind=1, N=5, V=100, ld=100, B=2, pos=P, token=P, u=P, v=P, draft=None, dkind=1, ldd=100, crd=None, vals=None, K=0, scale=1.0, scales=None,
           accepted=P, follow=P, length=None, work=P, size=1 << 40):
    return lib.comet_draft_verify(Z, kind, N, V, ld, B, pos, token, u, v, draft, dkind, ldd, crd, vals, K, scale, scales, accepted, follow, length, work, size, None)


def test_verify(lib):
    need = ctypes.c_int64(-1)
    assert lib.comet_draft_verify_work(1, 5, 100, 2, 0, 0, ctypes.byref(need)) == OK and need.value > 0
    assert lib.comet_draft_verify_work(1, 5, 100, 2, 0, 0, None) == INVALID
    for kw, status in ((dict(Z=None), INVALID), (dict(kind=3), INVALID), (dict(N=-1), INVALID), (dict(V=-1), INVALID), (dict(B=-1), INVALID), (dict(K=-1), INVALID),
                       (dict(K=1025, crd=P, vals=P), UNSUPPORTED), (dict(K=4), INVALID), (dict(K=4, crd=P), INVALID), (dict(draft=P, K=4, crd=P, vals=P), INVALID),
                       (dict(draft=P, dkind=5), INVALID), (dict(draft=P, ldd=99), SHAPE), (dict(ld=99), SHAPE), (dict(ld=1 << 41), UNSUPPORTED),
                       (dict(N=(1 << 23) + 1), UNSUPPORTED), (dict(V=1 << 31, ld=1 << 31), UNSUPPORTED), (dict(N=1 << 20, V=1 << 30, ld=1 << 30), UNSUPPORTED),
                       (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(pos=None), INVALID), (dict(token=None), INVALID),
                       (dict(u=None), INVALID), (dict(v=None), INVALID), (dict(accepted=None), INVALID), (dict(follow=None), INVALID), (dict(Z=ODD2), INVALID),
                       (dict(draft=ODD4, dkind=0), INVALID), (dict(u=ODD4), INVALID), (dict(scales=ODD4), INVALID), (dict(length=ODD4), INVALID), (dict(work=None), INVALID),
                       (dict(size=need.value - 1), INVALID), (dict(work=ctypes.c_void_p(4104)), INVALID), (dict(B=0), OK)):
        assert verify(lib, **kw) == status, kw


def test_the_binding_refuses_host_tensors():
    import paper_2102_05187_amd as comet
    i, x = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 16, 1, 64))
    q, row = torch.zeros((2, 1, 64)), torch.zeros((2, 10))
    pos, sel = torch.zeros(3, dtype=torch.int32), torch.zeros((2, 1, 1), dtype=torch.int32)
    for call in (lambda: comet.comet_cache_map(i, i, i, i[:, None], i, i[:1], 16, 4), lambda: comet.comet_cache_write(q, q, x, x, i.long()),
                 lambda: comet.comet_block_select(q, q, i[:, None], pos, i, 16, 2), lambda: comet.comet_block_attend(q, x, x, i[:, None], pos, i, sel),
                 lambda: comet.comet_draft_verify(row, i, pos, row[:, 0], row[:, 0])):
        with pytest.raises(TypeError):
            call()
