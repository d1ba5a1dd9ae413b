"""The K largest elements of dense rows, against a stable sort in 64 bits."""
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


def matrix(N, V, dtype, seed=0, ld=None, start=0, scale=3.0):
    """N rows of V logits that lie `ld` apart, the first one `start` elements into its memory."""
    g = torch.Generator().manual_seed(seed)
    ld = ld or V
    flat = (torch.randn(start + max(1, N) * ld, generator=g) * scale).to(dtype)
    flat = flat.cuda()
    return flat[start:start + max(1, N) * ld].view(max(1, N), ld)[:N, :V]


def check(Z, K, scale=1.0, by_coordinate=False, stream=None):
    comet = _comet()
    crd, vals, lse = comet.comet_rows_topk(Z, K, scale=scale, by_coordinate=by_coordinate, stream=stream)
    torch.cuda.synchronize()
    assert crd.dtype == torch.int32 and vals.dtype == torch.float32 and lse.dtype == torch.float32
    host = Z.double().cpu().numpy()
    for r in range(Z.shape[0]):
        c, v = ref.topk_row(host[r], K, by_coordinate)
        assert crd[r].tolist() == c, "row %d" % r
        assert vals[r].tolist() == v, "row %d" % r
        want, got = ref.lse_row(host[r] * scale), float(lse[r])
        if math.isfinite(want):
            bound = 2.0 ** -24 * abs(want) + ref.sum_error(Z.shape[1])
            assert abs(got - want) <= bound, (r, got, want)
        else:
            assert got == want or (math.isnan(want) and math.isnan(got)), (r, got, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("by_coordinate", [False, True])
@pytest.mark.parametrize("N,V,K", [(1, 1, 1), (2, 2, 1), (3, 7, 3), (2, 8, 8), (3, 63, 5), (2, 64, 64), (3, 65, 7), (2, 255, 100), (2, 1000, 1000),
                                   (3, 1000, 999), (2, 1024, 1024), (3, 2049, 50), (5, 4099, 1), (4, 5003, 64), (2, 5003, 1024), (2, 8192, 512),
                                   (2, 16411, 300), (3, 32003, 50), (1, 70001, 64), (1, 131072, 500), (1, 140001, 1024)])
def test_sizes(N, V, K, by_coordinate, dtype):
    check(matrix(N, V, dtype, seed=N * V + K), K, by_coordinate=by_coordinate)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1024, 1025, 2048, 2056, 8191, 16384, 16385, 32768, 32769, 65536, 65537, 131073, 262145])
def test_around_the_sizes_of_pieces(V, dtype):
    check(matrix(2, V, dtype, seed=V), 17)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_rows(dtype):
    check(matrix(2, 524288, dtype, seed=1), 1024, by_coordinate=True)
    check(matrix(1, 3000001, dtype, seed=2), 100)


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_kept_than_there_are(dtype):
    check(matrix(3, 5, dtype), 9)
    check(matrix(3, 5, dtype), 9, by_coordinate=True)
    check(matrix(2, 100, dtype), 1024)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("start", [0, 1, 3, 5, 7])
@pytest.mark.parametrize("ld", [1001, 1003, 1008, 1500])
def test_rows_anywhere(ld, start, dtype):
    check(matrix(5, 1001, dtype, seed=ld + start, ld=ld, start=start), 33, scale=0.4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 50, 3001, 40009, 131072])
@pytest.mark.parametrize("K", [1, 20, 700])
def test_rows_of_every_kind(V, K, dtype):
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(V + K)
    rows = [torch.full((V,), -INF),                                      # nothing is left
            torch.full((V,), low),                                       # masked by the lowest value throughout
            torch.zeros(V),                                              # all equal
            torch.full((V,), -0.0),
            torch.arange(V) % 97 * 1.0,                                  # many equal ones
            torch.arange(V) * (60000.0 / V),                             # the largest last
            torch.arange(V, 0, -1) * (60000.0 / V),                      # the largest first
            torch.randn(V, generator=g) * 3,
            torch.randn(V, generator=g) * 1e-4 + 11,                     # close together
            torch.where(torch.arange(V) % 256 < 3, torch.randn(V, generator=g) + 9, torch.randn(V, generator=g))]
    some = torch.full((V,), -INF)
    some[::max(1, V // 7)] = torch.randn(some[::max(1, V // 7)].shape, generator=g)
    rows.append(some)                                                    # a handful is left
    lowest = torch.full((V,), low)
    lowest[V // 2] = 1.5
    rows.append(lowest)                                                  # one is left, by the lowest value
    far = torch.randn(V, generator=g)
    far[V // 3] = 40000.0
    rows.append(far)
    block = torch.randn(V, generator=g)
    block[V // 2:V // 2 + 1500] += 50                                    # the largest ones next to each other
    rows.append(block)
    check(torch.stack(rows).to(dtype).cuda(), K)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [9, 2000, 50021])
def test_infinities_and_nan(V, dtype):
    g = torch.Generator().manual_seed(V)
    Z = torch.randn((5, V), generator=g)
    Z[0, V // 2] = INF
    Z[1, V // 3] = math.nan
    Z[2] = math.nan
    Z[3, 1:] = -INF
    Z[3, V - 1] = math.nan
    check(Z.to(dtype).cuda(), 4)


@pytest.mark.parametrize("scale", [0.25, 1.0, 3.0])
def test_scale(scale):
    check(matrix(4, 3001, torch.float32, seed=3), 10, scale=scale)


def test_many_rows():
    check(matrix(700, 300, torch.bfloat16, seed=5), 12)
    check(matrix(2000, 33, torch.float16, seed=6), 5, by_coordinate=True)


def test_no_rows_and_no_columns():
    comet = _comet()
    crd, vals, lse = comet.comet_rows_topk(torch.empty((0, 10), device="cuda"), 3)
    assert crd.shape == (0, 3) and lse.shape == (0,)
    crd, vals, lse = comet.comet_rows_topk(torch.empty((2, 0), device="cuda"), 3)
    assert crd.tolist() == [[-1] * 3] * 2 and vals.tolist() == [[-INF] * 3] * 2 and lse.tolist() == [-INF] * 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_beyond_four_gib(dtype):
    """The second row begins more than 2^32 bytes (and 2^31 elements in 16 bits) behind the first."""
    size = torch.empty(0, dtype=dtype).element_size()
    ld = (5 << 30) // size
    flat = torch.empty(ld + 5003, dtype=dtype, device="cuda")
    Z = flat.as_strided((2, 5003), (ld, 1))
    Z.copy_(matrix(2, 5003, dtype, seed=9))
    check(Z, 40)


def test_another_stream_and_given_results():
    comet = _comet()
    Z = matrix(6, 20011, torch.bfloat16, seed=11)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    check(Z, 64, stream=side)
    crd, vals, lse = (torch.full((6, 64), 7, dtype=torch.int32, device="cuda"), torch.zeros((6, 64), device="cuda"), torch.zeros(6, device="cuda"))
    out = comet.comet_rows_topk(Z, 64, crd=crd, vals=vals, lse=lse)
    again = comet.comet_rows_topk(Z, 64)
    torch.cuda.synchronize()
    assert out[0] is crd and all(torch.equal(a, b) for a, b in zip(out, again))


def test_graph_replays():
    comet = _comet()
    Z = matrix(3, 40009, torch.bfloat16, seed=12)
    out = [torch.empty((3, 50), dtype=torch.int32, device="cuda"), torch.empty((3, 50), device="cuda"), torch.empty(3, device="cuda")]
    comet.comet_rows_topk(Z, 50, crd=out[0], vals=out[1], lse=out[2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        comet.comet_rows_topk(Z, 50, crd=out[0], vals=out[1], lse=out[2])
    for seed in range(4):
        Z.copy_(matrix(3, 40009, torch.bfloat16, seed=20 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        eager = comet.comet_rows_topk(Z, 50)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_kept_entries_are_a_matrix_of_the_library():
    """By coordinate, crd and vals are the compressed level of a [D,CU] matrix: its product with a dense one."""
    comet = _comet()
    Z = matrix(50, 301, torch.float32, seed=13)
    crd, vals, _ = comet.comet_rows_topk(Z, 8, by_coordinate=True)
    pos = torch.arange(51, dtype=torch.int32, device="cuda") * 8
    A = comet.comet_tensor_create([50, 301], [comet.COMET_D, comet.COMET_CU], [torch.tensor([50], dtype=torch.int32, device="cuda"), pos],
                                  [None, crd.reshape(-1)], vals.double().reshape(-1))
    x = torch.randn((301, 4), dtype=torch.float64, device="cuda")
    dense = torch.zeros((50, 301), dtype=torch.float64, device="cuda").scatter_(1, crd.long(), vals.double())
    assert torch.allclose(comet.comet_spmm(A, x), dense @ x, rtol=1e-12, atol=1e-12)


def test_refusals():
    comet = _comet()
    Z = matrix(4, 100, torch.float32)
    for bad, error in ((lambda: comet.comet_rows_topk(Z, 0), comet.CometError), (lambda: comet.comet_rows_topk(Z, 1025), comet.CometError),
                       (lambda: comet.comet_rows_topk(Z, 3, scale=0.0), comet.CometError),
                       (lambda: comet.comet_rows_topk(torch.empty((1, 1 << 20), device="cuda"), 513), comet.CometError),
                       (lambda: comet.comet_rows_topk(Z, 3, scale=math.nan), comet.CometError),
                       (lambda: comet.comet_rows_topk(Z.double(), 3), TypeError), (lambda: comet.comet_rows_topk(Z.cpu(), 3), TypeError),
                       (lambda: comet.comet_rows_topk(Z.t(), 3), ValueError), (lambda: comet.comet_rows_topk(Z[0], 3), ValueError),
                       (lambda: comet.comet_rows_topk(Z[:1].expand(4, 100), 3), ValueError),
                       (lambda: comet.comet_rows_topk(Z, 3, crd=torch.empty((4, 2), dtype=torch.int32, device="cuda")), ValueError),
                       (lambda: comet.comet_rows_topk(Z, 3, vals=torch.empty((4, 3), dtype=torch.float64, device="cuda")), TypeError)):
        with pytest.raises(error):
            bad()
