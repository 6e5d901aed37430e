"""Tokens sorted by expert and back against plain 64-bit implementations."""
import numpy as np
import pytest

from tests.block_reference import SMALLEST, U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


@pytest.fixture(scope="module")
def ccdc():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_1805_01993_b200 import build, ccdc as mod

    build.build_library()
    mod.lib()
    return mod


def order_of(ids, E):
    """(offsets, slots, places) by the definition"""
    flat = np.asarray(ids).reshape(-1)
    inside = [s for s in range(flat.size) if 0 <= flat[s] < E]
    by = sorted(inside, key=lambda s: flat[s])          # stable
    slots, places = np.full(flat.size, -1), np.full(flat.size, -1)
    slots[:len(by)] = by
    places[by] = np.arange(len(by))
    below = np.searchsorted(np.sort(flat[inside]), np.arange(E + 1))        # slots of experts below each
    return below, slots, places.reshape(np.shape(ids))


def draw_ids(rng, M, k, E, drop=0.0):
    ids = rng.integers(0, E, (M, k))
    ids[rng.random((M, k)) < drop] = -1
    return ids


def rows_of(rng, rows, cols, dtype, pad=0, shift=0):
    flat = torch.from_numpy(rng.normal(size=rows * (cols + pad) + shift)).to(DT[dtype]).cuda()
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def f64(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------- the sort
# one warp's slots, a block's, a cluster's (more than 4096 slots); experts at and beyond the warps' number and at the limit
@pytest.mark.parametrize("M,k,E,drop", [(1, 1, 1, 0), (1, 8, 128, 0), (5, 3, 2, 0.5), (32, 1, 4, 0), (33, 2, 33, 0.1), (100, 7, 1000, 0),
                                        (1024, 4, 1025, 0.2), (1025, 4, 64, 0.1), (2049, 3, 7, 0.9), (3001, 5, 4096, 0.1), (700, 6, 1, 0),
                                        (300, 16, 1024, 1.0), (20001, 2, 100, 0.1), (9000, 4, 4096, 0.3)])
@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_sort(ccdc, M, k, E, drop, kind):
    ids = draw_ids(np.random.default_rng(M + E), M, k, E, drop)
    got = ccdc.expert_sort(torch.from_numpy(ids).to(kind).cuda(), E)
    for name, a, b in zip(got._fields, got, order_of(ids, E)):
        assert a.dtype is torch.int32 and np.array_equal(a.cpu().numpy(), b), name


def test_sort_of_ids_that_are_none(ccdc):
    """ids outside the range are dropped, 64-bit ones whose low words look like experts too"""
    ids = torch.tensor([[5, -1, 0], [(1 << 32) + 1, -(1 << 32), 1 << 62], [4, 3, 1]], dtype=torch.int64)
    got = ccdc.expert_sort(ids.cuda(), 5)
    for a, b in zip(got, order_of(ids.numpy(), 5)):
        assert np.array_equal(a.cpu().numpy(), b)
    none = ccdc.expert_sort(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 6)
    assert none.offsets.tolist() == [0] * 7 and none.slots.numel() == 0 and none.places.shape == (0, 4)
    same = ccdc.expert_sort(torch.full((3000, 2), 3, dtype=torch.int32, device="cuda"), 5)       # one expert takes all, twice
    assert same.offsets.tolist() == [0, 0, 0, 0, 6000, 6000] and same.slots.tolist() == list(range(6000))


# ---------------------------------------------------------------- there and back
SHAPES = [(1, 1, 1, 1, 0.0, 0, 0), (1, 8, 16, 4096, 0.0, 0, 0), (3, 2, 4, 8, 0.0, 0, 0), (7, 3, 5, 33, 0.3, 1, 1), (40, 8, 20, 264, 0.2, 8, 8),
          (129, 5, 3, 1001, 0.5, 5, 0), (20, 17, 30, 2056, 0.1, 0, 0), (64, 1, 7, 5000, 0.0, 0, 0), (9, 4, 6, 24, 1.0, 0, 0)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("own_weights", [False, True])
@pytest.mark.parametrize("M,k,E,D,drop,pad,shift", SHAPES)
def test_there_and_back(ccdc, M, k, E, D, drop, pad, shift, own_weights, dtype):
    rng = np.random.default_rng(M * 31 + D)
    ids = draw_ids(rng, M, k, E, drop)
    order = ccdc.expert_sort(torch.from_numpy(ids).cuda(), E)
    _, slots, places = order_of(ids, E)
    n = int((slots >= 0).sum())
    x, dy = (rows_of(rng, M, D, dtype, pad, shift) for _ in range(2))
    ys, dxs = (rows_of(rng, M * k, D, dtype, pad, shift) for _ in range(2))
    ys[n:], dxs[n:] = float("nan"), float("nan")        # what lies behind the last expert's rows is not read
    wt = DT[dtype] if own_weights else torch.float32
    w = torch.from_numpy(rng.random((M, k))).to(wt).cuda()
    xs = ccdc.expert_dispatch(x, order)
    want = np.zeros((M * k, D))
    want[:n] = f64(x)[slots[:n] // k]
    assert np.array_equal(f64(xs), want)
    u, tiny = U[dtype], SMALLEST[dtype]

    def back(rows, weights):
        total, size = np.zeros((M, D)), np.zeros((M, D))
        for m in range(M):
            for j in range(k):
                if places[m, j] >= 0:
                    term = weights[m, j] * rows[places[m, j]]
                    total[m] += term
                    size[m] += np.abs(term)
        return total, size

    # k products and sums in binary32, one rounding to the type
    for got, (want, size) in ((ccdc.expert_combine(ys, order, w), back(f64(ys), f64(w))),
                              (ccdc.expert_dispatch_backward(dxs, order), back(f64(dxs), np.ones((M, k))))):
        assert (np.abs(f64(got) - want) <= (k + 1) * 2.0 ** -24 * size * (1 + u) + u * np.abs(want) + tiny).all()
    dys, dw = ccdc.expert_combine_backward(dy, ys, order, w)
    want = np.zeros((M * k, D))
    want[:n] = f64(dy)[slots[:n] // k] * f64(w).reshape(-1)[slots[:n]][:, None]
    # the product is rounded to binary32 and then to the type
    assert (np.abs(f64(dys) - want) <= (u + 2.0 ** -24 * (1 + u)) * np.abs(want) + tiny).all() and not f64(dys)[n:].any()
    assert dw.dtype is wt
    want, size = np.zeros((M, k)), np.zeros((M, k))
    for m, j in zip(*np.nonzero(places >= 0)):
        terms = f64(dy)[m] * f64(ys)[places[m, j]]
        want[m, j], size[m, j] = terms.sum(), np.abs(terms).sum()
    uw, tw = (u, tiny) if own_weights else (2.0 ** -24, SMALLEST["float32"])
    # a lane adds ceil(D / 32) products rounded up to whole vectors of 8, then five sums join the lanes
    steps = -(-D // 256) * 8 + 5
    assert (np.abs(f64(dw) - want) <= steps * 2.0 ** -24 * size * (1 + uw) + uw * np.abs(want) + tw).all()
    # without weights: copies
    plain, none = ccdc.expert_combine_backward(dy, None, order, None)
    assert none is None and torch.equal(plain, ccdc.expert_dispatch(dy, order))


def test_into_given_tensors_only(ccdc):
    """outputs of any row stride, and nothing outside them is written"""
    rng = np.random.default_rng(3)
    M, k, D = 11, 3, 40
    order = ccdc.expert_sort(torch.from_numpy(draw_ids(rng, M, k, 4, 0.2)).cuda(), 4)
    x, ys = rows_of(rng, M, D, "bfloat16"), rows_of(rng, M * k, D, "bfloat16")
    w = torch.rand((M, k), device="cuda")
    for pad in (8, 3):
        big = [torch.full((r, D + pad), 7.0, dtype=torch.bfloat16, device="cuda") for r in (M * k, M, M * k)]
        a = ccdc.expert_dispatch(x, order, out=big[0][:, :D])
        b = ccdc.expert_combine(ys, order, w, out=big[1][:, :D])
        c, dw = ccdc.expert_combine_backward(x, ys, order, w, dys=big[2][:, :D], dweights=torch.empty_like(w))
        assert torch.equal(a, ccdc.expert_dispatch(x, order)) and torch.equal(b, ccdc.expert_combine(ys, order, w))
        assert torch.equal(c, ccdc.expert_combine_backward(x, ys, order, w)[0])
        assert all(bool((t[:, D:] == 7).all()) for t in big)
    given = [torch.full((n,), 9, dtype=torch.int32, device="cuda") for n in (5, M * k)] + [torch.zeros((M, k), dtype=torch.int32, device="cuda")]
    again = ccdc.expert_sort(order.places, 40, *given[:0])      # any integers are ids
    assert again.offsets.shape == (41,)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,k,D", [(5, 3, 40), (37, 2, 4096), (9, 1, 2048), (30, 5, 8)])
def test_rows_of_tokens_that_start_anywhere(ccdc, M, k, D, dtype):
    """the tokens' rows out of a padded batch, the sorted ones aligned: the bits of aligned tokens"""
    rng = np.random.default_rng(D)
    order = ccdc.expert_sort(torch.from_numpy(draw_ids(rng, M, k, 6, 0.1)).cuda(), 6)
    x, dy = (rows_of(rng, M, D, dtype, 5, 1) for _ in range(2))
    ys, w = rows_of(rng, M * k, D, dtype), torch.rand((M, k), device="cuda")
    assert torch.equal(ccdc.expert_dispatch(x, order), ccdc.expert_dispatch(x.contiguous(), order))
    for a, b in zip(ccdc.expert_combine_backward(dy, ys, order, w), ccdc.expert_combine_backward(dy.contiguous(), ys, order, w)):
        assert torch.equal(a, b)
    flat = torch.full((M * (D + 3) + 1,), 7.0, dtype=DT[dtype], device="cuda")
    out = ccdc.expert_combine(ys, order, w, out=flat[1:].view(M, D + 3)[:, :D])
    assert torch.equal(out, ccdc.expert_combine(ys, order, w))
    assert bool((flat[1:].view(M, D + 3)[:, D:] == 7).all()) and float(flat[0]) == 7


def test_infinities_and_nan(ccdc):
    """they stay in the tokens that they belong to"""
    order = ccdc.expert_sort(torch.tensor([[0, 1], [1, -1], [-1, -1]], device="cuda"), 2)
    ys = torch.ones((6, 16), device="cuda")
    ys[order.places[0, 1]] = float("inf")
    w = torch.ones((3, 2), device="cuda")
    w[1, 1] = w[2, 0] = float("nan")                    # weights of dropped slots are not read
    y = ccdc.expert_combine(ys, order, w)
    assert bool(y[0].isinf().all()) and bool((y[1] == 1).all()) and bool((y[2] == 0).all())
    dys, dw = ccdc.expert_combine_backward(torch.ones((3, 16), device="cuda"), ys, order, w)
    assert dw[0].tolist() == [16.0, float("inf")] and dw[1:].reshape(-1).tolist() == [16.0, 0, 0, 0] and bool(dys.isfinite().all())


def test_gradients_by_differences(ccdc):
    """combine's weights and rows, and the rows through dispatch, against central differences in binary32"""
    rng = np.random.default_rng(8)
    M, k, D, E = 6, 3, 12, 4
    order = ccdc.expert_sort(torch.from_numpy(draw_ids(rng, M, k, E, 0.2)).cuda(), E)
    x, g = rows_of(rng, M, D, "float32"), rows_of(rng, M, D, "float32")
    w = torch.from_numpy(rng.random((M, k))).float().cuda()

    def f(x, w):        # experts that square
        return float((ccdc.expert_combine(ccdc.expert_dispatch(x, order).square(), order, w).double() * g.double()).sum())

    xs = ccdc.expert_dispatch(x, order)
    dys, dw = ccdc.expert_combine_backward(g, xs.square(), order, w)
    dx = ccdc.expert_dispatch_backward(2 * xs * dys, order)
    for grad, at in ((dx, 0), (dw, 1)):
        d = torch.from_numpy(rng.normal(size=grad.shape)).float().cuda()
        h = 2.0 ** -6
        args = [x, w]
        up, down = (f(*[a + s * h * d if i == at else a for i, a in enumerate(args)]) for s in (1, -1))
        # the function is quadratic: the difference is exact but for binary32 roundings of values of size ~10 over 2h
        assert abs((up - down) / (2 * h) - float((grad.double() * d.double()).sum())) <= 400 * 2.0 ** -24 / h


def test_streams_and_graphs(ccdc):
    rng = np.random.default_rng(4)
    M, k, D, E = 700, 8, 72, 12                         # the sort takes a cluster
    ids = torch.from_numpy(draw_ids(rng, M, k, E, 0.1)).cuda()
    x = rows_of(rng, M, D, "float16")
    w = torch.rand((M, k), device="cuda")

    def all_of(stream=None):
        order = ccdc.expert_sort(ids, E, stream=stream)
        xs = ccdc.expert_dispatch(x, order, stream=stream)
        y = ccdc.expert_combine(xs, order, w, stream=stream)
        dys, dw = ccdc.expert_combine_backward(x, xs, order, w, stream=stream)
        return *order, xs, y, dys, dw, ccdc.expert_dispatch_backward(dys, order, stream=stream)

    want = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of()
    x.copy_(x.flip(0))
    ids.copy_(ids.flip(0))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, all_of()))


def test_more_than_two_to_the_31_elements(ccdc):
    M, k, D = 70000, 8, 4096
    x = torch.randn((M, D), device="cuda").bfloat16()
    ids = torch.randint(0, 5, (M, k), device="cuda")
    order = ccdc.expert_sort(ids, 5)
    xs = ccdc.expert_dispatch(x, order)
    last = order.slots[-50:].long()
    assert torch.equal(xs[-50:], x[last // k])
    w = torch.full((M, k), 0.125, device="cuda")
    assert torch.equal(ccdc.expert_combine(xs, order, w), x)            # eighths of eight copies: exact
    dys, dw = ccdc.expert_combine_backward(x, xs, order, w)
    assert torch.equal(dys[-50:], (x[last // k].float() * 0.125).bfloat16())
    m = int(last[-1]) // k
    assert torch.equal(dw[m], dw[m, :1].expand(k)) and abs(float(dw[m, 0]) / float(x[m].double().square().sum()) - 1) < 1e-5
