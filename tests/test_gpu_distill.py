"""The distillation loss and its gradient against a plain 64-bit implementation."""
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


def f64(t):
    return t.double().cpu().numpy()


def reference(z, ids, values, T, lse, dloss, u, tiny):
    """(loss, its bound, dz, its bound).  The sum of exponentials: each has 2^-22 (approximate exponential) and three roundings
    of (z - top) / T, whose mean over s is at most log V; a thread adds V / 512 of them (vectors to threads) and 40 more sums and
    rescalings join them.  Differences of logits carry the roundings of (z - top) and of log2(e) / T."""
    M, V = z.shape
    loss, loss_tol, dz, dz_tol = np.zeros(M), np.zeros(M), np.zeros((M, V)), np.zeros((M, V))
    e32 = 2.0 ** -24
    sums = 2.0 ** -22 + e32 * (3 * np.log(V + 1) + V / 512 + 60)
    for m in range(M):
        there = [j for j in range(ids.shape[1]) if 0 <= ids[m, j] < V and values[m, j] != -np.inf]
        if not there:
            continue
        v = values[m, there] / T
        whole = v.max() + np.log(np.exp(v - v.max()).sum()) if lse is None else lse[m]
        t = np.exp(v - whole)
        zt = z[m] / T
        top = zt.max()
        log_s = zt - top - np.log(np.exp(zt - top).sum())
        at = ids[m, there]
        used = t > 0
        loss[m] = (t[used] * (v[used] - whole - log_s[at][used])).sum()
        away = np.where(np.isfinite(zt), top - zt, 0.0)
        loss_tol[m] = t.sum() * sums + (t * away[at]).sum() * 2 * e32 + e32 * abs(loss[m])
        P, s, target = t.sum(), np.exp(log_s), np.zeros(V)
        np.add.at(target, at, t)
        g = dloss[m] / T
        dz[m] = g * (P * s - target)
        dz_tol[m] = abs(g) * (P * s * (sums + 2.0 ** -22 + e32 * (3 * away + 6)) + target * 4 * e32) * (1 + u) + u * abs(dz[m]) + tiny
    return loss, loss_tol, dz, dz_tol


def case(rng, M, V, k, dtype, kind, pad=0, shift=0, spread=2.0):
    flat = torch.from_numpy(rng.normal(0, spread, M * (V + pad) + shift)).to(DT[dtype]).cuda()
    z = flat[shift:].view(M, V + pad)[:, :V]
    ids = rng.integers(0, V, (M, k))                    # some twice
    ids[rng.random((M, k)) < 0.2] = -1
    ids[rng.random((M, k)) < 0.05] = V + 3
    if M > 1:
        ids[M // 2] = -1                                # a row without targets
    values = torch.from_numpy(rng.normal(3, spread, (M, k))).to(DT[dtype]).cuda()
    dloss = torch.from_numpy(rng.random(M) + 0.5).float().cuda()
    return z, torch.from_numpy(ids).to(kind).cuda(), values, dloss


def check(ccdc, z, ids, values, dloss, T, lse, dtype):
    want = reference(f64(z), ids.cpu().numpy(), f64(values), T, None if lse is None else f64(lse), f64(dloss), U[dtype], SMALLEST[dtype])
    how = dict(temperature=T, teacher_lse=lse)
    loss, stats = ccdc.distill_forward(z, ids, values, save=True, **how)
    dz = ccdc.distill_backward(dloss, z, ids, values, stats, **how)
    both = ccdc.distill(dloss, z, ids, values, **how)
    same = z.clone()
    inside = ccdc.distill(dloss, same, ids, values, dlogits=same, **how)       # the gradient takes the logits' place
    assert inside[1].data_ptr() == same.data_ptr()
    for l, g in ((loss, dz), both, inside):
        assert l.dtype is torch.float32 and g.dtype is z.dtype
        over = np.abs(f64(l) - want[0]) - want[1]
        assert over.max(initial=0) <= 0, ("loss", over.max(), over.argmax())
        over = np.abs(f64(g) - want[2]) - want[3]
        assert over.max(initial=0) <= 0, ("dz", over.max(), np.unravel_index(over.argmax(), over.shape))
    assert torch.equal(both[0], loss) and torch.equal(both[1], dz)
    assert torch.equal(ccdc.distill_forward(z, ids, values, **how), loss)
    if same.stride() == z.stride() and (same.data_ptr() - z.data_ptr()) % 16 == 0:     # rows that start alike: one order of sums
        assert torch.equal(inside[0], loss) and torch.equal(inside[1], dz)


SHAPES = [(1, 1, 1, 0, 0), (2, 2, 3, 0, 0), (3, 7, 2, 1, 1), (2, 8, 5, 0, 0), (4, 33, 8, 5, 3), (3, 1000, 1, 0, 0), (2, 4096, 64, 8, 0),
          (5, 4099, 100, 0, 0), (2, 16385, 1024, 0, 7), (3, 32000, 16, 0, 0), (300, 257, 9, 0, 0), (2, 70001, 50, 3, 0),
          (2, 131072, 40, 0, 0)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,V,k,pad,shift", SHAPES)
def test_distill(ccdc, M, V, k, pad, shift, dtype):
    rng = np.random.default_rng(M * 7 + V)
    for T, kind, whole in ((1.0, torch.int32, False), (2.5, torch.int64, True)):
        z, ids, values, dloss = case(rng, M, V, k, dtype, kind, pad, shift)
        # a whole teacher's sum that is larger than the slots' own
        lse = torch.from_numpy(np.log(np.exp(f64(values) / T).sum(1) * 1.25)).float().cuda() if whole else None
        check(ccdc, z, ids, values, dloss, T, lse, dtype)


@pytest.mark.parametrize("dtype", DT)
def test_values_in_32_bits_and_strides_of_the_gradient(ccdc, dtype):
    rng = np.random.default_rng(5)
    M, V, k = 6, 777, 12
    z, ids, _, dloss = case(rng, M, V, k, dtype, torch.int32)
    values = torch.from_numpy(rng.normal(3, 2, (M, k))).float().cuda()
    check(ccdc, z, ids, values, dloss, 0.7, None, dtype)
    loss, dz = ccdc.distill(dloss, z, ids, values)
    for pad, shift in ((8, 0), (3, 0), (0, 1), (5, 5)):         # rows that start elsewhere than the logits' do
        flat = torch.full((M * (V + pad) + shift + 9,), 7.0, dtype=DT[dtype], device="cuda")
        out = flat[shift:shift + M * (V + pad)].view(M, V + pad)[:, :V]
        l, g = ccdc.distill(dloss, z, ids, values, dlogits=out)
        assert torch.equal(g, dz) and torch.equal(l, loss)
        assert int((flat != 7).sum()) <= int((dz != 7).sum())
        assert bool((flat[:shift] == 7).all()) and bool((flat[shift + M * (V + pad):] == 7).all())
        if pad:
            assert bool((flat[shift:shift + M * (V + pad)].view(M, V + pad)[:, V:] == 7).all())


@pytest.mark.parametrize("dtype", DT)
def test_masked_logits_and_rows_that_say_nothing(ccdc, dtype):
    """-infinity and the type's lowest value have no probability; padding rows are zero whatever they hold"""
    rng = np.random.default_rng(6)
    M, V, k = 8, 600, 6
    z, ids, values, dloss = case(rng, M, V, k, dtype, torch.int32)
    ids[:] = torch.from_numpy(rng.integers(0, 300, (M, k))).int().cuda()
    z[0, 300:] = -float("inf")
    z[1, 300:] = torch.finfo(DT[dtype]).min
    z[2] = torch.finfo(DT[dtype]).min                   # a row of lowest values is uniform
    values[3, 2:] = -float("inf")                       # two slots left
    ids[4], z[4] = -1, float("nan")                     # padding
    values[5] = -float("inf")                           # no slot left
    z[5] = float("inf")
    check(ccdc, z[:4], ids[:4], values[:4], dloss[:4], 1.0, None, dtype)
    for loss, dz in (ccdc.distill(dloss, z, ids, values),):
        assert float(loss[4]) == 0 == float(loss[5]) and not dz[4].any() and not dz[5].any()
        assert not dz[0, 300:].any() and bool(loss.isfinite().all()) and bool(dz.isfinite().all())
    # a masked target: infinite loss, finite gradient; NaN and +infinity make their own row NaN
    z[6, int(ids[6, 0])] = -float("inf")
    z[7, 5] = float("nan")
    loss, stats = ccdc.distill_forward(z, ids, values, save=True)
    dz = ccdc.distill_backward(dloss, z, ids, values, stats)
    assert float(loss[6]) == float("inf") and bool(dz[6].isfinite().all()) and float(dz[6, int(ids[6, 0])]) < 0
    assert bool(loss[7].isnan()) and bool(dz[7].isnan().all()) and bool(loss[:6].isfinite().all())
    z[7, 5] = float("inf")
    assert bool(ccdc.distill_forward(z, ids, values)[7].isnan())
    z[7] = -float("inf")
    assert bool(ccdc.distill_forward(z, ids, values)[7].isnan())
    # a teacher's sum so large that nothing is left: P = 0
    lse = torch.full((M,), 1e30, device="cuda")
    loss, dz = ccdc.distill(dloss, z, ids, values, teacher_lse=lse)
    assert not loss.any() and not dz.any()


def test_one_id_in_every_slot(ccdc):
    """slots of one id add up, and are rounded once"""
    z = torch.zeros((1, 64), device="cuda", dtype=torch.bfloat16)
    ids = torch.full((1, 10), 9, dtype=torch.int64, device="cuda")
    values = torch.arange(10, device="cuda").bfloat16()[None]
    loss, dz = ccdc.distill(torch.ones(1, device="cuda"), z, ids, values)
    t = torch.softmax(values.double(), 1)
    assert abs(float(loss) - (float((t * t.log()).sum()) + np.log(64))) <= 2.0 ** -20
    assert float(dz[0, 9]) == float(torch.tensor(1 / 64 - 1).bfloat16()) and bool((dz[0, :9] == 1 / 64).all())


def test_no_rows_and_large_logits(ccdc):
    e = torch.empty((0, 50), device="cuda")
    i = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    loss, dz = ccdc.distill(e[:, 0], e, i, e[:, :3].contiguous())
    assert loss.shape == (0,) and dz.shape == (0, 50)
    # far from zero the differences alone count
    rng = np.random.default_rng(2)
    z = torch.from_numpy(rng.normal(0, 2, (3, 500)) + np.array([[0.0], [2.0 ** 14], [-2.0 ** 14]])).float().cuda()
    ids = torch.from_numpy(rng.integers(0, 500, (3, 4))).int().cuda()
    check(ccdc, z, ids, torch.randn((3, 4), device="cuda") + 2.0 ** 12, torch.ones(3, device="cuda"), 1.0, None, "float32")


def test_gradient_by_differences(ccdc):
    rng = np.random.default_rng(9)
    M, V, k, T = 4, 40, 5, 1.5
    z, ids, values, dloss = case(rng, M, V, k, "float32", torch.int32, spread=1.0)
    d = torch.from_numpy(rng.normal(size=(M, V))).float().cuda()
    h = 2.0 ** -5
    lse = torch.logsumexp(values / T, 1) + 0.3
    for whole in (None, lse):
        _, dz = ccdc.distill(dloss, z, ids, values, temperature=T, teacher_lse=whole)
        up, down = (float((ccdc.distill_forward(z + s * h * d, ids, values, temperature=T, teacher_lse=whole).double() * dloss.double()).sum())
                    for s in (1, -1))
        # third derivatives of a log of sums of exponentials are at most |d / T|^3 a row (d up to 4): 4 * 1.5 * (4 / 1.5)^3 h^2 / 6
        assert abs((up - down) / (2 * h) - float((dz.double() * d.double()).sum())) <= 19 * h * h + 100 * 2.0 ** -24 / h


def test_streams_and_graphs(ccdc):
    rng = np.random.default_rng(4)
    z, ids, values, dloss = case(rng, 400, 3001, 20, "bfloat16", torch.int64)

    def all_of(stream=None):
        loss, stats = ccdc.distill_forward(z, ids, values, save=True, stream=stream)
        dz = ccdc.distill_backward(dloss, z, ids, values, stats, stream=stream)
        return loss, dz, *ccdc.distill(dloss, z, ids, values, stream=stream)

    want = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = all_of(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of()
    z.copy_(z.flip(0))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, all_of()))


def test_more_than_two_to_the_31_elements(ccdc):
    M, V = 20000, 131072
    z = torch.zeros((M, V), dtype=torch.bfloat16, device="cuda")
    z[-3:].normal_()
    ids = torch.randint(0, V, (M, 4), device="cuda")
    ids[:-3] = -1
    values = torch.randn((M, 4), device="cuda").bfloat16()
    dloss = torch.ones(M, device="cuda")
    loss, dz = ccdc.distill(dloss, z, ids, values)
    l, g = ccdc.distill(dloss[-3:], z[-3:].clone(), ids[-3:], values[-3:])
    # three rows alone are cut into more parts: sums of 131072 positive terms in another order, a thread's at most 512 of them
    # one after the other and 40 more joins, in each call; a bf16 result may then round to the other side
    close = 2 * (512 + 40) * 2.0 ** -24
    assert bool(((loss[-3:] - l).abs() <= close + 2.0 ** -23 * l.abs()).all()) and not loss[:-3].any() and not dz[:-3].any()
    assert bool(((dz[-3:].float() - g.float()).abs() <= (2.0 ** -7 + close) * g.float().abs() + close * 2.0 ** -10).all())
