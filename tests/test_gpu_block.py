"""The block operators (dropout, norms with gate and residual, gated feed-forward block) against plain 64-bit
implementations, at the sizes, strides and masks where they can go wrong."""
import numpy as np
import pytest

from tests import block_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ccdc():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_1805_01993_b200 import build, ccdc as mod

    build.build_library()
    mod.lib()
    return mod


DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def tensor(rng, rows, cols, dtype, std=1.0, mean=0.0, pad=0, shift=0):
    """[rows][cols] with row stride cols + pad, starting `shift` elements into its memory"""
    flat = torch.from_numpy(rng.normal(mean, std, rows * (cols + pad) + shift)).to(DT[dtype]).cuda()
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def within(got, want, tol, what):
    got = f64(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    over = np.abs(got - want) - tol
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{what}{list(at)}: {got[at]} for {want[at]}, bound {np.broadcast_to(tol, want.shape)[at]}"


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,cols,pad,shift,offset", [(1, 1, 0, 0, 0), (1, 8, 0, 0, 0), (3, 7, 0, 0, 0), (5, 16, 8, 0, 16),
                                                        (5, 16, 8, 0, 3), (4, 33, 2, 1, 0), (2, 40, 0, 8, (1 << 34) + 8),
                                                        (1, 1000, 0, 3, (1 << 35) + 5),
                                                        (7, 301, 0, 0, 0), (300, 3, 1, 0, 6), (9, 256, 5, 1, 7), (5, 700, 3, 0, 0)])
def test_dropout(ccdc, dtype, rows, cols, pad, shift, offset):
    rng = np.random.default_rng(rows * 100 + cols)
    x = tensor(rng, rows, cols, dtype, pad=pad, shift=shift)
    seed = 0x1234567890ABCDEF
    keep = ref.keep_factors(rows, cols, 0.3, seed, offset)
    want = f64(x) * keep
    y = ccdc.dropout(x, 0.3, seed, offset)
    # the factor is rounded to binary32, the product once more, the result to its type
    within(y, want, np.abs(want) * (ref.U[dtype] + 3 * 2.0 ** -24) + ref.SMALLEST[dtype], "y")
    assert np.array_equal(f64(y) == 0, (keep == 0) | (f64(x) == 0))
    kept = ccdc.dropout(x, 0.3, seed, offset, out=x.clone(memory_format=torch.preserve_format))
    assert torch.equal(kept, y)
    ccdc.dropout(x, 0.3, seed, offset, out=x)               # in place
    assert torch.equal(x, y)


def test_dropout_extremes(ccdc):
    x = torch.full((3, 24), float("inf"), device="cuda")
    x[1] = float("nan")
    assert torch.equal(ccdc.dropout(x, 1.0, 5), torch.zeros_like(x))           # all dropped, whatever they hold
    assert torch.equal(ccdc.dropout(x, 0.0, 5).nan_to_num(7), x.nan_to_num(7))
    y = ccdc.dropout(x, 0.5, 5)
    keep = torch.from_numpy(ref.keep_factors(3, 24, 0.5, 5)).cuda()
    assert torch.equal(y == 0, keep == 0) and not y[keep > 0].isfinite().any()
    assert ccdc.dropout(torch.empty((0, 5), device="cuda"), 0.5, 1).shape == (0, 5)
    assert ccdc.dropout(torch.empty((5, 0), device="cuda"), 0.5, 1).shape == (5, 0)


def test_dropout_rate_and_scale(ccdc):
    x = torch.ones((1, 1 << 20), device="cuda")
    for p in (0.1, 0.5, 0.9):
        y = ccdc.dropout(x, p, 99)
        share = float((y != 0).double().mean())
        assert abs(share - (1 - p)) < 6 * (p * (1 - p) / (1 << 20)) ** 0.5 + 2.0 ** -17
        assert len(set(y.unique().tolist()) - {0.0}) == 1


# ---------------------------------------------------------------- norms, gate, residual
def norm_case(rng, M, D, dtype, gate, per, pad=0, shift=0, post=True, pre=True):
    t = dict(pad=pad, shift=shift)
    x, y = tensor(rng, M, D, dtype, 2.0, 0.3, **t), tensor(rng, M, D, dtype, 0.5, 0.2, **t)
    w_post = tensor(rng, 1, D, dtype, 0.2, 1.0).view(D) if post else None
    w_pre = tensor(rng, 1, D, dtype, 0.2, 1.0).view(D) if pre else None
    g = tensor(rng, -(-M // per), D, dtype, 0.5, 0.4) if gate else None
    return x, y, w_post, w_pre, g


NORMS = [(1, 1, 1), (1, 8, 1), (2, 5, 2), (3, 64, 1), (7, 129, 3), (300, 40, 7), (333, 1000, 50), (6, 1001, 2), (4, 2056, 4),
         (2, 4100, 1), (3, 8192, 3), (2, 8200, 1), (2, 9001, 2), (1, 20000, 1), (2, 32768, 2), (600, 16, 600),
         (5, 64, 5), (13, 48, 4), (5, 520, 5), (11, 1032, 11), (9, 2064, 4), (700, 256, 90), (1300, 128, 1300), (37, 4096, 10)]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("M,D,per", NORMS)
def test_residual_norm(ccdc, M, D, per, kind, dtype):
    """Forward and backward against the formulas in 64 bits.

    Bounds, relative to the terms' sizes: binary32 arithmetic over a row of D terms is within (D/4 + 64) 2^-24 (a
    thread adds at most D/32 + 32 terms in sequence), doubled where one norm reads the other's result; each output is
    rounded once to its type; the sum of M rows adds (M + 16) 2^-24 of the sum of absolute terms."""
    rng = np.random.default_rng(M * 7 + D)
    pad, shift = [(0, 0), (8, 0), (3, 1)][(M + D) % 3]
    x, y, w_post, w_pre, g = norm_case(rng, M, D, dtype, True, per, pad, shift)
    dout, dz = tensor(rng, M, D, dtype, pad=pad, shift=shift), tensor(rng, M, D, dtype, pad=pad)
    p, seed, offset, alpha, eps = 0.25, 77, 0 if D % 2 else 1 << 33, 0.5, 1e-5
    how = dict(w_post=w_post, w_pre=w_pre, gate=g, rows_per_gate=per, alpha=alpha, p=p, seed=seed, offset=offset, kind=kind)
    out, z, stats = ccdc.residual_norm_forward(x, y, save=True, eps=eps, **how)
    plain = ccdc.residual_norm_forward(x, y, eps=eps, **how)
    assert torch.equal(plain[0], out) and torch.equal(plain[1], z)
    if M * D <= 20000:
        keep = ref.keep_factors(M, D, p, seed, offset)
    else:       # the mask itself is tested above
        keep = f64(ccdc.dropout(torch.ones((M, D), device="cuda"), p, seed, offset))
        keep[keep > 0] = 65536.0 / (65536 - 16384)
    X, Y, WP, WQ, G, DO, DZ = (f64(t) for t in (x, y, w_post, w_pre, g, dout, dz))
    want, want_z = ref.norm_forward(X, Y, WP, WQ, G, per, alpha, keep, kind, eps)
    U, f = ref.U[dtype], (D / 4 + 64) * 2.0 ** -24
    tiny = ref.SMALLEST[dtype]

    def size(v):            # a row's terms before the mean is taken off
        return np.abs(v) + np.abs(v).mean(1, keepdims=True)

    def rstd(v):
        c = v - v.mean(1, keepdims=True) if kind == "layer" else v
        return 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)

    rows = np.arange(M) // per
    ry, ro = rstd(Y), rstd(want)
    # how much larger the row's terms are than what is left of them (the mean's subtraction), squared for the rstd
    ly, lo = (size(v).max(1, keepdims=True) * r + 1 for v, r in ((Y, ry), (want, ro)))
    n_err = f * ly * (size(Y) * ry + 1) * np.abs(WP)
    out_err = np.abs(alpha * X) * f + keep * np.abs(G[rows]) * n_err
    within(out, want, U * np.abs(want) + out_err * (1 + U) + tiny, "out")
    oh = ref.unit(want, kind, eps)
    oe = out_err.max(1, keepdims=True)
    oh_err = ro * out_err + ro * oe + np.abs(oh) * ro * oe + f * lo * (size(want) * ro + 1)
    within(z, want_z, U * np.abs(want_z) + oh_err * np.abs(WQ) * (1 + U) + tiny, "z")

    res = ccdc.residual_norm_backward(dout, dz, x, y, stats, **how)
    # gradients by 64-bit automatic differentiation of the formula
    leaves = [torch.from_numpy(v.copy()).requires_grad_() for v in (X, Y, WP, WQ, G)]
    tx, ty, twp, twq, tg = leaves

    def tunit(v):
        c = v - v.mean(1, keepdim=True) if kind == "layer" else v
        return c / ((c * c).mean(1, keepdim=True) + eps).sqrt()

    to = alpha * tx + tunit(ty) * twp * tg[torch.from_numpy(rows)] * torch.from_numpy(keep)
    tz = tunit(to) * twq
    grads = torch.autograd.grad((to, tz), leaves, (torch.from_numpy(DO), torch.from_numpy(DZ)))
    # sizes of the terms of t and dy
    e = np.abs(DZ * WQ)
    t_size = np.abs(DO) + ro * (e + e.mean(1, keepdims=True) + np.abs(oh) * (e * np.abs(oh)).mean(1, keepdims=True))
    t_err = f * lo * lo * t_size * 4 + ro * (e + e.mean(1, keepdims=True)) * (oh_err + oh_err.max(1, keepdims=True)) * (np.abs(oh) + 2)
    t_err += ro * ro * oe * (e + np.abs(oh) * (e * np.abs(oh)).mean(1, keepdims=True))
    yh = ref.unit(Y, kind, eps)
    yh_err = f * ly * (size(Y) * ry + 1)
    dn, dn_err = t_size * keep * np.abs(G[rows] * WP), t_err * keep * np.abs(G[rows] * WP)
    dy_size = ry * (dn + dn.mean(1, keepdims=True) + np.abs(yh) * (dn * np.abs(yh)).mean(1, keepdims=True))
    dy_err = (ry * (dn_err + dn_err.mean(1, keepdims=True) + np.abs(yh) * (dn_err * np.abs(yh)).mean(1, keepdims=True))
              + 4 * f * ly * ly * dy_size + ry * (dn + dn.mean(1, keepdims=True)) * (yh_err + yh_err.max(1, keepdims=True)) * (np.abs(yh) + 2))
    dx, dy, dw_post, dw_pre, dgate = res
    gr = [v.numpy() for v in grads]
    within(dx, gr[0], U * np.abs(gr[0]) + alpha * t_err + tiny, "dx")
    within(dy, gr[1], U * np.abs(gr[1]) + dy_err * (1 + U) + tiny, "dy")
    c = (M + 16) * 2.0 ** -23
    s_post, s_post_err = t_size * keep * np.abs(G[rows] * yh), t_err * keep * np.abs(G[rows]) * np.abs(yh) + t_size * keep * np.abs(G[rows]) * yh_err
    within(dw_post, gr[2], U * np.abs(gr[2]) + 2 * (s_post_err + c * s_post).sum(0) + tiny, "dw_post")
    within(dw_pre, gr[3], U * np.abs(gr[3]) + 2 * (np.abs(DZ) * oh_err + c * np.abs(DZ * oh)).sum(0) + tiny, "dw_pre")
    s_gate = t_err * keep * np.abs(WP * yh) + t_size * keep * np.abs(WP) * yh_err + c * t_size * keep * np.abs(WP * yh)
    bound = np.zeros_like(G)
    np.add.at(bound, rows, 2 * s_gate)
    within(dgate, gr[4], U * np.abs(gr[4]) + bound + tiny, "dgate")

    if dtype != "float32":
        f32 = ccdc.residual_norm_backward(dout, dz, x, y, stats, grad_dtype=torch.float32, **how)
        for a, b in zip(res[2:], f32[2:]):
            assert b.dtype == torch.float32 and torch.equal(b.to(a.dtype).view(-1), a.view(-1))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D", [48, 51])
def test_residual_norm_options(ccdc, dtype, D):
    """what may be left out: the norms, the gate, the dropout, the block itself, either gradient"""
    rng = np.random.default_rng(D)
    M, U = 19, ref.U[dtype]
    x, y, w_post, w_pre, g = norm_case(rng, M, D, dtype, True, M)
    out, z = ccdc.residual_norm_forward(x, y)
    assert z is None and torch.equal(out, (x.float() + y.float()).to(x.dtype))
    out, z = ccdc.residual_norm_forward(x, w_pre=w_pre)                 # the norm before the first block
    assert torch.equal(out, x)
    want = ref.unit(f64(x), "rms", 1e-5) * f64(w_pre)
    within(z, want, np.abs(want) * (U + 80 * 2.0 ** -24) + 2.0 ** -149, "z")
    out, _ = ccdc.residual_norm_forward(x, y, gate=g.view(D), alpha=1.0)
    want = f64(x) + f64(g) * f64(y)
    within(out, want, np.abs(want) * U + (np.abs(f64(x)) + np.abs(f64(g) * f64(y))) * 2.0 ** -22, "gated")
    # the fused dropout is the dropout
    out, _ = ccdc.residual_norm_forward(torch.zeros_like(x), y, p=0.5, seed=3, offset=8)
    assert torch.equal(out, ccdc.dropout(y, 0.5, 3, 8))
    # in place
    a, b = x.clone(), y.clone()
    want_out, want_z = ccdc.residual_norm_forward(x, y, w_post=w_post, w_pre=w_pre)
    ccdc.residual_norm_forward(a, b, w_post=w_post, w_pre=w_pre, out=a, z=b)
    assert torch.equal(a, want_out) and torch.equal(b, want_z)
    # zero gradients may be left out
    _, _, st = ccdc.residual_norm_forward(x, y, w_post=w_post, w_pre=w_pre, save=True)
    dz = tensor(rng, M, D, dtype)
    one = ccdc.residual_norm_backward(None, dz, x, y, st, w_post=w_post, w_pre=w_pre)
    two = ccdc.residual_norm_backward(torch.zeros_like(x), dz, x, y, st, w_post=w_post, w_pre=w_pre)
    assert all(torch.equal(s, t) for s, t in zip(one[:4], two[:4])) and one[4] is None
    _, _, st = ccdc.residual_norm_forward(x, y, save=True, alpha=2.0)
    dx, dy, a, b, c = ccdc.residual_norm_backward(dz, None, x, y, st, alpha=2.0)
    assert torch.equal(dx, 2 * dz) and torch.equal(dy, dz) and (a, b, c) == (None, None, None)


def test_residual_norm_rows_that_say_nothing(ccdc):
    """all of a row dropped, all of it zero, one infinite value under the mask, no rows"""
    D = 64
    w = torch.ones(D, device="cuda")
    x, y = torch.randn((3, D), device="cuda"), torch.randn((3, D), device="cuda")
    out, z = ccdc.residual_norm_forward(x, y, w_post=w, w_pre=w, p=1.0, seed=1)
    assert torch.equal(out, x) and z.isfinite().all()
    zero = torch.zeros_like(x)
    out, z, st = ccdc.residual_norm_forward(zero, zero, w_post=w, w_pre=w, save=True)
    assert not out.any() and not z.any()
    grads = ccdc.residual_norm_backward(x, y, zero, zero, st, w_post=w, w_pre=w)
    assert all(t.isfinite().all() for t in grads[:4])
    y[1, 5] = float("inf")
    keep = ccdc.dropout(torch.ones_like(y), 0.5, 9)
    seed = next(s for s in range(50) if ccdc.dropout(torch.ones_like(y), 0.5, s)[1, 5] == 0)
    out, _ = ccdc.residual_norm_forward(x, y, p=0.5, seed=seed)
    assert out.isfinite().all() and keep.isfinite().all()
    none = torch.empty((0, D), device="cuda")
    out, z, st = ccdc.residual_norm_forward(none, none, w_post=w, w_pre=w, gate=w, save=True)
    dx, dy, a, b, c = ccdc.residual_norm_backward(none, none, none, none, st, w_post=w, w_pre=w)
    assert dx.shape == (0, D) and not a.any() and not b.any()


def test_residual_norm_gradient_by_differences(ccdc):
    """central differences of the forward call itself, in binary32"""
    rng = np.random.default_rng(5)
    M, D, per, step = 4, 24, 2, 2.0 ** -6
    x, y, w_post, w_pre, g = norm_case(rng, M, D, "float32", True, per)
    dout, dz = tensor(rng, M, D, "float32"), tensor(rng, M, D, "float32")
    how = dict(alpha=0.5, p=0.25, seed=11, rows_per_gate=per, kind="layer")

    def loss(x, y, a, b, c):
        out, z = ccdc.residual_norm_forward(x, y, w_post=a, w_pre=b, gate=c, **how)
        return float((out.double() * dout.double()).sum() + (z.double() * dz.double()).sum())

    _, _, st = ccdc.residual_norm_forward(x, y, w_post=w_post, w_pre=w_pre, gate=g, save=True, **how)
    grads = ccdc.residual_norm_backward(dout, dz, x, y, st, w_post=w_post, w_pre=w_pre, gate=g, **how)
    args = [x, y, w_post, w_pre, g]
    for k, grad in enumerate(grads):
        d = torch.from_numpy(rng.normal(size=tuple(args[k].shape))).float().cuda()
        up, down = ([a + s * step * d if i == k else a for i, a in enumerate(args)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * step)
        want = float((grad.double() * d.double()).sum())
        # third derivatives times step^2, and roundoff over the step, of terms of size one
        assert abs(slope - want) <= 0.02 * (abs(want) + float(grad.double().norm() * d.double().norm())), k


# ---------------------------------------------------------------- gated feed-forward block
FFNS = [(1, 8, 8), (1, 1, 1), (2, 3, 5), (1, 64, 200), (3, 136, 72), (8, 128, 256), (16, 256, 264), (17, 64, 64), (24, 200, 136),
        (33, 72, 328), (64, 64, 128), (65, 130, 67), (100, 256, 128), (128, 128, 128), (129, 264, 136), (200, 65, 300),
        (257, 320, 512), (300, 512, 264), (520, 264, 520), (5, 1000, 31)]


def ffn_case(rng, M, D, F, dtype, pad, shift):
    x = tensor(rng, M, D, dtype, pad=pad, shift=shift)
    wg, wu = (tensor(rng, F, D, dtype, D ** -0.5, pad=pad) for _ in range(2))
    wd = tensor(rng, D, F, dtype, F ** -0.5, pad=pad, shift=shift)
    return x, wg, wu, wd, tensor(rng, M, D, dtype, pad=pad)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,D,F", FFNS)
def test_ffn(ccdc, M, D, F, dtype):
    rng = np.random.default_rng(M * 31 + D + F)
    act = ["silu", "gelu", "gelu_tanh", "relu"][(M + D + F) % 4]
    pad, shift = [(0, 0), (8, 0), (5, 1)][(M + F) % 3]
    x, wg, wu, wd, dy = ffn_case(rng, M, D, F, dtype, pad, shift)
    want = ref.ffn(*(f64(t) for t in (x, wg, wu, wd)), act, f64(dy), dtype)
    y = ccdc.ffn_forward(x, wg, wu, wd, act=act)
    within(y, *want["y"], "y")
    y2, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    within(y2, *want["y"], "y with save")
    grads = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)
    for name, g in zip(("dx", "dw_gate", "dw_up", "dw_down"), grads):
        within(g, *want[name], name)
    again = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))              # the same bits every time
    if dtype != "float32":
        want = ref.ffn(*(f64(t) for t in (x, wg, wu, wd)), act, f64(dy), dtype, "float32")
        f32 = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act, grad_dtype=torch.float32)
        for name, g in list(zip(("dx", "dw_gate", "dw_up", "dw_down"), f32))[1:]:
            assert g.dtype == torch.float32
            within(g, *want[name], name + " in 32 bits")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("dtype", DT)
def test_ffn_activations(ccdc, act, dtype):
    rng = np.random.default_rng(3)
    x, wg, wu, wd, dy = ffn_case(rng, 40, 64, 96, dtype, 0, 0)
    wg = wg * 6                                         # far into the tails
    want = ref.ffn(*(f64(t) for t in (x, wg, wu, wd)), act, f64(dy), dtype)
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    within(y, *want["y"], "y")
    for name, g in zip(("dx", "dw_gate", "dw_up", "dw_down"), ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)):
        within(g, *want[name], name)


def test_ffn_no_rows_and_slices(ccdc):
    D, F = 64, 96
    rng = np.random.default_rng(8)
    x, wg, wu, wd, dy = ffn_case(rng, 32, D, F, "bfloat16", 0, 0)
    y, saved = ccdc.ffn_forward(x[:0], wg, wu, wd, save=True)
    assert y.shape == (0, D)
    grads = ccdc.ffn_backward(dy[:0], x[:0], wg, wu, wd, saved)
    assert grads[0].shape == (0, D) and not any(g.any() for g in grads[1:])
    # gradients into consecutive slices of one row of 32-bit words, as a partition holds them
    row = torch.full((3 * D * F + 8,), 7.0, device="cuda")
    parts = [row[i * D * F:(i + 1) * D * F] for i in range(3)]
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    ccdc.ffn_backward(dy, x, wg, wu, wd, saved, grad_dtype=torch.float32, dw_gate=parts[0], dw_up=parts[1], dw_down=parts[2])
    own = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, grad_dtype=torch.float32)
    assert torch.equal(row[:-8], torch.cat([g.reshape(-1) for g in own[1:]])) and bool((row[-8:] == 7).all())


def test_ffn_does_not_write_outside(ccdc):
    """outputs with wider rows keep what lies between the rows"""
    rng = np.random.default_rng(9)
    for M, D, F in ((3, 40, 24), (150, 136, 72), (40, 33, 50)):
        x, wg, wu, wd, dy = ffn_case(rng, M, D, F, "bfloat16", 0, 0)
        wide = torch.full((M + 2, D + 16), 3.0, dtype=torch.bfloat16, device="cuda")
        ccdc.ffn_forward(x, wg, wu, wd, out=wide[1:-1, 8:8 + D])
        assert torch.equal(wide[1:-1, 8:8 + D], ccdc.ffn_forward(x, wg, wu, wd))
        wide[1:-1, 8:8 + D] = 3.0
        assert bool((wide == 3).all())


def test_ffn_infinities_stay_in_their_rows(ccdc):
    rng = np.random.default_rng(10)
    x, wg, wu, wd, _ = ffn_case(rng, 150, 72, 80, "bfloat16", 0, 0)
    clean = ccdc.ffn_forward(x, wg, wu, wd)
    x[7, 3], x[140, 0] = float("inf"), float("nan")
    y = ccdc.ffn_forward(x, wg, wu, wd)
    rest = [i for i in range(150) if i not in (7, 140)]
    assert torch.equal(y[rest], clean[rest]) and not y[140].isfinite().any()


def test_ffn_gradient_by_differences(ccdc):
    rng = np.random.default_rng(12)
    args = list(ffn_case(rng, 12, 24, 40, "float32", 0, 0))
    dy, args, step = args[4], args[:4], 2.0 ** -7

    def loss(*a):
        return float((ccdc.ffn_forward(*a).double() * dy.double()).sum())

    _, saved = ccdc.ffn_forward(*args, save=True)
    for k, grad in enumerate(ccdc.ffn_backward(dy, *args, saved)):
        d = torch.from_numpy(rng.normal(size=tuple(args[k].shape)) * float(args[k].std())).float().cuda()
        up, down = ([a + s * step * d if i == k else a for i, a in enumerate(args)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * step)
        want = float((grad.double() * d.double()).sum())
        assert abs(slope - want) <= 0.01 * (abs(want) + float(grad.double().norm() * d.double().norm())), k


def test_on_another_stream_and_in_a_graph(ccdc):
    rng = np.random.default_rng(13)
    x, wg, wu, wd, dy = ffn_case(rng, 70, 64, 96, "bfloat16", 0, 0)
    want, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    want_g = ccdc.ffn_backward(dy, x, wg, wu, wd, saved)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True, stream=side)
    grads = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, stream=side)
    side.synchronize()
    assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(grads, want_g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, z = ccdc.residual_norm_forward(x, ccdc.ffn_forward(x, wg, wu, wd), w_pre=wd[:, 0].contiguous(), p=0.5, seed=4)
        d = ccdc.dropout(z, 0.5, 5)
    x.copy_(dy)                                     # new values, same buffers
    graph.replay()
    torch.cuda.synchronize()
    e_out, e_z = ccdc.residual_norm_forward(x, ccdc.ffn_forward(x, wg, wu, wd), w_pre=wd[:, 0].contiguous(), p=0.5, seed=4)
    assert torch.equal(out, e_out) and torch.equal(z, e_z) and torch.equal(d, ccdc.dropout(e_z, 0.5, 5))


# ---------------------------------------------------------------- every tile shape of the products
@pytest.mark.parametrize("M,D,F,dtype", [(600, 520, 4104, "bfloat16"), (1100, 1032, 5000, "float16"), (2304, 1024, 4096, "bfloat16"),
                                         (300, 776, 1544, "float32"), (17, 2048, 4100, "bfloat16")])
def test_ffn_large_tiles(ccdc, M, D, F, dtype):
    """sizes at which the launches take the large tiles, cuts along k and several rounds of tiles, with ragged edges;
    compared in 64 bits on the device, by norm: a result's rounding, and those of a, dh and du, are independent and
    each at most U sqrt(1/3) of the values' size in the mean; 3 times their joint size is allowed"""
    g = torch.Generator(device="cuda").manual_seed(M + D)

    def randn(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])

    x, dy = randn(M, D), randn(M, D)
    wg, wu, wd = randn(F, D, std=D ** -0.5), randn(F, D, std=D ** -0.5), randn(D, F, std=F ** -0.5)
    leaves = [t.double().requires_grad_() for t in (x, wg, wu, wd)]
    h, u = leaves[0] @ leaves[1].t(), leaves[0] @ leaves[2].t()
    want = (h * torch.sigmoid(h) * u) @ leaves[3].t()
    grads = torch.autograd.grad(want, leaves, dy.double())
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    got = (y, *ccdc.ffn_backward(dy, x, wg, wu, wd, saved))
    tol = 2.0 ** -19 if dtype == "float32" else 3 * ref.U[dtype] * (4 / 3) ** 0.5
    for name, a, b in zip(("y", "dx", "dw_gate", "dw_up", "dw_down"), got, (want.detach(), *grads)):
        err = float((a.double() - b).norm() / b.norm())
        assert err <= tol, (name, err)
        # no element is off by more than the sum's size allows: a misplaced tile would be
        assert float((a.double() - b).abs().max() / b.abs().max()) <= 40 * tol, name
    ccdc.block_status()


# ---------------------------------------------------------------- the operators in a coded gradient job
def test_block_job(ccdc):
    """Map, shuffle and Reduce of the sub-block's gradients: replicas bit-identical, the Reduce output the sum over the
    files, the gradients those of automatic differentiation"""
    from paper_1805_01993_b200 import block_job

    nodes, load, files, rows, D, F, p, seed = 4, 2, 12, 40, 64, 96, 0.25, 77
    total, per_file, plan, losses = block_job.run(nodes, load, files, rows, D, F, p, seed, torch.float32)
    direct, size = per_file.double().sum(0), per_file.double().abs().sum(0)
    assert bool(((total.double() - direct).abs() <= 1e-5 * size + 1e-30).all())
    params = block_job.make_parameters(D, F, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(seed)
    data = [torch.randn((rows, D), generator=g, device="cuda") for _ in range(files)]
    for n in (0, 5, 11):
        leaves = {k: v.double().requires_grad_() for k, v in params.items()}

        def unit(v):
            return v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()

        x = data[n].double()
        z = unit(x) * leaves["w_pre"]
        h = z @ leaves["w_gate"].t()
        y = (h * torch.sigmoid(h) * (z @ leaves["w_up"].t())) @ leaves["w_down"].t()
        keep = torch.from_numpy(ref.keep_factors(rows, D, p, seed, n * rows * D)).cuda()
        out = x + unit(y) * leaves["w_post"] * leaves["gate"] * keep
        loss = out.square().mean()
        grads = torch.autograd.grad(loss, [leaves[k] for k in block_job.PARAMETERS])
        assert abs(float(losses[n]) - float(loss.detach())) <= 1e-5 * float(loss.detach())
        at = 0
        for k, want in zip(block_job.PARAMETERS, grads):
            got = per_file[n][at:at + want.numel()].double().view(want.shape)
            at += want.numel()
            assert float((got - want).norm() / want.norm()) <= 1e-5, (n, k)
    # the nodes' replicas agree bit by bit
    again = block_job.run(nodes, load, files, rows, D, F, p, seed, torch.float32)
    assert torch.equal(again[1], per_file) and torch.equal(again[0], total)


def test_block_job_replicas(ccdc):
    """a file mapped twice, from other addresses, leaves the same bits"""
    from paper_1805_01993_b200 import block_job

    D, F, rows = 136, 200, 33
    params = block_job.make_parameters(D, F, torch.bfloat16)
    x = torch.randn((rows, D), device="cuda").bfloat16()
    words = block_job.gradient_words(D, F)
    a, b = torch.zeros(words, device="cuda"), torch.ones(words + 64, device="cuda")[64:]
    block_job.map_file(x, params, 0.1, 5, 1000, a)
    block_job.map_file(x.clone(), {k: v.clone() for k, v in params.items()}, 0.1, 5, 1000, b)
    assert torch.equal(a, b) and bool(a.isfinite().all())


# ---------------------------------------------------------------- offsets beyond 32 bits
def test_more_than_two_to_the_31_elements(ccdc):
    """the last rows of tensors of over 2^31 elements against calls on those rows alone"""
    D = 8192
    M = (1 << 31) // D + 40
    x = torch.empty((M, D), dtype=torch.bfloat16, device="cuda")
    x[-64:].normal_()
    x[:64].normal_()
    x[64:-64].zero_()
    w = torch.ones(D, dtype=torch.bfloat16, device="cuda")
    y = ccdc.dropout(x, 0.5, 3)
    tail = x[-8:].clone()
    assert torch.equal(y[-8:], ccdc.dropout(tail, 0.5, 3, (M - 8) * D))
    gate = torch.randn((2, D), device="cuda").bfloat16()
    out, z, st = ccdc.residual_norm_forward(x, y, w_post=w, w_pre=w, gate=gate, rows_per_gate=M - 20, p=0.25, seed=4, save=True)
    how = dict(w_post=w, w_pre=w, gate=gate[1:], rows_per_gate=8, p=0.25, seed=4, offset=(M - 8) * D)
    o, zz, s = ccdc.residual_norm_forward(tail, y[-8:].clone(), save=True, **how)
    assert torch.equal(out[-8:], o) and torch.equal(z[-8:], zz)
    dx, dy, *_ = ccdc.residual_norm_backward(x, z, x, y, st, w_post=w, w_pre=w, gate=gate, rows_per_gate=M - 20, p=0.25, seed=4)
    tx, ty, *_ = ccdc.residual_norm_backward(tail, zz, tail, y[-8:].clone(), s, **how)
    assert torch.equal(dx[-8:], tx) and torch.equal(dy[-8:], ty)
    del out, z, st, dx, dy, y, x
    torch.cuda.empty_cache()
    M, D, F = (1 << 31) // 16384 + 300, 64, 16384
    x = torch.randn((M, D), device="cuda").bfloat16()
    wg, wu, wd = (torch.randn(s, device="cuda").bfloat16() * 0.1 for s in ((F, D), (F, D), (D, F)))
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    small, kept = ccdc.ffn_forward(x[-200:], wg, wu, wd, save=True)
    dx = ccdc.ffn_backward(y, x, wg, wu, wd, saved)[0]
    sx = ccdc.ffn_backward(y[-200:], x[-200:], wg, wu, wd, kept)[0]
    for a, b in ((y[-200:], small), (dx[-200:], sx)):       # other tiles, other orders of the sums
        assert float((a.double() - b.double()).norm() / b.double().norm()) <= 2.0 ** -8
    ccdc.block_status()
