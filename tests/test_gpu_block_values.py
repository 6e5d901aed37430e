"""The block operators at values and arguments where a plain formula and a fast kernel part ways: NaN and infinities,
the largest finite numbers, tails of the activations, element numbers and group sizes at the end of 64 bits, outputs that
are left out, buffers that a call cannot use."""
import numpy as np
import pytest

from tests import block_reference as ref
from tests.test_gpu_block import DT, ccdc, f64, ffn_case, norm_case, tensor, within  # noqa: F401 (ccdc: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
GRADS = ("dx", "dw_gate", "dw_up", "dw_down")


# ---------------------------------------------------------------- feed-forward: NaN
@pytest.mark.parametrize("M", [3, 20, 40])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DT)
def test_ffn_nan_in_one_weight(ccdc, dtype, act, M):
    """A NaN in w_gate alone reaches h of one inner column, and from there whatever that column enters: all of y and dx,
    one row of dw_gate and dw_up, one column of dw_down.  The rest keeps its bits."""
    rng = np.random.default_rng(M)
    x, wg, wu, wd, dy = ffn_case(rng, M, 64, 96, dtype, 0, 0)
    f = 37
    _, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    clean = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)
    bad = wg.clone()
    bad[f, 5] = float("nan")
    y, saved = ccdc.ffn_forward(x, bad, wu, wd, act=act, save=True)
    dx, *grads = ccdc.ffn_backward(dy, x, bad, wu, wd, saved, act=act)
    assert y.isnan().all() and dx.isnan().all()
    for name, g, c in zip(GRADS[1:], grads, clean[1:]):
        g, c = (g.t(), c.t()) if name == "dw_down" else (g, c)
        assert g[f].isnan().all(), name
        rest = [i for i in range(96) if i != f]
        assert torch.equal(g[rest], c[rest]), name


# ---------------------------------------------------------------- feed-forward: infinities
def same_kind(got, want, what):
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    big = np.isinf(want)
    assert np.array_equal(np.isinf(got), big) and np.array_equal(got[big], want[big]), what


@pytest.mark.parametrize("M", [8, 32, 33, 150])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DT)
def test_ffn_infinities(ccdc, dtype, act, M):
    """An infinity times a finite value is an infinity, whatever that value's bits (quarters here, which 8 bits hold) and
    however many rows the call has."""
    rng = np.random.default_rng(M)
    D, F = 72, 80

    def quarters(*shape, most=3):
        return torch.from_numpy(rng.integers(1, most + 1, shape) * rng.choice([-0.25, 0.25], shape)).to(DT[dtype]).cuda()

    # h stays within a few units, so that no activation's tail leaves the types' range
    x, wg, wu, wd, dy = quarters(M, D, most=1), quarters(F, D), quarters(F, D), quarters(D, F), quarters(M, D)
    wg[:, 3], wu[:, 3] = wg[:, 3].abs(), -wu[:, 3].abs()            # h = inf and u = -inf where x[., 3] is inf
    wd[::2], wd[1::2] = wd[::2].abs(), -wd[1::2].abs()              # and y an infinity of either sign
    clean, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    dirty = x.clone()
    dirty[5, 3] = float("inf")
    y = ccdc.ffn_forward(dirty, wg, wu, wd, act=act)
    rest = [i for i in range(M) if i != 5]
    assert torch.equal(y[rest], clean[rest])
    assert bool((y[5, ::2] == -float("inf")).all() and (y[5, 1::2] == float("inf")).all())
    # an infinite weight: every row of one inner column
    bad = wu.clone()
    bad[9, 7] = float("inf")
    with np.errstate(all="ignore"):
        h, u = f64(x) @ f64(wg).T, f64(x) @ f64(bad).T
        assert np.isinf(u[:, 9]).all() and np.isfinite(np.delete(u, 9, 1)).all()
        want = (ref.act(act, h)[0] * u) @ f64(wd).T
    same_kind(ccdc.ffn_forward(x, wg, bad, wd, act=act), want, "y")
    # an infinite gradient of one output: its row of da, and what that enters
    dirty = dy.clone()
    dirty[2, 4] = -float("inf")
    with np.errstate(all="ignore"):
        u = f64(x) @ f64(wu).T
        f, df, _ = ref.act(act, h)
        da = f64(dirty) @ f64(wd)
        assert np.isinf(da[2]).all()
        dh, du = da * u * df, da * f
        want = {"dx": dh @ f64(wg) + du @ f64(wu), "dw_gate": dh.T @ f64(x), "dw_up": du.T @ f64(x),
                "dw_down": f64(dirty).T @ (f * u)}
    for name, g in zip(GRADS, ccdc.ffn_backward(dirty, x, wg, wu, wd, saved, act=act)):
        same_kind(g, want[name], name)


@pytest.mark.parametrize("M", [32, 33, 150])
def test_ffn_largest_binary32(ccdc, M):
    """finite values that no 16-bit type holds: above the largest bf16, met by weights at the small end"""
    rng = np.random.default_rng(M)
    x, wg, wu, wd, dy = ffn_case(rng, M, 72, 80, "float32", 0, 0)
    large = float(np.finfo(np.float32).max)
    x[3, 2], x[4, 2] = large, -0.9999 * large
    x[:3, 2], x[5:, 2] = 0.0, 0.0
    wg[:, 2], wu[:, 2] = 2.0 ** -126, -(2.0 ** -126)
    wg[11, 6], wu[12, 6] = large, -large
    x[:, 6] = 2.0 ** -126 * (1 + torch.arange(M, device="cuda") % 2)
    want = ref.ffn(*(f64(t) for t in (x, wg, wu, wd)), "silu", None, "float32")
    within(ccdc.ffn_forward(x, wg, wu, wd), *want["y"], "y")


# ---------------------------------------------------------------- feed-forward: activations
@pytest.mark.parametrize("M", [7, 30, 200])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DT)
def test_activation_tails(ccdc, act, dtype, M):
    """act(h) and act'(h) one by one, relative to their own size far into the negative tail.

    h, u = 1 and the output weight 1 pass through the products exactly, so y is act(h) rounded and dx is act'(h) rounded
    (twice, dh and dx).  The exponential's argument t has a few roundings, |t| 2^-22 of it, which is the relative error
    they leave in the exponential; CUDA's fast exponential adds (2 + 1.2 |t|) 2^-23 and the operations around it less
    than 16 units of 2^-23.  gelu's erfc has |h / sqrt 2|^2 2^-22 in its argument likewise."""
    h = np.linspace(-4.6, 4.6, M)
    x = torch.zeros((M, 8), device="cuda", dtype=DT[dtype])
    x[:, 0], x[:, 1] = torch.from_numpy(h).to(DT[dtype]).cuda(), 1.0
    h = f64(x[:, 0])
    wg, wu, wd, dy = (torch.zeros(s, device="cuda", dtype=DT[dtype]) for s in ((8, 8), (8, 8), (8, 8), (M, 8)))
    wg[0, 0] = wu[0, 1] = wd[0, 0] = 1.0
    dy[:, 0] = 1.0
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    dx = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)[0]
    f, df, _ = ref.act(act, h)
    k = np.sqrt(2 / np.pi)
    t = {"silu": h, "gelu": h * h, "gelu_tanh": 2 * k * (h + 0.044715 * h ** 3), "relu": 0 * h}[act]
    rel = (np.abs(t) * 2 ** -22 + (18 + 1.2 * np.abs(t)) * 2 ** -23) if act != "relu" else 0 * h
    if act == "gelu":           # 1 + erf cancels in 64 bits too: the integral again, by erfc
        import math

        f = np.array([h_ * 0.5 * math.erfc(-h_ / math.sqrt(2)) for h_ in h])
        df = np.array([0.5 * math.erfc(-h_ / math.sqrt(2)) for h_ in h]) + h * np.exp(-h * h / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":      # as does 1 + tanh
        s = 1 / (1 + np.exp(-t))
        f, df = h * s, s + 2 * h * s * (1 - s) * k * (1 + 3 * 0.044715 * h * h)
    U, tiny = ref.U[dtype], ref.SMALLEST[dtype]
    within(y[:, 0], f, np.abs(f) * (rel + U) + tiny, "act")
    # the slope's two terms may cancel: relative to their sizes
    first = np.abs(f / np.where(h == 0, 1, h)) + np.abs(df - f / np.where(h == 0, 1, h)) if act != "relu" else np.abs(df)
    within(dx[:, 0], df, first * rel * 2 + np.abs(df) * (2 * U + U * U) + 2 * tiny, "slope")


@pytest.mark.parametrize("M", [8, 40])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DT)
def test_activations_of_huge_values(ccdc, act, dtype, M):
    """far out act(h) is h or 0 and act'(h) 1 or 0, however large h is"""
    h = torch.tensor([1e3, -1e3, 6e4, -6e4] if dtype == "float16" else [1e3, -1e3, 1e13, -1e13, 1e20, -1e20, 1e38, -1e38])
    x = torch.zeros((M, 8), device="cuda", dtype=DT[dtype])
    x[:, 0], x[:, 1] = h.repeat(M)[:M].to(DT[dtype]).cuda(), 1.0
    wg, wu, wd, dy = (torch.zeros(s, device="cuda", dtype=DT[dtype]) for s in ((8, 8), (8, 8), (8, 8), (M, 8)))
    wg[0, 0] = wu[0, 1] = wd[0, 0] = 1.0
    dy[:, 0] = 1.0
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, act=act, save=True)
    dx = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, act=act)[0]
    assert torch.equal(y[:, 0], x[:, 0].clamp(min=0)) and torch.equal(dx[:, 0], (x[:, 0] > 0).to(x.dtype))


# ---------------------------------------------------------------- products whose outputs take different ways out
@pytest.mark.parametrize("M,D,F,dtype", [(700, 512, 1111, "bfloat16"), (390, 264, 777, "float16"), (300, 256, 515, "float32")])
def test_ffn_mixed_outputs(ccdc, M, D, F, dtype):
    """one launch whose products leave partly by copies of whole tiles (widths of 16-byte multiples) and partly by plain
    stores (dw_down, whose rows of F are not), element by element"""
    rng = np.random.default_rng(M)
    x, wg, wu, wd, dy = ffn_case(rng, M, D, F, dtype, 0, 0)
    want = ref.ffn(*(f64(t) for t in (x, wg, wu, wd)), "silu", f64(dy), dtype)
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    within(y, *want["y"], "y")
    first = ccdc.ffn_backward(dy, x, wg, wu, wd, saved)
    for name, g in zip(GRADS, first):
        within(g, *want[name], name)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, ccdc.ffn_backward(dy, x, wg, wu, wd, saved)))


# ---------------------------------------------------------------- dropout: the last element numbers
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols,before", [(1, 64, 24), (4, 16, 40), (4, 16, 21), (3, 51, 100), (1, 8, 8), (5, 7, 1), (2, 64, 4)])
def test_dropout_counts_modulo_64_bits(ccdc, rows, cols, before, dtype):
    """elements are numbered modulo 2^64: offset = 2^64 - before passes the end inside the tensor"""
    offset, seed, n = (1 << 64) - before, 0xABCDEF0123456789, rows * cols
    keep = np.concatenate([ref.keep_factors(1, min(before, n), 0.4, seed, offset)[0],
                           ref.keep_factors(1, max(0, n - before), 0.4, seed, 0)[0]]).reshape(rows, cols)
    rng = np.random.default_rng(cols)
    x = tensor(rng, rows, cols, dtype)
    want = f64(x) * keep
    for off in (offset, -before):
        out = torch.full_like(x, 9.0)
        ccdc.dropout(x, 0.4, seed, off, out=out)
        within(out, want, np.abs(want) * (ref.U[dtype] + 3 * 2.0 ** -24) + ref.SMALLEST[dtype], "y")
        fused, _, stats = ccdc.residual_norm_forward(torch.zeros_like(x), x, p=0.4, seed=seed, offset=off, save=True)
        assert torch.equal(fused, out)
        _, dy, *_ = ccdc.residual_norm_backward(x, None, torch.zeros_like(x), x, stats, p=0.4, seed=seed, offset=off)
        assert torch.equal(dy, out)


# ---------------------------------------------------------------- norms: group sizes beyond the rows
@pytest.mark.parametrize("M,D", [(1, 64), (300, 64), (300, 51), (1000, 4096)])
def test_gate_row_for_more_rows_than_there_are(ccdc, M, D):
    rng = np.random.default_rng(M)
    x, y, w_post, w_pre, g = norm_case(rng, M, D, "float32", True, M)
    dout, dz = tensor(rng, M, D, "float32"), tensor(rng, M, D, "float32")
    res = []
    for per in (M, M + 1, (1 << 63) - 1):
        how = dict(w_post=w_post, w_pre=w_pre, gate=g, rows_per_gate=per, p=0.25, seed=3)
        out, z, st = ccdc.residual_norm_forward(x, y, save=True, **how)
        into = torch.full_like(g, 9.0)
        res.append((out, z, *ccdc.residual_norm_backward(dout, dz, x, y, st, dgate=into, **how)))
    for other in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(res[0], other))


# ---------------------------------------------------------------- outputs that are left out
@pytest.mark.parametrize("M,D,F,dtype", [(5, 64, 96, "bfloat16"), (300, 136, 200, "bfloat16"), (300, 136, 201, "float16"),
                                         (20, 64, 96, "float32"), (130, 72, 100, "float32")])
def test_ffn_outputs_left_out(ccdc, M, D, F, dtype):
    """every output may be NULL, and leaving some out changes no other output's bits"""
    rng = np.random.default_rng(M)
    x, wg, wu, wd, dy = ffn_case(rng, M, D, F, dtype, 0, 0)
    code, L = ccdc._block_dtype(x), ccdc.lib()
    _, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    want = ccdc.ffn_backward(dy, x, wg, wu, wd, saved)
    ws = torch.empty(L.ccdc_ffn_workspace_bytes(M, D, F, code, 1, 0), dtype=torch.uint8, device="cuda")
    for mask in range(16):
        out = [torch.full_like(w, 3.0) if mask >> i & 1 else None for i, w in enumerate(want)]
        ptr = [None if t is None else t.data_ptr() for t in out]
        status = L.ccdc_ffn_backward(M, D, F, code, code, 0, dy.data_ptr(), D, x.data_ptr(), D, wg.data_ptr(), wu.data_ptr(), D,
                                     wd.data_ptr(), F, saved.data_ptr(), ptr[0], D, *ptr[1:], ws.data_ptr(), ws.numel(), 0)
        assert status == ccdc.OK
        assert all(t is None or torch.equal(t, w) for t, w in zip(out, want)), mask
    ccdc.block_status()


@pytest.mark.parametrize("M,D", [(9, 64), (300, 51), (2, 8200)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_residual_norm_outputs_left_out(ccdc, M, D, dtype):
    rng = np.random.default_rng(M)
    per = 4
    x, y, w_post, w_pre, g = norm_case(rng, M, D, dtype, True, per)
    dout, dz = tensor(rng, M, D, dtype), tensor(rng, M, D, dtype)
    how = dict(w_post=w_post, w_pre=w_pre, gate=g, rows_per_gate=per, p=0.25, seed=3)
    out, z, st = ccdc.residual_norm_forward(x, y, save=True, **how)
    want = ccdc.residual_norm_backward(dout, dz, x, y, st, **how)
    code, L = ccdc._block_dtype(x), ccdc.lib()
    ws = torch.empty(L.ccdc_residual_norm_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    for mask in range(32):
        res = [torch.full_like(w, 3.0) if mask >> i & 1 else None for i, w in enumerate(want)]
        ptr = [None if t is None else t.data_ptr() for t in res]
        status = L.ccdc_residual_norm_backward(
            M, D, code, code, 0, dout.data_ptr(), D, dz.data_ptr(), D, x.data_ptr(), D, y.data_ptr(), D, st.data_ptr(),
            w_post.data_ptr(), w_pre.data_ptr(), g.data_ptr(), per, 1.0, 0.25, 3, 0, ptr[0], D, ptr[1], D, *ptr[2:],
            ws.data_ptr(), ws.numel(), 0)
        assert status == ccdc.OK
        assert all(t is None or torch.equal(t, w) for t, w in zip(res, want)), mask
    # z alone
    alone = torch.full_like(z, 3.0)
    status = L.ccdc_residual_norm_forward(M, D, code, 0, 1e-5, x.data_ptr(), D, y.data_ptr(), D, w_post.data_ptr(),
                                          w_pre.data_ptr(), g.data_ptr(), per, 1.0, 0.25, 3, 0, None, D, alone.data_ptr(), D,
                                          None, 0)
    assert status == ccdc.OK and torch.equal(alone, z)


# ---------------------------------------------------------------- buffers a call cannot use
def test_buffers_that_are_refused(ccdc):
    """a workspace or saved values on the host, or a view with holes, are refused before anything is launched"""
    rng = np.random.default_rng(1)
    x, wg, wu, wd, dy = ffn_case(rng, 40, 64, 96, "bfloat16", 0, 0)
    y, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    n = 1 << 22
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    _, _, st = ccdc.residual_norm_forward(x, w_pre=w, save=True)
    before = ccdc.num_kernel_launches()
    for bad in (torch.empty(n, dtype=torch.uint8), torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2],
                torch.empty(1, dtype=torch.uint8, device="cuda").expand(n)):
        with pytest.raises(ValueError, match="workspace"):
            ccdc.ffn_forward(x, wg, wu, wd, workspace=bad)
        with pytest.raises(ValueError, match="workspace"):
            ccdc.ffn_backward(dy, x, wg, wu, wd, saved, workspace=bad)
        with pytest.raises(ValueError, match="workspace"):
            ccdc.residual_norm_backward(None, dy, x, None, st, w_pre=w, workspace=bad)
        with pytest.raises(ValueError, match="saved"):
            ccdc.ffn_forward(x, wg, wu, wd, save=True, saved=bad)
        with pytest.raises(ValueError, match="saved"):
            ccdc.ffn_backward(dy, x, wg, wu, wd, bad)
    assert ccdc.num_kernel_launches() == before
    own = torch.empty(n, dtype=torch.uint8, device="cuda")
    assert torch.equal(ccdc.ffn_forward(x, wg, wu, wd, workspace=own), y)
# ---------------------------------------------------------------- feed-forward: what the backward pass keeps
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("M", [8, 40, 136])
def test_inner_gradients_are_rounded_once(ccdc, dtype, M):
    """h and u are kept in binary32: dh = da u act'(h) and du = da act(h) are off by their own rounding alone.

    x is two unit matrices side by side, so h and u are sums of two weights (more bits than the type has), and the
    weights' gradients are dh and du themselves.  Beside the rounding: the product da, within (D + 8) 2^-23 of its terms'
    size, and the elementwise work, 2^-17 of it."""
    rng = np.random.default_rng(M)
    F, D = 96, 2 * M
    eye = torch.eye(M, device="cuda", dtype=DT[dtype])
    x = torch.cat([eye, eye], 1)
    wg, wu = (tensor(rng, F, D, dtype, 1.0) for _ in range(2))
    wd, dy = tensor(rng, D, F, dtype, D ** -0.5), tensor(rng, M, D, dtype)
    _, saved = ccdc.ffn_forward(x, wg, wu, wd, save=True)
    _, dwg, dwu, _ = ccdc.ffn_backward(dy, x, wg, wu, wd, saved, grad_dtype=torch.float32)
    h, u = f64(x) @ f64(wg).T, f64(x) @ f64(wu).T
    f, df, _ = ref.act("silu", h)
    da = f64(dy) @ f64(wd)
    size = np.abs(f64(dy)) @ np.abs(f64(wd))
    for got, want, terms in ((dwg, da * u * df, size * np.abs(u)), (dwu, da * f, size * np.abs(f))):
        # rounding to the type: half a unit in the last place of the binade
        half = ref.U[dtype] * 2.0 ** np.floor(np.log2(np.maximum(np.abs(want), 1e-30)))
        slack = 1.2 * terms * ((D + 8) * 2.0 ** -23 + 2.0 ** -17)
        for at in (got[:, :M], got[:, M:]):
            within(at, want.T, (half * (1 + 2.0 ** -8) + slack + ref.SMALLEST[dtype]).T, "inner gradient")


# ---------------------------------------------------------------- waits that run out
NO_WAITS = r"""
import sys
sys.path.insert(0, sys.argv[1])
from pathlib import Path
import torch
from paper_1805_01993_b200 import build, ccdc
ccdc._LIB_PATH = build.build_variant(Path(sys.argv[2]) / "libccdc_waits.so", ("CCDC_FFN_WAIT_LIMIT=0",))

def block(M, dtype, D=136, F=200):
    x, w = torch.ones((M, D), device="cuda", dtype=dtype), torch.ones((F, D), device="cuda", dtype=dtype)
    y, saved = ccdc.ffn_forward(x, w, w, w.t().contiguous(), save=True)
    ccdc.ffn_backward(x, x, w, w, w.t().contiguous(), saved)
    torch.cuda.synchronize()
    return y

block(4, torch.float32)
ccdc.block_status()                     # no wait so far
for M, D, F in ((40, 136, 200), (700, 512, 1024), (2304, 1024, 4096)):
    for dtype in (torch.bfloat16, torch.float32):
        block(M, dtype, D, F)
        try:
            ccdc.block_status()
        except ccdc.CcdcError as e:
            assert e.status == ccdc.ESTATE
        else:
            raise AssertionError("a wait ran out and the status is good")
# the context is as good as before
assert bool((block(4, torch.float32)[0] == block(4, torch.float32)[3]).all())
x = torch.ones((40, 64), device="cuda")
assert torch.equal(ccdc.residual_norm_forward(x, x)[0], x + x)
print("bounded waits ok")
"""


def test_waits_that_run_out_are_reported(tmp_path):
    """The feed-forward kernels built with waits that run out at their first poll: every warp stops before it issues a copy
    or a product, the call ends, the status says so, and the process goes on."""
    import subprocess
    import sys

    from paper_1805_01993_b200.build import ROOT

    r = subprocess.run([sys.executable, "-c", NO_WAITS, str(ROOT), str(tmp_path)], capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "bounded waits ok" in r.stdout, r.stdout + r.stderr
