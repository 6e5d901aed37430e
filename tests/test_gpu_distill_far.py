"""The distillation loss of logits far from zero: finite masks of any size, rows that lie far out themselves, the ends of the
temperature's range, and targets at a type's lowest value."""
import numpy as np
import pytest

from tests.block_reference import SMALLEST, U
from tests.test_gpu_distill import DT, ccdc, f64, reference         # noqa: F401  (ccdc: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

MASKS = [-1e4, -1.1e7, -1.2e7, -1e9, -1e10, -1e12, -1e20, -1e29, -1e30, -3e38]
PARTS = {"start": lambda V: np.s_[:V // 2], "middle": lambda V: np.s_[V // 4:3 * V // 4], "end": lambda V: np.s_[V // 2:],
         "all but three": lambda V: np.s_[:V - 3], "all but the first": lambda V: np.s_[1:], "strides": lambda V: np.s_[::2]}


def inputs(M, V, k, dtype, allowed, seed, scale=1.0):
    """logits, ids out of `allowed`, values and the loss's gradients, times `scale`"""
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(0, 2, (M, V))).to(DT[dtype]).cuda()
    ids = torch.from_numpy(rng.choice(allowed, (M, k))).int().cuda()
    values = torch.from_numpy(rng.normal(3, 2, (M, k))).to(DT[dtype]).cuda()
    return z, ids, values, torch.from_numpy((rng.random(M) + 0.5) * scale).float().cuda()


def largest(dtype):
    return float(torch.finfo(DT[dtype]).max)


def check(ccdc, z, ids, values, dloss, T, dtype):
    """Loss and gradient in two calls, in one, and in place.  Beside the reference's bound: an exponential below 2^-126 is a
    whole multiple of 2^-149 in binary32 (exp2f: two of them off at most), and 0 for 16-bit logits.  Its sum is at least that of
    the largest term, 1, or 2^-0.5 where the reference of the exponents is rounded.  So s is off by 2^-148, or by 2^-125.5."""
    under = float(dloss.max()) / T * (2.0 ** -148 if dtype == "float32" else 2.0 ** -125.5)
    loss_is, loss_tol, dz_is, dz_tol = reference(f64(z), ids.cpu().numpy(), f64(values), T, None, f64(dloss), U[dtype], SMALLEST[dtype] + under)
    loss, stats = ccdc.distill_forward(z, ids, values, save=True, temperature=T)
    dz = ccdc.distill_backward(dloss, z, ids, values, stats, temperature=T)
    same = z.clone()
    for l, g in ((loss, dz), ccdc.distill(dloss, z, ids, values, temperature=T),
                 ccdc.distill(dloss, same, ids, values, temperature=T, dlogits=same)):
        over = np.abs(f64(l) - loss_is) - loss_tol
        assert over.max() <= 0, ("loss", over.max(), over.argmax())
        over = np.abs(f64(g) - dz_is) - dz_tol
        assert over.max() <= 0, ("dz", over.max(), np.unravel_index(over.argmax(), over.shape))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("part", PARTS)
@pytest.mark.parametrize("V", [600, 4099, 65536])         # one block to a row, and clusters of blocks
def test_finite_masks(ccdc, V, part, dtype):
    """a row for each mask; targets beside it, and everywhere"""
    masks = sorted({max(m, -largest(dtype)) for m in MASKS})
    masked = np.zeros(V, bool)
    masked[PARTS[part](V)] = True
    for allowed in (np.flatnonzero(~masked), np.arange(V)):
        for T in (0.1, 1.0, 2.0):
            if len(allowed) == V and T < 1:             # a masked target's loss, up to 3e38 / T, would leave binary32
                continue
            z, ids, values, dloss = inputs(len(masks), V, 5, dtype, allowed, V)
            for m, mask in enumerate(masks):
                z[m, torch.from_numpy(masked).cuda()] = mask
            check(ccdc, z, ids, values, dloss, T, dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [600, 65536])
def test_rows_that_lie_far_out(ccdc, V, dtype):
    """every logit far out, on either side: the largest share the probability alike"""
    far = sorted({min(max(v, -largest(dtype)), largest(dtype)) for m in MASKS for v in (m, -m)})
    z, ids, values, dloss = inputs(2 * len(far), V, 5, dtype, np.arange(V), 3)
    for i, v in enumerate(far):
        z[2 * i] = v
        z[2 * i + 1] = torch.where(torch.arange(V, device="cuda") % 7 == 3, v, v / 2)
    check(ccdc, z, ids, values, dloss, 2.0, dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [33, 600, 65536])
@pytest.mark.parametrize("T", [1e-6, 2e-5, 1e6])
def test_ends_of_the_temperature(ccdc, T, V, dtype):
    """gradients scaled with T, so that 16 bits hold them"""
    z, ids, values, dloss = inputs(6, V, 4, dtype, np.arange(V), 7, T)
    z[1] = 20000.0                                      # equal logits far out in units of T
    z[2, :V // 2] = -20000.0
    z[3, V // 2:] = -60000.0
    z[4] = z[4].sign() * 2.0                            # ties
    check(ccdc, z, ids, values, dloss, T, dtype)

@pytest.mark.parametrize("dtype", DT)
def test_targets_at_the_lowest_value(ccdc, dtype):
    """the formula's loss, which is finite; minus infinity alone gives an infinite one"""
    z, ids, values, dloss = inputs(4, 500, 6, dtype, np.arange(250), 9)
    z[:, 250:] = torch.finfo(DT[dtype]).min
    ids[:, 0] = 400
    check(ccdc, z, ids, values, dloss, 2.0, dtype)
    check(ccdc, z, ids, values, dloss, 1e6, dtype)
    z[:, 250:] = -float("inf")
    assert bool((ccdc.distill_forward(z, ids, values, temperature=2.0) == float("inf")).all())
