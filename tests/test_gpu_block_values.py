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
