"""Block operators on the host: the generator's published vectors, the refusals of the C entries (checked before
any launch, so no device is needed) and of the Python calls."""
import ctypes

import numpy as np
import pytest

from paper_1805_01993_b200 import build as ccdc_build
from paper_1805_01993_b200 import ccdc
from tests import block_reference as ref

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def built():
    ccdc_build.build_library()


def test_reference_generator_against_published_vectors():
    """known answers published with the generator (Random123, philox4x32 in 10 rounds)"""
    assert ref.philox_words([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert ref.philox_words([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.philox_words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_reference_gradients_by_differences():
    """the formulas' gradients that the device is compared with, against central differences in 64 bits"""
    rng = np.random.default_rng(0)
    x, wg, wu, wd, dy = (rng.normal(size=s) for s in ((3, 5), (7, 5), (7, 5), (5, 7), (3, 5)))
    for act in ("silu", "gelu", "gelu_tanh"):
        r = ref.ffn(x, wg, wu, wd, act, dy, "float32")
        for k, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
            args = [x, wg, wu, wd]
            d = rng.normal(size=args[k].shape)
            up, down = (ref.ffn(*[a + s * 1e-5 * d if i == k else a for i, a in enumerate(args)], act, None, "float32")["y"][0]
                        for s in (1, -1))
            assert abs((dy * (up - down)).sum() / 2e-5 - (r[name][0] * d).sum()) < 1e-6


P = 1 << 12         # a 16-byte aligned address that is never read


def test_dropout_refusals():
    L = ccdc.lib()

    def call(rows=2, cols=8, dtype=ccdc.F32, x=P, ldx=8, y=P, ldy=8, p=0.5):
        return L.ccdc_dropout(rows, cols, dtype, x, ldx, y, ldy, p, 1, 0, None)

    for bad in (dict(rows=-1), dict(cols=-1), dict(dtype=ccdc.I32), dict(dtype=9), dict(x=None), dict(y=None), dict(ldx=7),
                dict(ldy=7), dict(p=-0.1), dict(p=1.5), dict(p=float("nan"))):
        assert call(**bad) == ccdc.EINVAL, bad
    assert call(rows=1 << 40, cols=1 << 10, ldx=1 << 10, ldy=1 << 10) == ccdc.ESIZE
    assert call(rows=0, x=None, y=None) == ccdc.OK and call(cols=0) == ccdc.OK


def test_residual_norm_refusals():
    L = ccdc.lib()

    def forward(M=2, D=8, dtype=ccdc.BF16, kind=0, eps=1e-5, x=P, ldx=8, y=P, ldy=8, w_post=P, w_pre=P, gate=P, per=2,
                alpha=1.0, p=0.0, out=P, ldo=8, z=P, ldz=8, stats=P):
        return L.ccdc_residual_norm_forward(M, D, dtype, kind, eps, x, ldx, y, ldy, w_post, w_pre, gate, per, alpha, p, 0, 0,
                                            out, ldo, z, ldz, stats, None)

    for bad in (dict(M=-1), dict(D=0), dict(dtype=ccdc.I32), dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None),
                dict(ldx=7), dict(ldy=7), dict(ldo=7), dict(ldz=7), dict(y=None), dict(w_pre=None), dict(z=None), dict(per=0),
                dict(p=2.0), dict(alpha=float("nan")), dict(out=None, z=None, w_pre=None), dict(stats=P + 4)):
        assert forward(**bad) == ccdc.EINVAL, bad
    assert forward(D=32769, ldx=32769, ldy=32769, ldo=32769, ldz=32769) == ccdc.ESIZE
    assert forward(M=0) == ccdc.OK

    def backward(M=2, D=8, dtype=ccdc.BF16, grad=ccdc.F32, kind=0, dout=P, lddout=8, dz=P, lddz=8, x=P, ldx=8, y=P, ldy=8,
                 stats=P, w_post=P, w_pre=P, gate=P, per=2, p=0.0, dx=P, lddx=8, dy=P, lddy=8, dw_post=P, dw_pre=P, dgate=P):
        return L.ccdc_residual_norm_backward(M, D, dtype, grad, kind, dout, lddout, dz, lddz, x, ldx, y, ldy, stats, w_post,
                                             w_pre, gate, per, 1.0, p, 0, 0, dx, lddx, dy, lddy, dw_post, dw_pre, dgate, None,
                                             0, None)

    for bad in (dict(M=-1), dict(grad=ccdc.F16), dict(grad=ccdc.I32), dict(lddout=7), dict(lddz=7), dict(lddx=7), dict(lddy=7),
                dict(stats=None), dict(dout=None, dz=None), dict(dz=None), dict(w_pre=None), dict(w_post=None),
                dict(gate=None), dict(y=None), dict(p=-1.0)):
        assert backward(**bad) == ccdc.EINVAL, bad
    assert L.ccdc_residual_norm_workspace_bytes(-1, 8) == 0 and L.ccdc_residual_norm_workspace_bytes(4, 0) == 0


def test_ffn_refusals():
    L = ccdc.lib()

    def forward(M=2, D=8, F=16, dtype=ccdc.BF16, act=0, x=P, ldx=8, wg=P, wu=P, ldw=8, wd=P, ldd=16, y=P, ldy=8, saved=P,
                ws=P, size=1 << 30):
        return L.ccdc_ffn_forward(M, D, F, dtype, act, x, ldx, wg, wu, ldw, wd, ldd, y, ldy, saved, ws, size, None)

    for bad in (dict(M=-1), dict(D=0), dict(F=0), dict(dtype=ccdc.I32), dict(act=-1), dict(act=4), dict(x=None), dict(wg=None),
                dict(wu=None), dict(wd=None), dict(y=None), dict(ldx=7), dict(ldw=7), dict(ldd=15), dict(ldy=7),
                dict(saved=P + 2), dict(ws=P + 8), dict(ws=None)):
        assert forward(**bad) == ccdc.EINVAL, bad
    assert forward(size=16) == ccdc.ESIZE and forward(M=1 << 22) == ccdc.ESIZE
    assert forward(M=0, x=None, y=None) == ccdc.OK

    def backward(M=2, D=8, F=16, dtype=ccdc.BF16, grad=ccdc.F32, act=0, dy=P, lddy=8, x=P, ldx=8, wg=P, wu=P, ldw=8, wd=P,
                 ldd=16, saved=P, dx=P, lddx=8, dwg=P, dwu=P, dwd=P, ws=P, size=1 << 30):
        return L.ccdc_ffn_backward(M, D, F, dtype, grad, act, dy, lddy, x, ldx, wg, wu, ldw, wd, ldd, saved, dx, lddx, dwg, dwu,
                                   dwd, ws, size, None)

    for bad in (dict(M=-1), dict(grad=ccdc.F16), dict(dtype=ccdc.F32, grad=ccdc.BF16), dict(dy=None), dict(x=None),
                dict(saved=None), dict(lddy=7), dict(lddx=7), dict(ldw=7), dict(ldd=15), dict(ws=None), dict(act=7)):
        assert backward(**bad) == ccdc.EINVAL, bad
    assert backward(size=16) == ccdc.ESIZE
    assert L.ccdc_ffn_saved_bytes(4, 16, ccdc.I32) == 0 and L.ccdc_ffn_workspace_bytes(4, 0, 16, ccdc.F32, 0, 0) == 0


def test_python_refusals_need_no_device():
    x = torch.zeros((2, 8))
    with pytest.raises(ValueError, match="CUDA"):
        ccdc.dropout(x, 0.5, 1)
    with pytest.raises(ValueError, match="2-D"):
        ccdc.dropout(x[0], 0.5, 1)
    with pytest.raises(ValueError, match="contiguous columns"):
        ccdc.dropout(x.t(), 0.5, 1)
    with pytest.raises(ValueError, match="CUDA"):
        ccdc.residual_norm_forward(x)
    with pytest.raises(ValueError, match="CUDA"):
        ccdc.ffn_forward(x, x, x, x.t().contiguous())


def test_buffers_are_one_piece_of_the_tensors_device():
    like = torch.zeros(4)
    t = torch.empty(64, dtype=torch.int16)
    assert ccdc._buffer(t, "workspace", like, 128) == (t.data_ptr(), 128)
    assert ccdc._buffer(torch.empty(0), "workspace", like)[1] == 0
    for bad in (t[::2], t.view(8, 8).t(), t[:1].expand(64), t[1:]):
        with pytest.raises(ValueError, match="workspace"):
            ccdc._buffer(bad, "workspace", like, 128 if bad.is_contiguous() else 0)


def test_plans_refuse_the_block_types():
    for dtype in (ccdc.BF16, ccdc.F16):
        h = ctypes.c_void_p()
        assert ccdc.lib().ccdc_plan(4, 2, 12, 4, 8, dtype, ctypes.byref(h)) == ccdc.EINVAL and not h.value
