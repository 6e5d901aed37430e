"""Experts, distillation and 8-bit products on the host: refusals of the C entries (checked before any launch, so no device is
needed) and of the Python calls."""
import pytest

from paper_1805_01993_b200 import build as ccdc_build
from paper_1805_01993_b200 import ccdc

torch = pytest.importorskip("torch")

P = 1 << 12         # a 16-byte aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def built():
    ccdc_build.build_library()


def refuses(call, status, *cases):
    for bad in cases:
        assert call(**bad) == status, bad


def test_expert_refusals():
    L = ccdc.lib()

    def sort(M=4, k=2, experts=8, size=4, ids=P, offsets=P, slots=P, places=P):
        return L.ccdc_expert_sort(M, k, experts, size, ids, offsets, slots, places, None)

    refuses(sort, ccdc.EINVAL, dict(M=-1), dict(k=0), dict(experts=0), dict(size=2), dict(ids=None), dict(offsets=None), dict(slots=None),
            dict(places=None), dict(ids=P + 2), dict(ids=P + 4, size=8), dict(offsets=P + 1), dict(slots=P + 2), dict(places=P + 3))
    refuses(sort, ccdc.ESIZE, dict(M=1 << 30), dict(experts=4097), dict(M=1 << 40))

    def dispatch(M=4, k=2, D=8, dtype=ccdc.BF16, x=P, ldx=8, slots=P, places=P, xs=P, ldxs=8):
        return L.ccdc_expert_dispatch(M, k, D, dtype, x, ldx, slots, places, xs, ldxs, None)

    refuses(dispatch, ccdc.EINVAL, dict(M=-1), dict(k=0), dict(D=0), dict(dtype=ccdc.I32), dict(x=None), dict(ldx=7), dict(slots=None),
            dict(places=None), dict(xs=None), dict(ldxs=7))
    refuses(dispatch, ccdc.ESIZE, dict(M=1 << 30), dict(D=(1 << 20) + 1, ldx=1 << 21, ldxs=1 << 21))
    assert dispatch(M=0, x=None, xs=None, slots=None, places=None) == ccdc.OK

    def combine(M=4, k=2, D=8, dtype=ccdc.F16, ys=P, ldys=8, places=P, weights=P, wt=ccdc.F32, y=P, ldy=8):
        return L.ccdc_expert_combine(M, k, D, dtype, ys, ldys, places, weights, wt, y, ldy, None)

    refuses(combine, ccdc.EINVAL, dict(M=-1), dict(k=0), dict(D=0), dict(dtype=7), dict(ys=None), dict(ldys=7), dict(places=None),
            dict(wt=ccdc.BF16), dict(y=None), dict(ldy=7))
    assert combine(M=0) == ccdc.OK

    def back(M=4, k=2, D=8, dtype=ccdc.F32, dy=P, lddy=8, ys=P, ldys=8, slots=P, places=P, weights=P, wt=ccdc.F32, dys=P, lddys=8, dw=P):
        return L.ccdc_expert_combine_backward(M, k, D, dtype, dy, lddy, ys, ldys, slots, places, weights, wt, dys, lddys, dw, None)

    refuses(back, ccdc.EINVAL, dict(M=-1), dict(k=0), dict(D=0), dict(dtype=7), dict(dy=None), dict(lddy=7), dict(ys=None), dict(ldys=7),
            dict(slots=None), dict(places=None), dict(wt=ccdc.BF16), dict(dys=None, dw=None), dict(lddys=7))
    assert back(M=0) == ccdc.OK


def test_distill_refusals():
    L = ccdc.lib()

    def call(M=2, V=8, k=3, dtype=ccdc.BF16, z=P, ldz=8, size=4, ids=P, vt=ccdc.F32, values=P, lse=None, T=1.0, dloss=P, loss=P,
             stats=None, dz=P, lddz=8):
        return L.ccdc_distill(M, V, k, dtype, z, ldz, size, ids, vt, values, lse, T, dloss, loss, stats, dz, lddz, None)

    refuses(call, ccdc.EINVAL, dict(M=-1), dict(V=0), dict(k=0), dict(dtype=ccdc.I32), dict(z=None), dict(ldz=7), dict(size=3),
            dict(ids=None), dict(ids=P + 2), dict(vt=ccdc.F16), dict(values=None), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")),
            dict(T=float("inf")), dict(T=1e-7), dict(dloss=None), dict(loss=None), dict(loss=None, dz=None), dict(lddz=7), dict(stats=P + 4))
    refuses(call, ccdc.ESIZE, dict(k=1025), dict(V=1 << 31, ldz=1 << 31, lddz=1 << 31))
    assert call(M=0) == ccdc.OK


def test_fp8_refusals():
    L = ccdc.lib()

    def quantise(groups=1, M=4, K=40, rows=1, dtype=ccdc.BF16, x=P, xg=0, ldx=40, q=P, qg=0, ldq=48, s=P):
        return L.ccdc_quantize_fp8(groups, M, K, rows, dtype, x, xg, ldx, q, qg, ldq, s, 0, 1, 1, None)

    refuses(quantise, ccdc.EINVAL, dict(groups=-1), dict(M=-1), dict(K=0), dict(rows=2), dict(dtype=ccdc.I32), dict(groups=2), dict(x=None),
            dict(ldx=39), dict(q=None), dict(q=P + 8), dict(ldq=39), dict(ldq=40), dict(s=None), dict(groups=2, rows=128, qg=8))
    refuses(quantise, ccdc.ESIZE, dict(groups=1 << 17, rows=128), dict(K=(1 << 23) + 1))
    assert quantise(M=0) == ccdc.OK and quantise(groups=0, rows=128) == ccdc.OK

    def product(M=4, N=20, K=40, E=2, x=P, ldx=48, xs=P, w=P, we=960, ldw=48, ws=P, offsets=P, y=P, yt=ccdc.BF16, ldy=20):
        return L.ccdc_matmul_fp8(M, N, K, E, x, ldx, xs, 1, 4, w, we, ldw, ws, offsets, y, yt, ldy, None)

    refuses(product, ccdc.EINVAL, dict(M=-1), dict(N=0), dict(K=0), dict(E=0), dict(x=None), dict(x=P + 8), dict(ldx=40), dict(ldx=32),
            dict(xs=None), dict(w=None), dict(w=P + 4), dict(ldw=56), dict(ldw=32), dict(we=968), dict(we=-16), dict(we=0), dict(ws=None),
            dict(offsets=None), dict(y=None), dict(yt=ccdc.I32), dict(ldy=19))
    refuses(product, ccdc.ESIZE, dict(M=(1 << 30) + 1), dict(N=(1 << 22) + 1, ldy=1 << 23), dict(K=(1 << 23) + 1), dict(E=1025))
    assert product(M=0) == ccdc.OK


def test_python_refusals_need_no_device():
    x, ids = torch.zeros((2, 8)), torch.zeros((2, 3), dtype=torch.int32)
    order = ccdc.ExpertOrder(torch.zeros(3, dtype=torch.int32), ids.view(-1), ids)
    for bad in (ids.float(), ids[0], ids.short(), ids.t(), ids.bool()):
        with pytest.raises(ValueError, match="int32 or int64"):
            ccdc.expert_sort(bad, 2)
    with pytest.raises(ValueError, match="CUDA"):
        ccdc.expert_sort(ids, 2)
    for call in (lambda: ccdc.expert_dispatch(x, order), lambda: ccdc.expert_combine(x, order), lambda: ccdc.distill_forward(x, ids, x[:, :3]),
                 lambda: ccdc.expert_combine_backward(x, x, order, None), lambda: ccdc.quantize_fp8(x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="block_rows"):
        ccdc.quantize_fp8(x, 64)
    q = torch.zeros((4, 16), dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="CUDA"):
        ccdc.matmul_fp8(q, x, q, x)
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        ccdc.matmul_fp8(x, x, q, x)
