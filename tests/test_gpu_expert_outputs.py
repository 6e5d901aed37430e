"""The sort by expert into given tensors, its refusals, and counts beyond what the calls take."""
import numpy as np
import pytest

from tests.test_gpu_expert import ccdc, draw_ids, order_of          # noqa: F401  (ccdc: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("M,k,E,drop", [(1, 1, 1, 0.0), (11, 3, 4, 0.2), (700, 8, 60, 0.1), (3, 2, 4096, 0.0), (5000, 8, 33, 0.1), (0, 4, 6, 0.0)])
@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_into_given_tensors(ccdc, M, k, E, drop, kind):
    """they are what is returned, and nothing beside them is written"""
    ids = draw_ids(np.random.default_rng(M + E), M, k, E, drop)
    guarded = [torch.full((n + 10,), 77, dtype=torch.int32, device="cuda") for n in (E + 1, M * k, M * k)]
    offsets, slots, places = (t[5:-5] for t in guarded)
    places = places.view(M, k)
    got = ccdc.expert_sort(torch.from_numpy(ids).to(kind).cuda(), E, offsets, slots, places)
    assert got.offsets is offsets and got.slots is slots and got.places is places
    for a, b in zip(got, order_of(ids, E)):
        assert np.array_equal(a.cpu().numpy(), b)
    assert all(bool((t[:5] == 77).all()) and bool((t[-5:] == 77).all()) for t in guarded)
    again = ccdc.expert_sort(torch.from_numpy(ids).to(kind).cuda(), E, slots=slots)             # some given, some made
    assert again.slots is slots and torch.equal(again.places, places) and torch.equal(again.offsets, offsets)


def test_refusals(ccdc):
    ids = torch.zeros((6, 2), dtype=torch.int32, device="cuda")

    def empty(*shape, dtype=torch.int32, device="cuda"):
        return torch.empty(shape, dtype=dtype, device=device)

    for name, bad in (("offsets", (empty(4), empty(6), empty(5, dtype=torch.int64), empty(5, device="cpu"), empty(10)[::2])),
                      ("slots", (empty(11), empty(13), empty(12, dtype=torch.float32), empty(12, device="cpu"), empty(24)[::2])),
                      ("places", (empty(6, 1), empty(2, 6), empty(12), empty(6, 2, dtype=torch.int64), empty(2, 6).t(),
                                  empty(6, 2, device="cpu")))):
        for t in bad:
            with pytest.raises(ValueError, match=name):
                ccdc.expert_sort(ids, 4, **{name: t})
    for n in (4097, 1 << 31, (1 << 32) + 4):            # also counts whose low 32 bits look like few experts
        with pytest.raises(ccdc.CcdcError) as e:
            ccdc.expert_sort(ids, n)
        assert e.value.status == ccdc.ESIZE
    for n in (0, -1, -4):
        with pytest.raises(ccdc.CcdcError) as e:
            ccdc.expert_sort(ids, n)
        assert e.value.status == ccdc.EINVAL
    # a stack of weights whose number's low 32 bits are 1
    x, xs = ccdc.quantize_fp8(torch.ones((4, 128), device="cuda"))
    w, ws = ccdc.quantize_fp8(torch.ones((1, 16, 128), device="cuda"), 128)
    with pytest.raises(ccdc.CcdcError) as e:
        ccdc.matmul_fp8(x, xs, w.expand((1 << 32) + 1, 16, 128), ws, offsets=empty(2))
    assert e.value.status == ccdc.ESIZE
