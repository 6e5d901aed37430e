"""Counts beyond 32 bits are refused by the Python calls: tensors without memory, so no device is needed."""
import pytest

from paper_1805_01993_b200 import build as ccdc_build
from paper_1805_01993_b200 import ccdc

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def built():
    ccdc_build.build_library()


@pytest.mark.parametrize("k", [1 << 31, (1 << 32) + 2])      # the second's low 32 bits are 2
def test_slots_beyond_32_bits(k):
    ids = torch.empty((1, k), dtype=torch.int32, device="meta")
    order = ccdc.ExpertOrder(None, ids.view(-1), ids)
    for call in (lambda: ccdc._ids(ids, "ids", ids), lambda: ccdc._order(order, ids)):
        with pytest.raises(ccdc.CcdcError) as e:
            call()
        assert e.value.status == ccdc.ESIZE
    small = torch.empty((5, 3), dtype=torch.int64, device="meta")
    assert ccdc._ids(small, "ids", small) == 8
