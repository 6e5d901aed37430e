"""The context that a call takes for tensors of another device than the current one, on stand-ins for tensors: no device is
needed."""
import pytest

from paper_1805_01993_b200 import ccdc

torch = pytest.importorskip("torch")


class Somewhere:
    """as much of a tensor as the choice looks at"""

    def __init__(self, index):
        self.is_cuda, self.device = index >= 0, torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def get_device(self):
        return self.device.index if self.is_cuda else -1


def test_device_of_a_call(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)        # the public call decides
    assert ccdc._elsewhere(Somewhere(1), None) is None and ccdc._elsewhere(Somewhere(-1), None) is None
    ctx = ccdc._elsewhere(Somewhere(2), None)
    assert isinstance(ctx, torch.cuda.device) and ctx.idx == 2
    with pytest.raises(ValueError, match="another device"):
        ccdc._elsewhere(Somewhere(0), type("Stream", (), {"device": torch.device("cuda", 1)})())
