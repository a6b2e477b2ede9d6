"""A workspace that the caller gives is handed to kernels by its address: one in
host memory, with gaps, or on another device is refused.  CPU only."""
import pytest
import torch

bk = pytest.importorskip("paper_2210_00038_amd", reason="libbk.so not built")


class _OnDevice:
    """Stands for a device tensor."""

    def __init__(self, index, contiguous=True):
        self.device, self.index, self.contiguous = torch.device("cuda", index), index, contiguous

    is_cuda = True

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.index

    def numel(self):
        return 100

    def element_size(self):
        return 4


def test_refused(monkeypatch):
    for device in ("cuda", torch.device("cuda"), torch.device("cuda", 0)):
        with pytest.raises(ValueError, match="the workspace must be a device"):
            bk._workspace(16, device, torch.empty(64, dtype=torch.uint8))
        with pytest.raises(TypeError, match="the workspace"):
            bk._workspace(16, device, 0x1000)
    monkeypatch.setattr(bk.torch, "Tensor", _OnDevice)
    with pytest.raises(ValueError, match="contiguous"):
        bk._workspace(16, torch.device("cuda", 0), _OnDevice(0, contiguous=False))
    with pytest.raises(ValueError, match="cuda:0, not on cuda:1"):
        bk._workspace(16, torch.device("cuda", 0), _OnDevice(1))
    for device in ("cuda", torch.device("cuda"), torch.device("cuda", 1)):
        ws = _OnDevice(1)
        assert bk._workspace(16, device, ws) == (ws, 400)
    assert bk._workspace(0, "cuda", None) == (None, 0)
