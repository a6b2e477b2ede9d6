"""The binding needs no undocumented name of torch: without them it takes the
documented way to the same stream."""
import importlib.util

import pytest
import torch

bk = pytest.importorskip("paper_2210_00038_amd", reason="libbk.so not built")
UNDOCUMENTED = ("_cuda_getCurrentRawStream", "_cuda_getDevice")


@pytest.fixture
def other(monkeypatch):
    """The binding as it loads where torch lacks these names."""
    keep = {n: getattr(torch._C, n) for n in UNDOCUMENTED if hasattr(torch._C, n)}
    for n in UNDOCUMENTED:
        monkeypatch.delattr(torch._C, n, raising=False)
    spec = importlib.util.spec_from_file_location("bk_without_names", bk.__file__)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    for n, f in keep.items():
        monkeypatch.setattr(torch._C, n, f, raising=False)
    return m


def test_loads_and_asks_the_documented_way(other, monkeypatch):
    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream())
    assert other._raw_stream(torch.zeros(1)) == 77
    assert other._device_now is torch.cuda.current_device
    with open(bk.__file__) as f:
        text = f.read()
    assert all(text.count(n) == 1 for n in UNDOCUMENTED)


@pytest.mark.gpu
def test_same_results(other):
    x = torch.randn(7, 300, generator=torch.Generator().manual_seed(1)).to("cuda")
    want = bk.bk_rmsnorm(x, keep=True)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        assert other._raw_stream(x) == bk._raw_stream(x) == s.cuda_stream
        got = other.bk_rmsnorm(x, keep=True)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want) if a is not None)
