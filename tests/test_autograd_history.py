"""bk_rmsnorm stands in a model's forward but is not followed by autograd: it
says so, once grad mode is on and its input requires grad."""
import warnings

import pytest
import torch

bk = pytest.importorskip("paper_2210_00038_amd", reason="libbk.so not built")


@pytest.fixture
def no_library(monkeypatch):
    """On the CPU: the device's check is passed over, and the call ends before the library's."""
    class Reached(Exception):
        pass

    def on(t, stream):
        raise Reached

    monkeypatch.setattr(bk, "_dev", lambda t, name: t)
    monkeypatch.setattr(bk, "_on", on)
    return Reached


def test_says_so(no_library):
    assert "Autograd does not follow" in " ".join(bk.bk_rmsnorm.__doc__.split())
    assert "Autograd does not follow" in " ".join(bk.bk_rmsnorm_grad.__doc__.split())
    x, leaf = torch.zeros(2, 8), torch.zeros(2, 8, requires_grad=True)
    for args in (dict(x=leaf), dict(x=x, residual=leaf), dict(x=leaf, residual=x)):
        with pytest.warns(UserWarning, match="bk_rmsnorm: autograd does not follow"), pytest.raises(no_library):
            bk.bk_rmsnorm(**args)
        with torch.no_grad(), warnings.catch_warnings(), pytest.raises(no_library):
            warnings.simplefilter("error")
            bk.bk_rmsnorm(**args)
    with warnings.catch_warnings(), pytest.raises(no_library):
        warnings.simplefilter("error")
        bk.bk_rmsnorm(x, gamma=torch.ones(8, requires_grad=True), residual=leaf.detach())


@pytest.mark.gpu
def test_results_are_the_same():
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(3, 5, 96, generator=gen).to("cuda")
    want = bk.bk_rmsnorm(x, keep=True)
    leaf = x.clone().requires_grad_()
    with pytest.warns(UserWarning, match="autograd does not follow"):
        got = bk.bk_rmsnorm(leaf, keep=True)
    assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want) if a is not None)
