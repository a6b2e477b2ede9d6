"""Refusals of kept affine layers in the binding.  A kept layer takes its sizes
from P alone, so tensors that do not fit P would be read or written past their
end.  On the CPU: the check of the device is replaced, and the library by one
that fails if it is called.  On the GPU: a kept layer that still names its tokens."""
import pytest
import torch

bk = pytest.importorskip("paper_2210_00038_amd", reason="libbk.so not built")


@pytest.fixture
def host_tensors(monkeypatch):
    def dev(t, name):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a torch.Tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t

    monkeypatch.setattr(bk, "_dev", dev)


def _spec(**kw):
    s = {"kind": bk.BK_NORM_AFFINE, "kept": True, "bias": True, "P": torch.zeros(3, 8), "Pb": torch.zeros(3, 8),
         "G": torch.zeros(8), "Gb": torch.zeros(8)}
    s.update(kw)
    return s


@pytest.mark.parametrize("kw,said", [
    (dict(P=None), "needs P"), (dict(Pb=None), "Pb"), (dict(P=torch.zeros(24)), "P must be float32"),
    (dict(P=torch.zeros(3, 8, dtype=torch.bfloat16)), "P must be float32"),
    (dict(Pb=torch.zeros(3, 7)), "Pb of a kept layer"), (dict(Pb=torch.zeros(2, 8)), "Pb of a kept layer"),
    (dict(Pb=torch.zeros(3, 8, dtype=torch.bfloat16)), "Pb of a kept layer"), (dict(Pb=torch.zeros(8, 3).T), "contiguous"),
    (dict(G=torch.zeros(7)), "G of a kept layer"), (dict(G=torch.zeros(8, dtype=torch.bfloat16)), "G of a kept layer"),
    (dict(G=torch.zeros(16)[::2]), "contiguous"), (dict(G=torch.zeros(8, device="meta")), "G of a kept layer"),
    (dict(Gb=torch.zeros(4)), "Gb of a kept layer"), (dict(Gb=torch.zeros(8, dtype=torch.float64)), "Gb of a kept layer"),
])
def test_refused(host_tensors, kw, said):
    with pytest.raises(ValueError, match=said):
        bk.make_layers([_spec(**kw)])


def test_taken(host_tensors):
    arr = bk.make_layers([_spec(), _spec(G=None, Gb=None), _spec(bias=False, Pb=None, Gb=None), _spec(G=torch.zeros(1, 8))])
    assert [arr[k].p for k in range(4)] == [8] * 4 and arr[0].flags == bk.BK_LAYER_KEPT | bk.BK_LAYER_BIAS


class _Untouched:
    """A library of which only the workspace queries may be called."""

    def __getattr__(self, name):
        def call(*_):
            assert name.endswith("_workspace_size"), name
            return 0

        return call


def test_more_samples_than_kept(host_tensors, monkeypatch):
    arr = bk.make_layers([_spec(), _spec(P=torch.zeros(2, 8), Pb=torch.zeros(2, 8))])
    monkeypatch.setattr(bk, "lib", _Untouched())
    C = torch.zeros(4)
    for call in (lambda n, B: bk.bk_layer_norms(arr, n, bk.BK_F32, B, C, stream=0),
                 lambda n, B: bk.bk_weighted_grads(arr, n, C, bk.BK_F32, B, stream=0),
                 lambda n, B: bk.bk_private_grad(arr, n, bk.BK_F32, B, 0, 1.0, 0.0, 0.0, 1, 0, C, C, stream=0),
                 lambda n, B: bk.bk_private_grad_noalloc(arr, n, bk.BK_F32, B, 0, 1.0, 0.0, 0.0, 1, 0, C, C, stream=0)):
        for n, B in ((2, 3), (1, 4)):
            with pytest.raises(ValueError, match="holds"):
                call(n, B)
    assert bk._batch(arr, 1, 3) == 3 and bk._batch(arr, 2, 2) == 2


@pytest.mark.gpu
def test_tokens_are_not_read():
    """T may be any, and x and g NULL, as the header says."""
    gen = torch.Generator().manual_seed(3)
    B, p = 4, 300
    P, Pb = (torch.randn(B, p, generator=gen).to("cuda") for _ in range(2))
    got = []
    for T in (0, 1, 77):
        G, Gb = torch.empty(p, device="cuda"), torch.empty(p, device="cuda")
        arr = bk.make_layers([{"kind": bk.BK_NORM_AFFINE, "kept": True, "bias": True, "P": P, "Pb": Pb, "G": G, "Gb": Gb}])
        arr[0].T = T
        n, C = torch.empty(1, B, device="cuda"), torch.empty(B, device="cuda")
        bk.bk_private_grad(arr, 1, bk.BK_BF16, B, bk.BK_CLIP_ABADI, 1.0, 0.0, 0.0, 1, 0, n, C)
        got.append([n, C, G, Gb])
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))
    norm = (P.double().square().sum(1) + Pb.double().square().sum(1)).sqrt()
    assert torch.allclose(got[0][1].double(), (1 / norm).clamp(max=1), rtol=1e-5)
    assert torch.allclose(got[0][2].double(), (got[0][1].double()[:, None] * P.double()).sum(0), rtol=1e-5, atol=1e-6)
