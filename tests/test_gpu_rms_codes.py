"""The e4m3 codes of bk_rmsnorm's 8-bit rows, one by one."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TABLE = so.e4m3_values()


@pytest.fixture(scope="module")
def bk():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2210_00038_amd as m
    return m


def _codes(v):
    """Values of e4m3 nearest to v (ties to the even code)."""
    mid = (TABLE[1:] + TABLE[:-1]) / 2
    lo, hi = np.searchsorted(mid, np.abs(v), side="left"), np.searchsorted(mid, np.abs(v), side="right")
    return np.copysign(TABLE[np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))], v)


def _near_midpoints(rng, groups):
    """Groups of 32 float32 numbers: the largest, and numbers whose quotient by the group's scale lies within a few
    steps of a midpoint between two codes."""
    mid = (TABLE[1:] + TABLE[:-1]) / 2
    y = np.empty((groups, 32), np.float32)
    for row in y:
        top = np.float32(2.0 ** rng.integers(-20, 20) * rng.uniform(1, 2))
        scale = top / np.float32(448)
        row[:] = (rng.choice(mid[8:], 32) * np.float64(scale)).astype(np.float32)
        for _ in range(3):
            row[:] = np.nextafter(row, rng.choice([np.float32(0), np.float32(np.inf)], 32))
        row *= rng.choice([-1, 1], 32).astype(np.float32)
        row[rng.integers(32)] = top
    return y


def _quotients(y):
    scale = np.abs(y).max(-1, keepdims=True) / np.float32(448)
    return (y / scale).astype(np.float32), scale[:, 0]


def test_the_inputs_tell_a_reciprocal_from_a_quotient():
    """(Of the inputs, on the host.)  A product with the scale's reciprocal changes some of the codes."""
    y = _near_midpoints(np.random.default_rng(0), 512)
    q, scale = _quotients(y)
    other = y * (np.float32(1) / scale[:, None])
    assert (_codes(q) != _codes(other)).sum() > 100


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p", [32, 64, 320, 1024, 2048, 4096, 16384])
def test_quotients_next_to_midpoints(bk, p, dtype):
    """Rows of ones have rstd 1 exactly (eps 0), so y is gamma: the codes are those of float32's own quotients."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gamma = _near_midpoints(np.random.default_rng(p), p // 32)
    q, scale = _quotients(gamma)
    x = torch.ones(3, p, dtype=dt, device=DEV)
    x[1].neg_()
    out = bk.bk_rmsnorm(x, torch.tensor(gamma).reshape(-1).to(DEV), eps=0.0, keep=True, q8=32)
    assert (out.rstd == 1).all()
    for row, sign in ((0, 1.0), (1, -1.0), (2, 1.0)):
        assert np.array_equal(out.q_scale[row].cpu().numpy(), scale)
        assert np.array_equal(out.q[row].double().cpu().numpy(), sign * _codes(q.astype(np.float64)).reshape(-1))


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("p", [20, 100, 768, 777, 3000, 5120, 9000])
def test_codes_of_ordinary_rows(bk, p, group):
    """Every code is the one nearest to the exact quotient, except where that lies next to a midpoint: y and the
    scale are each within 36 2^-24 of their values, the quotient's rounding and fma add two steps."""
    gen = torch.Generator().manual_seed(p + group)
    x = (torch.randn(9, p, generator=gen)).to(torch.bfloat16).to(DEV)
    r = (torch.randn(9, p, generator=gen) * 3).to(torch.bfloat16).to(DEV)
    gamma = (torch.randn(p, generator=gen) * 0.2 + 1).to(DEV)
    out = bk.bk_rmsnorm(x, gamma, residual=r, eps=1e-6, q8=group)
    y, _, _ = so.rmsnorm(out.h.double().cpu().numpy(), gamma.double().cpu().numpy(), 1e-6)
    want, scales = so.quantise_e4m3(y, group)
    v = y / np.repeat(scales, group or p, -1)[..., :p]
    mid = (TABLE[1:] + TABLE[:-1]) / 2
    near = np.abs(np.abs(v)[..., None] - mid).min(-1) <= 76 * U * np.abs(v)
    got = out.q.double().cpu().numpy()
    assert (got == want)[~near].all()
    # next to a midpoint it is one of the two beside it
    step = np.abs(got - want) <= 2.0 ** -3 * np.abs(v) * (1 + 2.0 ** -3) + 2.0 ** -9
    assert step.all() and near.mean() < 1e-3 + 2 / near.size
