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


def _rounded_once(t, group):
    """Codes of t 448 / max |t| over groups of columns, the quotient rounded to float32 once: 1 / rms drops out of y /
    scale.  (In float64 a tie is off by its rounding, which float32's takes away.)"""
    p, w = t.shape[-1], group or t.shape[-1]
    top = np.stack([np.abs(t[..., c:c + w]).max(-1) for c in range(0, p, w)], -1)
    return _codes((t * 448 / np.repeat(top, w, -1)[..., :p]).astype(np.float32).astype(np.float64))


def _near_midpoints(rng, groups):
    """Groups of 32 float32 numbers: the largest, and numbers whose quotient by it times 448 lies on a midpoint between
    two codes or within a few steps."""
    mid = (TABLE[1:] + TABLE[:-1]) / 2
    y = np.empty((groups, 32), np.float32)
    for row in y:
        top = np.float32(2.0 ** rng.integers(-20, 20) * rng.uniform(1, 2))
        row[:] = (rng.choice(mid, 32) * np.float64(top) / 448).astype(np.float32)
        for _ in range(2):
            row[:] = np.nextafter(row, rng.choice([np.float32(0), np.float32(np.inf)], 32))
        row *= rng.choice([-1, 1], 32).astype(np.float32)
        row[rng.integers(32)] = top
    return y


def test_the_inputs_tell_float32_from_one_rounding():
    """(Of the inputs, on the host.)  Float32's quotient of y by the rounded scale changes some of the codes."""
    y = _near_midpoints(np.random.default_rng(0), 512)
    scale = np.abs(y).max(-1, keepdims=True) / np.float32(448)
    assert (_rounded_once(y.astype(np.float64), 32) != _codes((y / scale).astype(np.float64))).sum() > 100


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p", [32, 64, 320, 1024, 2048, 4096, 5120, 8192, 16384, 32768])
def test_quotients_next_to_midpoints(bk, p, dtype):
    """Rows of ones have rstd 1 exactly (eps 0), so y is gamma; rows of threes a third of that."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gamma = _near_midpoints(np.random.default_rng(p), p // 32)
    want = _rounded_once(gamma.astype(np.float64), 32).reshape(-1)
    x = torch.ones(3, p, dtype=dt, device=DEV)
    x[1].neg_()
    x[2] *= 3
    out = bk.bk_rmsnorm(x, torch.tensor(gamma).reshape(-1).to(DEV), eps=0.0, keep=True, q8=32)
    assert (out.rstd[:2] == 1).all()
    for row, sign in ((0, 1.0), (1, -1.0), (2, 1.0)):
        assert np.array_equal(out.q[row].double().cpu().numpy(), sign * want), row
    scale = np.abs(gamma).max(-1) / np.float32(448)
    assert np.array_equal(out.q_scale[0].cpu().numpy(), scale) and np.array_equal(out.q_scale[1].cpu().numpy(), scale)


@pytest.mark.parametrize("gdt", ["bf16", "f32", None])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("p", [20, 100, 200, 768, 777, 1500, 3000, 5120, 6150, 9000])
def test_codes_of_ordinary_rows(bk, p, group, dtype, gdt):
    """Every code is that of the exact quotient, rounded to float32 once: of bf16 rows with a bf16 gamma some lie on a
    midpoint exactly."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(p + group)
    x = (torch.randn(40, p, generator=gen)).to(dt).to(DEV)
    r = (torch.randn(40, p, generator=gen) * 3).to(dt).to(DEV)
    gamma = None
    if gdt is not None:
        gamma = (torch.randn(p, generator=gen) * 0.2 + 1).to(torch.bfloat16 if gdt == "bf16" else torch.float32).to(DEV)
    out = bk.bk_rmsnorm(x, gamma, residual=r, eps=1e-6, q8=group)
    t = out.h.double().cpu().numpy() * (1.0 if gamma is None else gamma.double().cpu().numpy())
    got = out.q.double().cpu().numpy()
    differ = got != _rounded_once(t, group)
    # (a thread takes the largest |h gamma| from its largest |y|; two within 2^-23 of each other may change places,
    # which moves quotients that lie within 2^-23 of a midpoint: for less than one in 10^9 of these)
    assert not differ.any(), (int(differ.sum()), np.argwhere(differ)[:3])
    y, _, _ = so.rmsnorm(out.h.double().cpu().numpy(), None if gamma is None else gamma.double().cpu().numpy(), 1e-6)
    _, scales = so.quantise_e4m3(y, group)
    assert (np.abs(out.q_scale.double().cpu().numpy() - scales) <= 36 * U * scales).all()


def test_largest_out_of_range(bk):
    """Where the largest y is next to zero, or infinite, the quotient is y's own; gamma's values may lie as far apart as
    float32 allows."""
    x = torch.ones(2, 96, device=DEV)
    gamma = torch.full((96,), 1e-38, device=DEV)
    gamma[32:64] = torch.tensor(np.geomspace(1e-30, 1e38, 32), dtype=torch.float32)
    gamma[70] = float("inf")
    out = bk.bk_rmsnorm(x, gamma, eps=0.0, q8=32)
    q, s = out.q.float(), out.q_scale
    assert (s[:, 0] == 2.0 ** -126).all() and (q[:, :32] == 0.875).all()         # 1e-38 2^126 = 0.85
    want = _rounded_once(gamma[32:64].double().cpu().numpy()[None], 32)
    assert np.array_equal(q[:, 32:64].double().cpu().numpy(), np.repeat(want, 2, 0))
    assert s[:, 2].isinf().all() and q[:, 70].isnan().all()
    assert (q[:, 64:70] == 0).all() and (q[:, 71:] == 0).all()
    x[1] *= 1e-30                                                                # y as before, h gamma far smaller
    again = bk.bk_rmsnorm(x, gamma, eps=0.0, q8=32)
    assert torch.equal(again.q[0].view(torch.uint8), out.q[0].view(torch.uint8))


def test_small_rows_with_an_eps(bk):
    """h of 1e-30 under eps 1e-6: y of 1e-27, whose quotients are as exact."""
    gen = torch.Generator().manual_seed(2)
    x = (torch.randn(7, 640, generator=gen) * 1e-30).to(torch.bfloat16).to(DEV)
    out = bk.bk_rmsnorm(x, eps=1e-6, q8=64)
    assert np.array_equal(out.q.double().cpu().numpy(), _rounded_once(x.double().cpu().numpy(), 64))


@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("p", [8, 40, 64, 100, 128, 200, 256, 400])
def test_rows_that_share_a_wave(bk, p, group):
    """Several rows to a wave, the last of them missing: maxima stay within their row."""
    gen = torch.Generator().manual_seed(p)
    gamma = (torch.randn(p, generator=gen) * 0.2 + 1).to(DEV)
    size = torch.logspace(-4, 4, 29)[:, None]
    for rows in (1, 2, 3, 5, 7, 9, 15, 17, 29):
        x = (torch.randn(rows, p, generator=gen) * size[:rows]).to(DEV)
        out = bk.bk_rmsnorm(x, gamma, eps=1e-6, q8=group)
        t = x.double().cpu().numpy() * gamma.double().cpu().numpy()
        assert np.array_equal(out.q.double().cpu().numpy(), _rounded_once(t, group)), rows
        y, _, _ = so.rmsnorm(x.double().cpu().numpy(), gamma.double().cpu().numpy(), 1e-6)
        _, scales = so.quantise_e4m3(y, group)
        assert (np.abs(out.q_scale.double().cpu().numpy() - scales) <= 36 * U * scales).all()
