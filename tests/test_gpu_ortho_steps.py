"""Orthogonalisation with more steps than five, and of updates that lack
directions (low rank, equal rows, singular values down to 1e-9 of the largest),
in all three forms: in one workgroup, thin, and general.

Bounds.  Exact singular values stay within the largest value that the
polynomials reach.  That value is an extremum (of slope zero) of each
polynomial used here, so what the roundings of one step add does not grow in the
next: the spectral norm of a rounding of X is at most u |X|_F <= u sqrt(m) top,
with u = 2^-11 for fp16 operands and 2^-21 for the others, once for X, once for
Bm X, and twice that for the float32 sums and the store.  The thin form multiplies
X by float32 products P of several steps' polynomials, of a gain of 2^9 at most: an
entry of P is off by 2^-24 2^9, so u = 2^-15 there.

Directions that U lacks are filled by rounding errors, in any arithmetic, and
grow with the steps.  What has one value is the part within U's own row and column
space, and only where the polynomials contract (the cubic and the quintic that
converge to 1): it may be off by four times what the same steps leave in plain
float32 products of X, plus float32 sums (4e-6); in the thin form also by u = 2^-15
for each P, and as much for the sums of its product with X."""
import functools

import numpy as np
import pytest
import torch

from oracle import step_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda"
SUMS = 4e-6
CUBIC, QUINTIC = (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)
SMALL, THIN, GENERAL = [(16, 768), (64, 96), (400, 33)], [(16, 4096), (48, 3000), (2000, 64), (900, 33)], [(100, 201), (300, 70)]


@pytest.fixture(scope="module")
def bk():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2210_00038_amd as m
    return m


def _update(kind, d, p):
    rng = np.random.default_rng(d * 31 + p + len(kind))
    m, n = min(d, p), max(d, p)
    if kind == "full":
        U = rng.standard_normal((m, n))
    elif kind == "equal rows":
        U = rng.standard_normal((m, n))
        U[m // 2] = U[0]
    elif kind == "falling":
        left, _ = np.linalg.qr(rng.standard_normal((m, m)))
        right, _ = np.linalg.qr(rng.standard_normal((n, m)))
        U = (left * np.logspace(0, -9, m)) @ right.T
    else:
        r = int(kind.split()[1])
        U = rng.standard_normal((m, r)) @ rng.standard_normal((r, n))
    return np.ascontiguousarray(U if d <= p else U.T, np.float32)


def _orthogonalized(bk, U, prec, steps, coef=None):
    O = torch.full(U.shape, float("nan"), device=DEV)
    bk.bk_orthogonalize(bk.make_matrices([{"G": torch.tensor(U).to(DEV), "O": O}]), 1, prec, steps=steps, coef=coef)
    return O.double().cpu().numpy()


@functools.lru_cache(None)
def _top(steps, coef):
    """The largest value that the polynomials reach from [0, 1], after `steps` of them."""
    a, b, c = coef or so.NS_QUINTIC
    s = 1.0
    for _ in range(steps):
        x = np.linspace(0, s, 100001)
        s = np.abs(x * (a + x * x * (b + x * x * c))).max()
    return s


@pytest.mark.parametrize("kind", ["rank 1", "rank 8", "equal rows", "falling", "full"])
@pytest.mark.parametrize("d,p", SMALL + THIN + GENERAL)
def test_bounded(bk, d, p, kind):
    U = _update(kind, d, p)
    m = min(d, p)
    for prec in (bk.BK_NS_F16, bk.BK_NS_F32):
        u = 2.0 ** -15 if (d, p) in THIN else 2.0 ** -11 if prec == bk.BK_NS_F16 and m > 64 else 2.0 ** -21
        for coef in (None, CUBIC, QUINTIC):
            for steps in (5, 8, 12, 18, 20, 32, 48, 64):
                O = _orthogonalized(bk, U, prec, steps, coef)
                assert np.isfinite(O).all(), (prec, coef, steps)
                top = np.linalg.norm(O, 2)
                assert top <= _top(steps, coef) * (1 + 4 * u * np.sqrt(m)), (prec, coef, steps, top)


def _float32_steps(U, steps, coef):
    X = U if U.shape[0] <= U.shape[1] else U.T
    X = (X / (np.linalg.norm(X.astype(np.float64)) + 1e-7)).astype(np.float32)
    a, b, c = (np.float32(v) for v in coef or so.NS_QUINTIC)
    for _ in range(steps):
        A = X @ X.T
        X = (a * np.eye(len(A), dtype=np.float32) + b * A + c * (A @ A)) @ X
    return X if U.shape[0] <= U.shape[1] else X.T


@pytest.mark.parametrize("kind", ["rank 8", "equal rows", "full"])
@pytest.mark.parametrize("d,p", SMALL + THIN + GENERAL)
def test_own_directions(bk, d, p, kind):
    U = _update(kind, d, p)
    left, s, right = np.linalg.svd(U.astype(np.float64), full_matrices=False)
    r = int((s > 1e-5 * s[0]).sum())
    assert r == {"rank 8": 8, "equal rows": min(d, p) - 1, "full": min(d, p)}[kind]
    inside = lambda O: left[:, :r].T @ O @ right[:r].T       # noqa: E731
    for coef, steps in ((CUBIC, 8), (CUBIC, 20), (CUBIC, 48), (CUBIC, 64), (QUINTIC, 16), (QUINTIC, 32), (QUINTIC, 64)):
        want = inside(so.orthogonalize(U, steps, [coef] * steps))
        plain = np.linalg.norm(inside(_float32_steps(U, steps, coef).astype(np.float64)) - want)
        err = np.linalg.norm(inside(_orthogonalized(bk, U, bk.BK_NS_F32, steps, coef)) - want)
        # steps that together gain at most 2^9 share a P
        products = -(-steps // int(9 / np.log2(coef[0]))) if (d, p) in THIN else 0
        tol = 4 * plain + (SUMS + products * 2.0 ** -14) * np.linalg.norm(want)
        assert err <= tol, (coef, steps, err, plain, np.linalg.norm(want))


@pytest.mark.parametrize("d,p", SMALL + THIN)
def test_usual_coefficients(bk, d, p):
    """Six to twelve steps of the usual coefficients on full-rank updates: four times float32's own error."""
    U = _update("full", d, p)
    for steps in (6, 7, 8, 9, 12):
        want = so.orthogonalize(U, steps)
        norm = np.linalg.norm(want)
        plain = np.linalg.norm(_float32_steps(U, steps, None).astype(np.float64) - want)
        err = np.linalg.norm(_orthogonalized(bk, U, bk.BK_NS_F32, steps) - want)
        assert err <= 4 * plain + SUMS * norm, (steps, err / norm, plain / norm)


# What the header says of updates of rank r after the five default steps, relative to O, times sqrt(r), and of
# long sums.  fp16 operands: X and Bm of each step are rounded, by 2e-4 root mean square (half a step is 2^-12 to
# 2^-11 of a number); each error is multiplied by at most 3.4445^5 = 485 and O has norm sqrt(r):
# sqrt(10) 485 2e-4 = 0.3.  22-bit operands: 6e-8 in place of 2e-4 is 9e-5; the float32 sum of a
# product is of up to 3 n / 16 additions, off by 2^-25 0.6 sqrt(3 n / 16) (2.7e-4 after 485 at n = 5120; 3e-4 at 8192).
# Float32 (side of at most 64): 2.4e-8 is 4e-5, and n / 4 additions 485 2^-25 0.6 sqrt(n / 4), 1.2e-4 at n = 768.
LOW_RANK = {"f16": 0.3, "f32": 4e-4, "side": 2e-4}
LONG = 1.5e-8


def _exact_steps(G, steps=5):
    """Steps of the usual coefficients in float64 on the GPU."""
    X = G.double()
    X = (X.T if X.shape[0] > X.shape[1] else X).contiguous() / X.norm()
    a, b, c = so.NS_QUINTIC
    for _ in range(steps):
        A = X @ X.T
        B = b * A + c * (A @ A)
        B.diagonal().add_(a)
        X = B @ X
    return X.T if G.shape[0] > G.shape[1] else X


def _error(bk, G, prec):
    O, want = torch.empty_like(G), _exact_steps(G)
    bk.bk_orthogonalize(bk.make_matrices([{"G": G, "O": O}]), 1, prec)
    return ((O.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("d,p", [(16, 768), (96, 64), (16, 4096), (2000, 64), (200, 300), (768, 768), (1280, 5120), (2999, 201)])
def test_low_rank_accuracy(bk, d, p):
    gen = torch.Generator(device=DEV).manual_seed(d + p)
    for r in (1, 2, 8, 32, 128):
        if r >= min(d, p):
            continue
        G = torch.randn(d, r, generator=gen, device=DEV) @ torch.randn(r, p, generator=gen, device=DEV)
        for prec, name in ((bk.BK_NS_F16, "f16"), (bk.BK_NS_F32, "f32")):
            err = _error(bk, G, prec)
            assert err <= LOW_RANK["side" if min(d, p) <= 64 else name] / r ** 0.5, (r, name, err)


def test_long_sums(bk):
    gen = torch.Generator(device=DEV).manual_seed(7)
    for n in (4000, 1 << 17, 1 << 20):
        G = torch.randn(70, n, generator=gen, device=DEV)
        assert _error(bk, G, bk.BK_NS_F16) <= 5e-3
        assert _error(bk, G, bk.BK_NS_F32) <= 3e-6 + LONG * n ** 0.5, n


def test_muon_step_of_many_steps(bk):
    """Momentum is brought up to date once, however often U is read; a stack equals single calls, a captured
    call its eager one, and nothing behind the workspace is written."""
    rng = np.random.default_rng(3)
    shapes = [(16, 4096), (2000, 64), (16, 300), (100, 70), (33, 900)] + [(int(rng.integers(1, 65)), 2000 + 7 * k) for k in range(31)]
    start = [[torch.tensor(rng.standard_normal(s), dtype=torch.float32).to(DEV) for _ in range(3)] for s in shapes]

    def specs(state):
        return [{"G": g, "M": m, "W": w, "O": o, "scale": 0.5} for g, m, w, o in state]

    def fresh():
        return [[t.clone() for t in ts] + [torch.empty_like(ts[0])] for ts in start]

    kw = dict(lr=0.25, beta=0.5, nesterov=True, weight_decay=0.5, steps=20)
    n = len(shapes)
    want = fresh()
    mats = bk.make_matrices(specs(want))
    need = bk.bk_orthogonalize_workspace_size(mats, n, bk.BK_NS_F32)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    bk.bk_muon_step(mats, n, bk.BK_NS_F32, ws=ws[:need], **kw)
    assert (ws[need:] == 0x5A).all()
    for (g, m, w, o), (_, m0, w0) in zip(want, start):
        assert torch.equal(m, torch.addcmul(g, m0, torch.tensor(0.5, device=DEV)))      # exact: times a power of two, one sum
        # 0.875 W - 0.125 O, of exact scalars: one rounding of the product, one of the sum
        new = 0.875 * w0.double() - 0.125 * o.double()
        assert ((w.double() - new).abs() <= 2.0 ** -23 * (new.abs() + w0.abs())).all()
        u = (g.double() + 0.5 * m.double()).float()           # the update, as the kernels round it
        alone = torch.empty_like(o)
        bk.bk_orthogonalize(bk.make_matrices([{"G": u, "O": alone}]), 1, bk.BK_NS_F32, steps=20)
        assert torch.equal(alone, o), g.shape
    got = fresh()
    mats = bk.make_matrices(specs(got))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        bk.bk_muon_step(mats, n, bk.BK_NS_F32, ws=ws[:need], **kw)
    for rep in range(3):
        for ts, src in zip(got, start):
            for t, v in zip(ts, src):
                t.copy_(v)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y)), rep


@pytest.mark.parametrize("d,p", [(16, 768), (16, 4096), (1, 5000), (900, 33), (100, 201)])
def test_zero_nan_and_infinity(bk, d, p):
    """After many steps too a zero update stays zero, and a NaN or an infinity spoils its whole matrix and no other."""
    U = _update("full", d, p)
    for steps in (1, 20, 64):
        for poison in (float("nan"), float("inf"), float("-inf")):
            G = [torch.tensor(U).to(DEV) for _ in range(4)]
            G[1].zero_()
            G[2][d - 1, p // 2] = poison
            O = [torch.empty(d, p, device=DEV) for _ in G]
            bk.bk_orthogonalize(bk.make_matrices([{"G": g, "O": o} for g, o in zip(G, O)]), 4, bk.BK_NS_F32, steps=steps)
            assert (O[1] == 0).all() and O[2].isnan().all(), (steps, poison)
            assert O[0].isfinite().all() and torch.equal(O[0], O[3])
