"""How the steps of thin matrices are cut into rounds (each from a Gram matrix of
its own): the host code under AddressSanitizer and UndefinedBehaviorSanitizer,
with stand-ins for the launchers (tests/host_sanitize/thin_driver.cpp); and the
rounds' arithmetic, emulated, on updates of low rank.  CPU only."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import step_oracle as so

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2210_00038_amd", "csrc")


def test_rounds_under_asan_and_ubsan(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers are missing")
    exe = str(tmp_path / "thin_rounds")
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, "step_api.cpp"),
           os.path.join(ROOT, "tests", "host_sanitize", "thin_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), (r.stdout[-2000:], r.stderr[-4000:])


def _sym(A):
    return np.triu(A) + np.triu(A, 1).T


def _thin(U, steps, coef, per_round):
    """X after `steps`, `per_round` of them from one Gram matrix in float64, whose product P is rounded to float32."""
    X = (U / np.linalg.norm(U)).astype(np.float32)
    a, b, c = coef
    eye = np.eye(len(X))
    for first in range(0, steps, per_round):
        A = _sym(X.astype(np.float64) @ X.astype(np.float64).T)
        P = eye
        for _ in range(min(per_round, steps - first)):
            Bm = _sym(a * eye + b * A + c * (A @ A))
            A, P = _sym(_sym(Bm @ A) @ Bm), _sym(Bm @ P)
        X = P.astype(np.float32) @ X
    return X


@pytest.mark.parametrize("coef,per_round", [(so.NS_QUINTIC, 5), ((1.5, -0.5, 0.0), 15), ((1.875, -1.25, 0.375), 9)])
def test_rounds_keep_low_rank_updates_bounded(coef, per_round):
    """64 steps in rounds of a gain of at most 2^9 stay within the polynomials' range (1.21, 1 and 1); from one Gram
    matrix they do not."""
    assert coef[0] ** per_round <= 512 < coef[0] ** (per_round + 1)
    rng = np.random.default_rng(1)
    U = rng.standard_normal((24, 8)) @ rng.standard_normal((8, 600))
    X = _thin(U, 64, coef, per_round)
    assert np.isfinite(X).all() and np.linalg.norm(X.astype(np.float64), 2) < 1.21
    with np.errstate(all="ignore"):
        assert not np.isfinite(_thin(U, 64, coef, 64)).all()
