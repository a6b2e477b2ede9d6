"""The workspace of the RMS norm's backward pass: its size for a batch serves
every smaller one, as the other workspaces' do.  The host code under
AddressSanitizer and UndefinedBehaviorSanitizer (tests/host_sanitize/
rms_driver.cpp), and on the GPU the smaller batches themselves."""
import os
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2210_00038_amd", "csrc")


def test_sizes_under_asan_and_ubsan(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the HIP headers are missing")
    exe = str(tmp_path / "rms_workspace")
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, os.path.join(CSRC, "step_api.cpp"),
           os.path.join(ROOT, "tests", "host_sanitize", "rms_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), (r.stdout[-2000:], r.stderr[-4000:])


@pytest.mark.gpu
@pytest.mark.parametrize("full,T,p", [(512, 16, 2048), (40, 500, 100), (300, 9, 4096), (1200, 40, 768)])
def test_last_batch_on_the_full_one_s_workspace(full, T, p):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2210_00038_amd as bk
    need = bk.bk_rmsnorm_grad_workspace_size(full, T, p)
    gen = torch.Generator().manual_seed(p)
    dy, xhat = (torch.randn(full, T, p, generator=gen).to(torch.bfloat16).to("cuda") for _ in range(2))
    rstd = (torch.rand(full, T, generator=gen) + 0.1).to("cuda")
    ws = torch.full((need + 1024,), 0x5A, dtype=torch.uint8, device="cuda")
    for B in (full, full // 2, full // 8 + 1, 3, 1):
        assert bk.bk_rmsnorm_grad_workspace_size(B, T, p) <= need
        dx, P = bk.bk_rmsnorm_grad(dy[:B], xhat[:B], rstd[:B], ws=ws[:need])
        want, wantP = bk.bk_rmsnorm_grad(dy[:B], xhat[:B], rstd[:B])
        assert torch.equal(dx, want) and torch.equal(P, wantP)
        assert (ws[need:] == 0x5A).all()
