"""CPU sanitizer leg of include/quartet_block.h's host side: argument checks and sequencing under AddressSanitizer and
UndefinedBehaviorSanitizer, the kernels replaced by counting stand-ins, driven by tests/test_block_host.py in a child process."""
import glob
import os
import shutil
import subprocess

import pytest
from test_sanitizers import ROOT, TESTS, child_env, run_child


@pytest.mark.timeout(600)
def test_block_argument_checks_pass_under_sanitizers(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    rts = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    if not rts:
        pytest.skip("clang's AddressSanitizer runtime is not installed")
    csrc, package = os.path.join(ROOT, "paper_2505_14669_amd", "csrc"), tmp_path / "checked"
    package.mkdir()
    # sanitizers on the host pass only; neither file of the C ABI has kernels of its own
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-I", csrc,
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
           os.path.join(csrc, "api.hip"), os.path.join(csrc, "api_block.hip"), os.path.join(TESTS, "hostcheck", "launcher_stubs.cpp"),
           os.path.join(TESTS, "hostcheck", "block_stubs.cpp"), "-o", str(package / "libquartet.so")]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
    shutil.copy(os.path.join(ROOT, "paper_2505_14669_amd", "binding.py"), package / "binding.py")
    out = run_child([os.path.join(TESTS, "test_block_host.py")], child_env(rts[0], QUARTET_HOSTCHECK_DIR=str(package)), 500)
    assert " passed" in out
