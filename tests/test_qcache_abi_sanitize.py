"""The 8-bit token cache's argument checks at the largest sizes under the host sanitizers (CPU only).

abi.hip, where the checks are, and tests/qcache_limits_host.hip are compiled with AddressSanitizer and
UndefinedBehaviorSanitizer on the host code and linked to the built library for the rest.
"""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_largest_sizes_under_host_sanitizers(tmp_path):
    import paper_2604_24391_amd as fc
    fc.lib()
    exe, lib = str(tmp_path / "qcache_limits"), fc.freqcache.LIB
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xarch_host", "-g",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-value", "-Wno-unused-result",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer",
           os.path.join(ROOT, "paper_2604_24391_amd", "csrc", "abi.hip"), os.path.join(ROOT, "tests", "qcache_limits_host.hip"),
           "-L" + os.path.dirname(lib), "-l:" + os.path.basename(lib), "-Wl,-rpath," + os.path.dirname(lib), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="")          # never a device, even where one exists
    env.pop("FC_DEBUG", None)
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0:halt_on_error=1"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    out = run.stdout + run.stderr
    assert run.returncode == 0, out[-6000:]
    assert "OK (0 failed expectations)" in run.stdout
    assert "runtime error" not in out and "AddressSanitizer" not in out
