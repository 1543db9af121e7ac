"""AddressSanitizer and UndefinedBehaviorSanitizer run of the sizes that the key/value cache's host side
computes, on the CPU: its sources and tests/sanitize/kv_limits_driver.cpp built with hipcc, the
sanitizers on the host pass only, run without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]


def test_sizes_under_asan_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    csrc = os.path.join(ROOT, "paper_2203_00448_amd", "csrc")
    srcs = sorted(os.path.join(csrc, f) for f in os.listdir(csrc) if f.startswith("kv") and f.endswith(".hip"))
    host_san = [a for flag in SAN for a in ("-Xarch_host", flag)]
    exe = str(tmp_path / "kv_limits_driver")
    subprocess.run([hipcc, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", *host_san,
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "sanitize", "kv_limits_driver.cpp"), *srcs, "-o", exe],
                   check=True, capture_output=True)
    r = subprocess.run([exe], cwd=tmp_path, capture_output=True, text=True, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "all checks passed" in out, out
    assert "runtime error" not in out and "AddressSanitizer" not in out, out
