"""The C-ABI layer of the 8-bit head and of beam search under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU: csrc/aal_head_api.hip and csrc/aal_beam_api.hip with host
stand-ins for their launchers (tests/sanitize/head_beam_driver.cpp), linked with the sanitized
rest of the layer, which holds the error text."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")


def test_head_and_beam_abi_layer_under_asan_and_ubsan(tmp_path):
    from paper_2609_24150_amd import build as B
    try:
        hipcc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not found")
    objs = [B.compile_api_sanitized(str(tmp_path / f"{s}.o"), s + ".hip") for s in ("aal_api", "aal_head_api", "aal_beam_api")]
    exe = tmp_path / "head_beam_sanitize"
    cmd = [hipcc, "-std=c++17", f"--offload-arch={B.ARCH}", *B.SANITIZE_FLAGS, f"-I{B.INCLUDE}", f"-I{B.CSRC}", *objs,
           os.path.join(SAN, "launch_stubs.cpp"), os.path.join(SAN, "head_beam_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "all checks passed" in r.stdout
    assert "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
