"""The 4-bit calls through the host-sanitizer build (tests/native/packed_driver.cpp)."""
import os
import subprocess

import pytest

pytestmark = pytest.mark.gpu


def test_host_sanitizer_driver():
    from paper_2608_07855_amd import build
    if not os.path.exists(build.PACKED_DRIVER):
        pytest.fail("the sanitizer driver is not built (python -m paper_2608_07855_amd.build asan)")
    env = dict(os.environ)
    # as for the other driver: the GPU runtime maps memory where the shadow gap would be
    env["ASAN_OPTIONS"] = "protect_shadow_gap=0:detect_leaks=0:halt_on_error=1"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    print("[tools] sanitizer driver of the 4-bit calls", flush=True)
    r = subprocess.run([build.PACKED_DRIVER], env=env, capture_output=True, text=True, timeout=100)
    text = r.stdout + r.stderr
    print(text[-3000:], flush=True)
    assert "AddressSanitizer" not in text and "runtime error" not in text
    assert r.returncode == 0, text[-2000:]
    assert "[driver] ok" in r.stdout
