"""The host side of layers in the clear under AddressSanitizer and UndefinedBehaviorSanitizer; the launchers are stubs."""
import os
import shutil

import pytest

from test_sanitizers import CSRC, ROOT, SAN, run


def test_checks_of_clear_layers_under_sanitizers(tmp_path):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if not shutil.which("g++") or not os.path.exists(os.path.join(rocm, "lib", "libamdhip64.so")):
        pytest.skip("no g++ or no HIP runtime to link against")
    exe = str(tmp_path / "clear_san")
    src = [os.path.join(ROOT, "tests", "sanitize", "clear_driver.cpp")] + [os.path.join(CSRC, f) for f in ("clear_layers.cpp", "host_keys.cpp")]
    b = run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include", "-pthread", *src,
             f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib", "-o", exe])
    assert b.returncode == 0, b.stdout
    r = run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
    assert r.returncode == 0 and "checks: ok" in r.stdout, r.stdout
