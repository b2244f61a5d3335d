"""The argument checks of the operators around the layers under AddressSanitizer and UndefinedBehaviorSanitizer (host code
only), as test_host_sanitizers does for the layers': every call is refused before the first GPU call."""
import os
import subprocess

import pytest

from test_host_sanitizers import COMMON, HIPCC, ROOT, SAN


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_argument_checks_under_host_sanitizers(tmp_path):
    lib, exe = tmp_path / "libfasth_san.so", tmp_path / "token_host_check"
    for out, args in ((lib, ["-fPIC", "-shared", os.path.join(ROOT, "paper_2009_13977_amd", "csrc", "fasth.hip")]),
                      (exe, [os.path.join(ROOT, "tests", "token_host_check.cpp"), "-L", str(tmp_path), "-lfasth_san", f"-Wl,-rpath,{tmp_path}"])):
        r = subprocess.run(COMMON + SAN + ["-o", str(out)] + args, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    env = {**os.environ, "ASAN_OPTIONS": "detect_leaks=0:protect_shadow_gap=0"}  # the HIP runtime reserves address space of its own
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout[-4000:], r.stderr[-4000:])
    assert "token_host_check: ok" in r.stdout
