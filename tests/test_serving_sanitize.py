"""The argument checks of the calls around a decoding step under AddressSanitizer and
UndefinedBehaviorSanitizer (no GPU needed): tests/sanitize/serving_errors.cpp, built like the
other entry points' drivers (see test_sanitize.py), must end with status 0 and no report."""

import hashlib
import os
import subprocess

import test_sanitize as T


def test_argument_checks_under_sanitizers(monkeypatch):
    driver = os.path.join(T.ROOT, "tests", "sanitize", "serving_errors.cpp")
    monkeypatch.setattr(T, "DRIVER", driver)
    monkeypatch.setattr(T, "OUT", os.path.join(T.ROOT, "_build", "asan_serving_" +
                                               hashlib.sha256(open(driver, "rb").read()).hexdigest()[:8]))
    exe = T._build()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1",
               HIP_VISIBLE_DEVICES="")  # refusals only: no device may be touched
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "serving_errors ok" in r.stdout and "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
