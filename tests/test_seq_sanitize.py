"""The argument checks of the calls over several sequences under AddressSanitizer and
UndefinedBehaviorSanitizer (no GPU needed): tests/sanitize/seq_errors.cpp, built like the
other entry points' driver (see test_sanitize.py), must end with status 0 and no report."""

import hashlib
import os
import subprocess

import test_sanitize as T


def test_argument_checks_under_sanitizers(monkeypatch):
    driver = os.path.join(T.ROOT, "tests", "sanitize", "seq_errors.cpp")
    monkeypatch.setattr(T, "DRIVER", driver)
    monkeypatch.setattr(T, "OUT", os.path.join(T.ROOT, "_build", "asan_seq_" +
                                               hashlib.sha256(open(driver, "rb").read()).hexdigest()[:8]))
    exe = T._build()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1",
               HIP_VISIBLE_DEVICES="")  # refusals only: no device may be touched
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "seq_errors ok" in r.stdout and "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr


def test_device_query_under_thread_sanitizer(tmp_path):
    """Launches of several threads at once share one query of the device: no data race (tests/sanitize/device_query.cpp)."""
    hipcc, clang = T._tools()
    obj, exe = str(tmp_path / "device_query.o"), str(tmp_path / "device_query")
    src = os.path.join(T.ROOT, "tests", "sanitize", "device_query.cpp")
    for cmd in ([hipcc, "--offload-host-only", "-x", "hip", "-O1", "-g", "-std=c++17", "-I", T.CSRC, "-Xarch_host",
                 "-fsanitize=thread", "-c", src, "-o", obj], [clang, "-Xarch_host", "-fsanitize=thread", obj, "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert "data race" not in r.stderr and r.returncode == 0, r.stderr[-4000:]
    assert "device_query ok" in r.stdout
