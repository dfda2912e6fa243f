"""The sampling operators' host entry points under AddressSanitizer and UndefinedBehaviourSanitizer: as test_host_sanitized.py, with
the CPU tests that call them (their refusals, their largest sizes).  No GPU is needed: no kernel is launched."""
import os
import subprocess
import sys

from paper_2602_24082_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sampling_host_tests_pass_under_asan_and_ubsan(tmp_path):
    lib = build.build_host_sanitized(str(tmp_path / "libppattn_asan.so"))
    preload = build.asan_runtime()
    if os.environ.get("LD_PRELOAD"):
        preload += ":" + os.environ["LD_PRELOAD"]  # the sanitizer runtime must come first
    env = dict(os.environ, PP_LIB_PATH=lib, LD_PRELOAD=preload, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    files = [os.path.join(ROOT, "tests", f) for f in ("test_sample_host.py", "test_sample_limits.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-k", "refusals or limits", *files],
                       env=env, capture_output=True, text=True, cwd=ROOT, timeout=900)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, out
    assert "10 passed" in r.stdout and "runtime error" not in out and "AddressSanitizer" not in out, out
