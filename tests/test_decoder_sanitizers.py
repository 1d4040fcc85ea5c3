"""The host checks, sizes and plans of a decoder's steps in 8 bits under AddressSanitizer and UndefinedBehaviorSanitizer (CPU
only): tests/asan/decoder_driver.cpp calls every entry point over the whole range of its sizes and is refused by each before
anything is launched."""
import os
import subprocess

from tests import test_host_sanitizers as H
from tests.test_serving_sanitizers import MODEL, program

SOURCES = MODEL + [os.path.join(H.CSRC, f) for f in ("decoder.cpp", "rows8.hip", "linear8.hip", "logprobs.hip")]


def test_decoder_checks_under_sanitizers():
    driver = program(SOURCES + [os.path.join(H.ROOT, "tests", "asan", "decoder_driver.cpp")], "decoder_driver")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([driver], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]
    assert r.returncode == 0 and "0 failed checks" in r.stdout, out[-4000:]
