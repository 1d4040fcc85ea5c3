"""The host checks and sizes of decoding with a paged cache under AddressSanitizer and UndefinedBehaviorSanitizer (CPU
only): tests/asan/serving_driver.cpp calls every entry point over the whole range of its sizes and is refused by each before
anything is launched.  A program without the decoding kernels (partial_driver.cpp) refuses models that need them."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from tests import test_host_sanitizers as H

MODEL = [s for s in H.SOURCES if not s.endswith("driver.cpp")]
SOURCES = [os.path.join(H.CSRC, f) for f in ("abi.cpp", "plan.cpp", "model.cpp", "gemm.hip", "kernels.hip", "lstm.hip", "noalloc.hip",
                                             "serving.cpp", "rotary.hip", "attention.hip")]
SOURCES.append(os.path.join(H.ROOT, "tests", "asan", "serving_driver.cpp"))


def program(sources, name):
    if not shutil.which(H.HIPCC):
        pytest.skip("hipcc not found")
    os.makedirs(H.BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(H._compile, sources))
    exe = os.path.join(H.BUILD, name)
    r = subprocess.run([H.HIPCC, "--offload-arch=gfx950", *H.HOST_SAN, *objs, "-o", exe], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr[-3000:])
    return exe


def test_serving_checks_under_sanitizers():
    driver = program(SOURCES, "serving_driver")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([driver], capture_output=True, text=True, env=env, timeout=300)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]
    assert r.returncode == 0 and "0 failed checks" in r.stdout, out[-4000:]


def test_a_program_without_the_decoding_kernels_refuses_their_models():
    driver = program(MODEL + [os.path.join(H.ROOT, "tests", "asan", "partial_driver.cpp")], "partial_driver")
    r = subprocess.run([driver], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
