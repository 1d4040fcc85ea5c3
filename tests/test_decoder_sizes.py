"""Sizes of a decoder's steps in 8 bits (CPU only, tests/asan/decoder_sizes_driver.cpp): workspaces hold what their launches write, and
the products that the GPU tests run reach every form that any size chooses."""
import os
import subprocess

import pytest

from tests import test_host_sanitizers as H
from tests.test_decoder_sanitizers import SOURCES
from tests.test_gpu_decoder import LINEAR_SIZES, test_linear_large as linear_large
from tests.test_gpu_decoder_forms import FORMS, SHARED
from tests.test_serving_sanitizers import program


@pytest.fixture(scope="module")
def driver():
    return program(SOURCES + [os.path.join(H.ROOT, "tests", "asan", "decoder_sizes_driver.cpp")], "decoder_sizes_driver")


def lines(driver, *args, text=None):
    r = subprocess.run([driver, *args], input=text, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    return [tuple(map(int, line.split())) for line in r.stdout.splitlines()]


def test_logprobs_workspaces_hold_their_parts(driver):
    r = subprocess.run([driver], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "0 failed checks" in r.stdout, (r.stdout + r.stderr)[-4000:]


def test_the_products_that_are_tested_reach_every_form(driver):
    large = [mark.args[1] for mark in linear_large.pytestmark if mark.args[0] == "m,n,k"][0]
    sizes = LINEAR_SIZES + large + FORMS + SHARED
    plans = lines(driver, "plan", text="\n".join("%d %d %d" % s for s in sizes))
    assert len(plans) == len(sizes)
    shares = dict(zip(sizes, plans))
    assert all(shares[s][4] > 1 for s in SHARED), shares
    reached = {p[:4] + (2 if p[4] > 1 else 1,) for p in plans}
    every = set(lines(driver, "forms"))
    assert len(every) >= 14 and every <= reached, every - reached
