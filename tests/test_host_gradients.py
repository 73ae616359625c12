"""The stage executor (csrc/stage.cpp) on host launchers that compute, built with g++ under sanitizers: gradients are the same wherever the caller wants the input's, over an operand of
the pass as well, and of layers that are linear they are what the outputs change by (tests/host/gradients_over_operands.cpp)."""
import os
import subprocess

import pytest

from tests.test_host_sanitizers import build


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    return build(tmp_path_factory, "gradients_over_operands", ["tests/host/gradients_over_operands.cpp", "tests/host/arithmetic.cpp", "paper_2410_14312_amd/csrc/stage.cpp"])


def run(driver, which):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([driver, which], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and not r.stderr, r.stderr[-2000:]


def test_joins_of_the_stage_input(driver):
    run(driver, "joins")


def test_additions_of_the_stage_input(driver):
    run(driver, "additions")


def test_stages_of_one_layer(driver):
    run(driver, "alone")


def test_random_layers(driver):
    run(driver, "random")


def test_rotary_positions_on_a_shared_input(driver):
    run(driver, "rotary")
