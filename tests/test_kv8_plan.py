"""How calls over the 8-bit cache are laid out, as the library's planner says (through
tests/sanitize/host_kv8_layout_driver), on a machine without a GPU.
"""
import os
import subprocess

import pytest

import test_host_sanitize as sanitize

DRIVER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "sanitize", "host_kv8_layout_driver")


def _driver(*args, **more):
    if not os.path.exists(DRIVER):
        pytest.skip("tests/sanitize/host_kv8_layout_driver is not built (run build())")
    res = subprocess.run([DRIVER, *args], capture_output=True, text=True, env=sanitize.ENV, timeout=120, **more)
    assert res.returncode == 0, res.stdout[-1000:] + res.stderr[-3000:]
    return res.stdout


def test_a_layout_that_the_merge_does_not_take_is_refused_before_the_launch():
    assert "all checks passed" in _driver()
