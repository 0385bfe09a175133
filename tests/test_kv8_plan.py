"""How calls over the 8-bit cache are laid out, as the library's planner says (through
tests/sanitize/host_kv8_layout_driver), on a machine without a GPU. The GPU tests' sizes are
chosen to land on one layout or another: here they are held to it.
"""
import os
import subprocess

import pytest

import test_gpu_kv8 as kv8
import test_gpu_kv8_range as wide
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


def _layout(B, H, Hk, D, window, n_q, lengths):
    """The kind of layout of a call, and the parts of a split tile."""
    out = _driver("layouts", input=" ".join(map(str, [B, H, Hk, D, window, n_q, *lengths])) + "\n")
    few, n_tiles, n_whole, parts, cut, blocks, workspace = map(int, out.split())
    tiles = n_tiles * B * Hk
    assert workspace == (tiles - n_whole) * parts * (32 if few else 256) * (D + 2) * 4 * (parts > 1)
    if few:
        return "32 rows, split" if parts > 1 else f"32 rows, {few} waves", parts
    if parts == 1:
        return "256 rows", 1
    return "256 rows, cut" if cut else "256 rows, last ones split" if n_whole else "256 rows, split", parts


# what test_gpu_kv8.test_attention's cases are there for, in their order
ATTENTION = (["32 rows, 4 waves"] * 5 + ["32 rows, 8 waves"] * 2 + ["32 rows, split"] * 3 + ["32 rows, 8 waves"]
             + ["256 rows", "256 rows, last ones split", "256 rows", "256 rows, split", "256 rows, cut",
                "256 rows, split", "256 rows, split"])


@pytest.mark.parametrize("D", [64, 128])
def test_layouts_of_the_attention_tests(D):
    cases = next(m.args[1] for m in kv8.test_attention.pytestmark if m.args[0] != "D")
    assert len(cases) == len(ATTENTION)
    most = 0
    for (B, H, Hk, lengths, window, n_q), kind in zip(cases, ATTENTION):
        got, parts = _layout(B, H, Hk, D, window, n_q, lengths)
        assert got == kind, (B, H, Hk, lengths, window, n_q)
        most = max(most, parts * (kind == "256 rows, split"))
        now = [lengths[0]] + lengths[max(1, len(lengths) - 1 - window):]
        assert kv8.in_tiles(B, Hk, n_q * (H // Hk), now, D) == kind.startswith("256")
    assert most > 16  # (whose merge is another one)


@pytest.mark.parametrize("D", [64, 128])
def test_layouts_of_the_tests_of_ranges(D):
    kinds = ["32 rows, 8 waves", "32 rows, split", "32 rows, 8 waves", "256 rows", "256 rows, split", "256 rows, cut"]
    for (n_q, H, blocks, tiles), kind in zip(wide.FORMS, kinds, strict=True):
        assert _layout(1, H, H, D, 0, n_q, [64 * blocks])[0] == kind
        assert tiles == kind.startswith("256")


# (B, H, Hk, D, window, n_q, lengths) of the other calls whose tests say whether they go in tiles of 256 rows
OTHERS = [(1, H, H, 128, 0, n_q, [1000]) for n_q, H in [(1, 2), (300, 2), (300, 170)]]
OTHERS += [(1, H, H, 64, 0, n_q, [512]) for n_q, H in [(1, 1), (257, 1), (512, 120)]]
OTHERS += [(1, H, H, 128, 0, n_q, [300]) for n_q, H in [(3, 1), (300, 1), (300, 250)]]
OTHERS += [(1, H, H, 64, 0, n_q, [10000]) for n_q, H in [(2, 1), (100, 40)]]
OTHERS += [(2, H, H, 64, 0, n_q, [200]) for n_q, H in [(4, 1), (60, 1), (510, 60)]]
OTHERS += [(1, H, H, D, 0, 256, [640]) for D, H in [(64, 1), (128, 1), (64, 250), (128, 200)]]
OTHERS += [(1, 4, 2, 128, 1, 1000, [9000, 200]), (1, 1, 1, 128, 0, 64, [(1 << 25) + 200])]


@pytest.mark.parametrize("B,H,Hk,D,window,n_q,lengths", OTHERS)
def test_the_tests_rule_is_the_librarys(B, H, Hk, D, window, n_q, lengths):
    assert _layout(B, H, Hk, D, window, n_q, lengths)[0].startswith("256") == \
        kv8.in_tiles(B, Hk, n_q * (H // Hk), lengths, D)
