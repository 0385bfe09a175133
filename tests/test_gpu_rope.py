"""Rotary positions with three axes (tm_rope3d_*) against the definition in 64 bits.

Tolerances. The table holds cosines and sines rounded from fp64, so each is
within 2^-25 + 2^-49 of the exact value (values up to 1: half an fp32 ulp is
2^-25). A rotated element a c - b s is one product, one fma of fp32, so its
error is at most (|a| + |b|) (2^-25 + 2 * 2^-24) <= 2^-22 (|a| + |b|), and a bf16
result adds half a bf16 ulp, at most 2^-8 |y| (8 significant bits).
"""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def angles64(frames, gh, gw, pairs, theta):
    """The angle tables of the three axes, [positions, pairs] in 64 bits."""
    return [np.arange(n, dtype=np.float64)[:, None] * np.float64(theta) ** (-np.arange(p) / max(p, 1))
            for n, p in zip((frames, gh, gw), pairs)]


def rotate64(x, first, gh, gw, frames, pairs, theta, halves, sign=1.0):
    """x: numpy [B, n, H, D] in 64 bits, rotated by the definition, pair by pair."""
    B, n, H, D = x.shape
    p = first + np.arange(n)
    f, j = p // (gh * gw), p % (gh * gw)
    tables = angles64(frames, gh, gw, pairs, theta)
    y = x.copy()
    i = 0
    for pos, t in zip((f, j // gw, j % gw), tables):
        for a in range(t.shape[1]):
            c, s = np.cos(t[pos, a])[None, :, None], sign * np.sin(t[pos, a])[None, :, None]
            m, k = (i, i + D // 2) if halves else (2 * i, 2 * i + 1)
            y[..., m] = x[..., m] * c - x[..., k] * s
            y[..., k] = x[..., m] * s + x[..., k] * c
            i += 1
    return y


def partner(x, halves):
    """The other element of every element's pair."""
    if halves:
        return np.roll(x, x.shape[-1] // 2, -1)
    return x.reshape(*x.shape[:-1], -1, 2)[..., ::-1].reshape(x.shape)


def check(got, x, want, halves, what):
    bound = 2.0 ** -22 * (np.abs(x) + np.abs(partner(x, halves)))
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * np.abs(want)
    err = np.abs(got.double().cpu().numpy() - want)
    worst = float(np.max(err / np.maximum(bound, 1e-300)))
    say(f"  {what}: largest error / bound = {worst:.3f}")
    assert np.all(err <= bound), what


@pytest.mark.parametrize("pairs,theta", [((22, 21, 21), 10000.0), ((0, 0, 0), 10000.0), ((64, 0, 0), 500.0),
                                         ((1, 2, 3), 1.0)])
def test_table_holds_rounded_cosines_and_sines(tm, pairs, theta):
    frames, gh, gw = 5000, 30, 52
    d = tm.make_rope_desc(128, frames, gh, gw, pairs, theta)
    t = tm.tm_rope3d_table(d).cpu().numpy()
    want = np.concatenate([a.reshape(-1) for a in angles64(frames, gh, gw, pairs, theta)])
    assert t.shape == (want.size, 2)
    # angles up to 5000 in fp64: argument and function errors below 1e-11
    assert np.all(np.abs(t[:, 0] - np.cos(want)) <= 2.0 ** -25 + 1e-11)
    assert np.all(np.abs(t[:, 1] - np.sin(want)) <= 2.0 ** -25 + 1e-11)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("B,n,H,Hk,first", [(1, 1, 1, 1, 0), (2, 7, 3, 1, 11), (1, 131, 5, 0, 1000),
                                            (3, 64, 40, 8, 77), (1, 3000, 8, 8, 5)])
def test_forward_and_backward_against_the_definition(tm, dtype, D, halves, B, n, H, Hk, first):
    gh, gw = 9, 13
    frames = (first + n - 1) // (gh * gw) + 1
    pairs = (D // 2 - 2 * (D // 6), D // 6, D // 6)
    desc = tm.make_rope_desc(D, frames, gh, gw, pairs, 10000.0, halves, dtype)
    table = tm.tm_rope3d_table(desc)
    g = torch.Generator().manual_seed(B * 1000 + n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.randn((B, n, H, D), generator=g).to(dt).cuda()
    k = torch.randn((B, n, Hk, D), generator=g).to(dt).cuda() if Hk else None
    for fn, sign in ((tm.tm_rope3d_fwd, 1.0), (tm.tm_rope3d_bwd, -1.0)):
        out = fn(desc, table, q, k, first)
        for x, y, what in ((q, out[0], "q"), (k, out[1], "k")):
            if x is None:
                assert y is None
                continue
            x64 = x.double().cpu().numpy()
            want = rotate64(x64, first, gh, gw, frames, pairs, 10000.0, halves, sign)
            check(y, x64, want, halves, f"{fn.__name__} {what}")


@pytest.mark.parametrize("pairs", [(3, 0, 5), (0, 16, 0), (20, 1, 1), (0, 0, 0)])
def test_pairs_that_no_axis_turns_keep_their_bits(tm, pairs):
    D, gh, gw, n = 64, 4, 6, 100
    desc = tm.make_rope_desc(D, 5, gh, gw, pairs, 10000.0, False, "f32")
    table = tm.tm_rope3d_table(desc)
    x = torch.randn((1, n, 2, D), generator=torch.Generator().manual_seed(3)).cuda()
    y, _ = tm.tm_rope3d_fwd(desc, table if sum(pairs) else None, x, first_token=1)
    at = 2 * sum(pairs)
    assert torch.equal(x[..., at:], y[..., at:])
    x64 = x.double().cpu().numpy()
    check(y, x64, rotate64(x64, 1, gh, gw, 5, pairs, 10000.0, False), False, str(pairs))


def test_in_place_and_other_stream_give_the_same_bits(tm):
    desc = tm.make_rope_desc(128, 8, 30, 52)
    table = tm.tm_rope3d_table(desc)
    q = torch.randn((1, 4680, 5, 128), device="cuda").bfloat16()
    k = torch.randn((1, 4680, 1, 128), device="cuda").bfloat16()
    want = tm.tm_rope3d_fwd(desc, table, q, k, 1560)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = tm.tm_rope3d_fwd(desc, table, q, k, 1560)
    s.synchronize()
    for a, b in zip(want, other):
        assert torch.equal(a, b)
    tm.tm_rope3d_fwd(desc, table, q, k, 1560, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_backward_against_differences(tm):
    """The forward is linear, so (f(x + d) - f(x - d)) / 2 is its derivative along d, up to the
    roundings of the two fp32 results: each within 2^-22 of its pair's size."""
    desc = tm.make_rope_desc(128, 12, 5, 7, (22, 21, 21), 10000.0, True, "f32")
    table = tm.tm_rope3d_table(desc)
    g = torch.Generator().manual_seed(9)
    x, d, dy = (torch.randn((2, 300, 3, 128), generator=g).cuda() for _ in range(3))
    up = tm.tm_rope3d_fwd(desc, table, x + d, first_token=17)[0].double()
    down = tm.tm_rope3d_fwd(desc, table, x - d, first_token=17)[0].double()
    dx = tm.tm_rope3d_bwd(desc, table, dy, first_token=17)[0].double()
    along = float((dy.double() * (up - down) / 2).sum())
    size = (x.abs() + d.abs()).double()
    size = size + torch.roll(size, 64, -1)
    bound = float((dy.abs().double() * 2.0 ** -22 * size).sum()) + \
        float((d.abs().double() * 2.0 ** -22 * (dy.abs() + torch.roll(dy.abs(), 64, -1)).double()).sum())
    assert abs(along - float((dx * d.double()).sum())) <= bound


def test_a_captured_call_replays_to_the_eager_bits(tm):
    desc = tm.make_rope_desc(64, 4, 3, 11)
    table = tm.tm_rope3d_table(desc)
    q = torch.randn((1, 50, 4, 64), device="cuda").bfloat16()
    out = torch.empty_like(q)
    tm.tm_rope3d_fwd(desc, table, q, first_token=3, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tm.tm_rope3d_fwd(desc, table, q, first_token=3, q_out=out)
    for i in range(4):
        q.copy_(torch.randn((1, 50, 4, 64), device="cuda").bfloat16())
        want = tm.tm_rope3d_fwd(desc, table, q, first_token=3)[0]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_tokens_and_refusals(tm):
    desc = tm.make_rope_desc(128, 2, 3, 5)
    table = tm.tm_rope3d_table(desc)
    q = torch.zeros((1, 30, 2, 128), dtype=torch.bfloat16, device="cuda")
    y, _ = tm.tm_rope3d_fwd(desc, table, q[:, :0])
    assert y.shape == (1, 0, 2, 128)

    def refused(status, fn):
        with pytest.raises(tm.TMError) as e:
            fn()
        assert e.value.status == status, e.value

    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table, q, first_token=1))    # past the frames
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table, q, first_token=-1))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table, q.float()))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table, q, q[:, :29].contiguous()))
    refused(tm.TM_E_ARG, lambda: tm.tm_rope3d_fwd(desc, table, q.transpose(1, 2).contiguous().transpose(1, 2)))
    refused(tm.TM_E_ARG, lambda: tm.tm_rope3d_fwd(desc, None, q))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table[:-1].clone(), q))      # a table too short
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(desc, table, q, q_out=q[:, :29].clone()))
    # (one tensor of 60 tokens: the output starts inside the input)
    buf = torch.zeros(31 * 256, dtype=torch.bfloat16, device="cuda")
    a, b = buf[:7680].view(1, 30, 2, 128), buf[256:].view(1, 30, 2, 128)
    refused(tm.TM_E_ARG, lambda: tm.tm_rope3d_fwd(desc, table, a, q_out=b))
    refused(tm.TM_E_ARG, lambda: tm.tm_rope3d_fwd(desc, table, a, q, q_out=torch.empty_like(q), k_out=a))
