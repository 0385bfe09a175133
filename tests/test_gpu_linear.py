"""Linear layers with bias, activation, gate and residual (tm_linear_*) against the definition in 64 bits.

Tolerances, in units u = 2^-24 (half an fp32 step, relative). A sum of K products of bf16 numbers, exact in
fp32, in any order: at most K roundings of partial sums, each at most 2 u (a matrix instruction may cut instead of
round) of the sum of magnitudes S = |x| |W|^T + |bias|, so z is within 2 (K + 8) u S. An activation's slope is
below 1.13, its own arithmetic (two products, exp2 and rcp of 1 ulp each, and for gelu an argument that is off by
4 u of itself, which its slope times z turns into at most 16 u of |z|) within 32 u |z|; gate, residual
and the sums in fp32 another 4 u of their terms. Results in bf16 add half a step, 2^-8 of themselves.
Backward: dz within 64 u of |dout gate| times (1 + |z|), rounded to bf16 for the products (2^-8 relative). With 5 to 16
rows dz goes into them as the sum of two bf16 numbers, hi = dz rounded and lo = dz - hi rounded: |dz - hi| <=
2^-8 |dz|, so what lo's rounding leaves out is at most 2^-8 of that, 2^-16 |dz|; with up to 4 rows it is not rounded.
A product of it is within that times |W| (|x|), and 2 (terms + 8) u S. Roundings of
half a step at most have a root mean square of 2^-8 / sqrt(3) at most, and two of them, dz's and the result's,
sqrt(2 / 3) 2^-8 of the result's norm: products are held to 2^-8 of their norm as well.
"""
import pytest
import torch

from block_reference import activate, as64, group_rows, linear
from block_sizes import FEW_ROWS, PRODUCTS
from gpu_helpers import say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def make(B, n, K, N, out, parts, groups, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, size=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)

    return {"x": normal((B, n, K), 1.0, torch.bfloat16), "weight": normal((N, K), K ** -0.5, torch.bfloat16),
            "bias": normal((N,), 0.1) if "b" in parts else None,
            "gate": normal((B, groups, N), 0.5) if "g" in parts else None,
            "residual": normal((B, n, N), 2.0, DT[out]) if "r" in parts else None}


def held(got, want, bound, what):
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs()
    err = (got.double() - want).abs()
    worst = float((err / bound.clamp_min(1e-300)).max()) if err.numel() else 0.0
    say(f"  {what}: largest error / bound = {worst:.3f}")
    assert bool((err <= bound).all()), what


def near(got, want, what):
    rel = float((got.double() - want).norm() / want.norm().clamp_min(1e-300))
    say(f"  {what}: {rel * 2 ** 8:.3f} of 2^-8 of its norm")
    assert rel <= 2.0 ** -8, what


# one row to several tiles of either size, widths and rows that end inside tiles and stages
SHAPES = [(1, 1, 8, 8), (1, 1, 5120, 520), (2, 8, 72, 200), (1, 16, 1000, 64), (1, 17, 64, 64), (3, 111, 1000, 1352),
          (1, 129, 40, 136), (2, 65, 2568, 264), (1, 300, 8, 1032), (1, 700, 520, 2056), (1, 1, 8, 4104), (1, 5, 20480, 8)]
SETS = [("none", "bf16", "", 1, 0, 0), ("gelu", "bf16", "bz", 1, 0, 5), ("silu", "f32", "bgrz", 5, 300, 40),
        ("none", "f32", "bgrz", 9, 90, 11), ("gelu", "f32", "gz", 800, 1, 3)]


@pytest.mark.parametrize("B,n,K,N", SHAPES)
@pytest.mark.parametrize("act,out,parts,groups,group,first", SETS)
def test_forward_and_backward(tm, B, n, K, N, act, out, parts, groups, group, first):
    p = make(B, n, K, N, out, parts, groups, n + K + N)
    g = group_rows(B, n, groups, group, first, "cuda")
    d = tm.make_linear_desc(B, K, N, act, out, groups, group)
    pre = torch.full((B, n, N), float("nan"), dtype=torch.bfloat16, device="cuda") if "z" in parts else None
    o = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], p["residual"], first, pre=pre)
    assert o.dtype == DT[out]
    p64 = as64(p)
    o64, z64 = linear(p64, act, g)
    S = p64["x"].abs() @ p64["weight"].abs().t() + (p64["bias"].abs() if p["bias"] is not None else 0)
    zb = 2 * (K + 8) * U * S
    gate = p64["gate"][:, g] if p["gate"] is not None else torch.ones_like(z64)
    bound = gate.abs() * (1.13 * zb + (32 * U * z64.abs() if act != "none" else 0)) + 4 * U * (
        (gate * z64).abs() + (p64["residual"].abs() if p["residual"] is not None else 0))
    held(o, o64, bound, "o")
    if pre is not None:
        held(pre, z64, zb, "pre")

    gen = torch.Generator(device="cuda").manual_seed(9)
    dout = torch.randn((B, n, N), generator=gen, device="cuda").to(DT[out])
    got = tm.tm_linear_bwd(d, p["x"], p["weight"], dout, p["gate"], pre, first,
                           dbias=None if p["bias"] is not None else False)
    z = pre.double().requires_grad_() if pre is not None else torch.zeros_like(z64).requires_grad_()
    value = activate(z, act)
    slope, = torch.autograd.grad(value.sum(), z)
    value, z, d64 = value.detach(), z.detach(), dout.double()
    dz = d64 * gate * slope
    dzb = (64 * U if act != "none" else 4 * U) * (d64 * gate).abs() * (1 + z.abs())
    dzb_r = dzb + (2.0 ** -8 if B * n > 16 else 2.0 ** -16 if B * n > 4 else 0) * dz.abs()
    flat, xf, w = dz.view(-1, N), p64["x"].view(-1, K), p64["weight"]
    held(got.dx, dz @ w, dzb_r @ w.abs() + 2 * (N + 8) * U * (dz.abs() @ w.abs()), "dx")
    held(got.dweight, flat.t() @ xf, dzb_r.view(-1, N).t() @ xf.abs() + 2 * (B * n + 8) * U * (flat.abs().t() @ xf.abs()),
         "dweight")
    near(got.dx, dz @ w, "dx")
    near(got.dweight, flat.t() @ xf, "dweight")
    if p["bias"] is not None:
        held(got.dbias, flat.sum(0), dzb.view(-1, N).sum(0) + (B * n + 8) * U * flat.abs().sum(0), "dbias")
    else:
        assert got.dbias is None
    if p["gate"] is not None:
        t = d64 * value
        def sums(v):
            return torch.zeros((B, groups, N), dtype=torch.float64, device="cuda").index_add_(1, g, v)
        held(got.dgate, sums(t), sums((64 * U if act != "none" else 4 * U) * d64.abs() * (1 + z.abs())) + (n + 8) * U * sums(t.abs()), "dgate")
    else:
        assert got.dgate is None


# Tiles of 64, 128 and 256: of one to six stages (the loads run two or four ahead), the first one whole or what K
# leaves over 64; workgroups that take one tile or several; tiles shared out, in shares of one stage and of parts
# of two tiles.
STAGES = [(140, 64, 16), (18, 128, 96), (82, 192, 24), (25, 256, 64), (27, 448, 24), (35, 72, 32), (32, 136, 16), (24, 232, 16),
          (194, 72, 4336), (1676, 64, 4632), (2374, 128, 3376), (2382, 144, 3336), (8257, 208, 904), (174, 832, 16),
          (66, 8968, 32), (18, 8784, 2688), (7905, 328, 472), (76, 9024, 2056), (136, 5408, 3392), (1025, 136, 3952),
          (2308, 192, 3528), (3084, 256, 2720), (2482, 392, 4016)]


@pytest.mark.parametrize("n,K,N", STAGES)
def test_stages_rounds_and_shares(tm, n, K, N):
    test_forward_and_backward(tm, 1, n, K, N, "gelu", "bf16", "bz", 1, 0, 5)


def test_gradients_against_differences(tm):
    B, n, K, N, groups, group, first, act = 2, 7, 136, 72, 3, 4, 2, "gelu"
    p = make(B, n, K, N, "f32", "bgr", groups, 1)
    g = group_rows(B, n, groups, group, first, "cuda")
    d = tm.make_linear_desc(B, K, N, act, "f32", groups, group)
    pre = torch.empty((B, n, N), dtype=torch.bfloat16, device="cuda")
    tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], p["residual"], first, pre=pre)
    gen = torch.Generator(device="cuda").manual_seed(2)
    dout = torch.randn((B, n, N), generator=gen, device="cuda")
    got = tm.tm_linear_bwd(d, p["x"], p["weight"], dout, p["gate"], pre, first)
    p64 = as64(p)
    for name in ("x", "weight", "bias", "gate"):
        v = torch.randn(p[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        step = 1e-5
        plus, minus = (linear({**p64, name: p64[name] + s * step * v}, act, g)[0] for s in (1, -1))
        diff = float(((plus - minus) * dout.double()).sum()) / (2 * step)
        grad = getattr(got, "d" + name).double()
        # 14 rows: dz is not rounded; pre is bf16, within 2^-8 of z, and the slope changes by at most 1.6 of
        # that (value: 1.13), so an element's terms are off by 2^-8 * 1.6 |z| (largest |z| below 6) of at most
        # |dout gate| and the result's bf16 by 2^-8; their signs are random: a tenth of the sum of sizes
        dz_size = (dout.double().abs() * (p64["gate"].abs()[:, g] if name != "gate" else 1.0))
        reach = {"x": lambda: (dz_size @ p64["weight"].abs()), "weight": lambda: dz_size.view(-1, N).t() @ p64["x"].abs().view(-1, K),
                 "bias": lambda: dz_size.sum((0, 1)),
                 "gate": lambda: torch.zeros_like(p64["gate"]).index_add_(1, g, dz_size * 6)}[name]()
        bound = 0.1 * 2.0 ** -8 * (1 + 1.6 * 6) * float((reach * v.abs()).sum())
        say(f"  d{name}: differences {diff:.6g}, gradient {float((grad * v).sum()):.6g}, bound {bound:.2g}")
        assert abs(diff - float((grad * v).sum())) <= bound


def test_few_rows_and_tiles_agree_and_in_place(tm):
    """The forms for few rows and for tiles on the same rows, with and without a workspace, in place."""
    K, N = 20008, 776  # long enough that tiles are split
    p = make(1, 40, K, N, "f32", "br", 1, 3)
    d = tm.make_linear_desc(1, K, N, "silu", "f32")
    whole = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], None, p["residual"])
    some = tm.tm_linear_fwd(d, p["x"][:, :16].contiguous(), p["weight"], p["bias"], None, p["residual"][:, :16].contiguous())
    S = p["x"].double().abs() @ p["weight"].double().abs().t() + 3
    assert bool(((whole[:, :16] - some).double().abs() <= 4 * (K + 40) * U * S[:, :16]).all())
    o = p["residual"].clone()
    assert tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], None, o, o=o) is o
    assert torch.equal(o, whole)
    nbytes = tm.lib().tm_linear_fwd_workspace(d, 40)
    assert nbytes > 0
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")  # NaNs: nothing of it is read unwritten
    assert torch.equal(tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], None, p["residual"], workspace=ws), whole)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(whole)
    tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], None, p["residual"], o=out, stream=side)
    side.synchronize()
    assert bool(((whole - out).double().abs() <= 4 * (K + 40) * U * S).all())


@pytest.mark.parametrize("rows,K,N", [(24, 64, 64), (24, 4096, 64), (600, 4000, 2312), (2100, 96, 4104), (5000, 2000, 1032)])
def test_split_tiles_against_whole_ones(tm, rows, K, N):
    p = make(1, rows, K, N, "bf16", "b", 1, rows)
    d = tm.make_linear_desc(1, K, N, "none", "f32")
    o = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"])
    again = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"])
    assert torch.equal(o, again)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(o)
    tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], o=out, stream=side)
    side.synchronize()
    S = p["x"].float().abs() @ p["weight"].float().abs().t() + p["bias"].abs()
    bound = 2 * (K + 8) * U * S.double() * 1.01
    o64, _ = linear({**as64(p), "residual": None}, "none", torch.zeros(rows, dtype=torch.long, device="cuda"))
    for t, what in ((o, "split"), (out, "whole")):
        held(t, o64, bound, what)


def test_rows_behind_the_last_and_nan_rows(tm):
    """What lies behind the outputs stays as it was; a row with a NaN leaves the others' bits alone."""
    for n, K, N in ((3, 200, 72), (150, 200, 136)):
        p = make(1, n, K, N, "bf16", "b", 1, n)
        d = tm.make_linear_desc(1, K, N, "gelu", "bf16")
        want = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"])
        buf = torch.full((n * N + 512,), -3.0, dtype=torch.bfloat16, device="cuda")
        pre = buf.clone()
        tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], o=buf[:n * N].view(1, n, N), pre=pre[:n * N].view(1, n, N))
        assert torch.equal(buf[:n * N].view(1, n, N), want)
        assert bool((buf[n * N:] == -3).all()) and bool((pre[n * N:] == -3).all())
        x = p["x"].clone()
        x[0, n - 1, K - 1] = float("nan")
        x[0, 1, 0] = float("inf")
        got = tm.tm_linear_fwd(d, x, p["weight"], p["bias"])
        rows = [i for i in range(n) if i not in (1, n - 1)]
        assert torch.equal(got[:, rows], want[:, rows]) and bool(got[0, n - 1].isnan().all())
        dx = torch.full((n * K + 512,), -3.0, dtype=torch.bfloat16, device="cuda")
        dw = torch.full((N * K + 512,), -3.0, dtype=torch.bfloat16, device="cuda")
        pr = pre[:n * N].view(1, n, N)
        tm.tm_linear_bwd(d, p["x"], p["weight"], want, pre=pr, dx=dx[:n * K].view(1, n, K), dweight=dw[:N * K].view(N, K))
        assert bool((dx[n * K:] == -3).all()) and bool((dw[N * K:] == -3).all())


def test_large_arguments_of_the_activations(tm):
    """Sums far outside the activations' bend, finite gradients there, and none that are NaN."""
    z = torch.tensor([-3e38, -1e13, -1e4, -90, -20, -5, 0, 5, 20, 90, 1e4, 1e13, 3e38, 1, -1, 2], device="cuda")
    x = torch.zeros((1, 1, 16), dtype=torch.bfloat16, device="cuda")
    x[0, 0, 0] = 1
    w = torch.zeros((16, 16), dtype=torch.bfloat16, device="cuda")
    for act in ("gelu", "silu"):
        d = tm.make_linear_desc(1, 16, 16, act, "f32")
        pre = torch.empty((1, 1, 16), dtype=torch.bfloat16, device="cuda")
        o = tm.tm_linear_fwd(d, x, w, z.clone(), pre=pre)[0, 0].double()
        want = torch.where(z.double() > 50, z.double(), torch.where(z < -50, 0.0, activate(z.double().clamp(-60, 60), act)))
        assert bool(((o - want).abs() <= 40 * U * z.double().abs().clamp(max=60) + U * want.abs()).all())
        got = tm.tm_linear_bwd(d, x, w, torch.ones((1, 1, 16), device="cuda"), pre=pre)
        s = got.dbias.double()
        zz = pre[0, 0].double()
        t = zz.clamp(-60, 60).requires_grad_()
        slope, = torch.autograd.grad(activate(t, act).sum(), t)
        assert bool(((s - slope).abs() <= 64 * U * (1 + t.detach().abs())).all())


def test_no_tokens_and_parts_of_the_gradients(tm):
    p = make(1, 64, 72, 200, "bf16", "bg", 3, 5)
    d = tm.make_linear_desc(1, 72, 200, "silu", "bf16", 3, 30)
    e = torch.empty((1, 0, 72), dtype=torch.bfloat16, device="cuda")
    o = tm.tm_linear_fwd(d, e, p["weight"], p["bias"], p["gate"])
    assert o.shape == (1, 0, 200)
    got = tm.tm_linear_bwd(d, e, p["weight"], o, p["gate"], o, 0)
    assert got.dx.shape == (1, 0, 72)
    assert all(bool((t == 0).all()) for t in got[1:])
    pre = torch.empty((1, 64, 200), dtype=torch.bfloat16, device="cuda")
    o = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], pre=pre)
    all_ = tm.tm_linear_bwd(d, p["x"], p["weight"], o, p["gate"], pre)
    for i, name in enumerate(("dx", "dweight", "dbias", "dgate")):
        only = {k: False for k in ("dx", "dweight", "dbias", "dgate") if k != name}
        got = tm.tm_linear_bwd(d, p["x"], p["weight"], o, p["gate"], pre, **only)
        assert torch.equal(got[i], all_[i]) and sum(t is not None for t in got) == 1


@pytest.mark.parametrize("rows", [5, 300])
def test_captured_calls(tm, rows):
    p = make(1, rows, 520, 1032, "f32", "bgr", 4, 7)
    d = tm.make_linear_desc(1, 520, 1032, "gelu", "f32", 4, 100)
    pre = torch.empty((1, rows, 1032), dtype=torch.bfloat16, device="cuda")
    dout = torch.randn((1, rows, 1032), device="cuda")
    nbytes = tm.lib().tm_linear_fwd_workspace(d, rows)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    o = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], p["residual"], pre=pre, workspace=ws)
    want = tm.tm_linear_bwd(d, p["x"], p["weight"], dout, p["gate"], pre)
    graph = torch.cuda.CUDAGraph()
    pre2 = torch.empty_like(pre)
    with torch.cuda.graph(graph):
        o2 = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], p["residual"], pre=pre2, workspace=ws)
        got = tm.tm_linear_bwd(d, p["x"], p["weight"], dout, p["gate"], pre2)
    for _ in range(3):
        for t in (o2, pre2, *got):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o2, o) and torch.equal(pre2, pre)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        tm.tm_linear_bwd(d, p["x"], p["weight"], dout, p["gate"], pre)


@pytest.mark.parametrize("rows", [3, 8, 40])
def test_infinite_gradients_stay_in_their_rows(tm, rows):
    """An infinity in dout makes its row of dx and of dweight infinite, not NaN, and no other."""
    K, N = 72, 136
    p = make(1, rows, K, N, "f32", "", 1, 3)
    p["weight"] = p["weight"].abs()  # no cancellation of infinities: sums are +inf
    d = tm.make_linear_desc(1, K, N, "none", "f32")
    dout = torch.randn((1, rows, N), device="cuda")
    want = tm.tm_linear_bwd(d, p["x"], p["weight"], dout)
    dout[0, 1, 5] = float("inf")
    got = tm.tm_linear_bwd(d, p["x"], p["weight"], dout)
    others = [i for i in range(rows) if i != 1]
    assert torch.equal(got.dx[:, others], want.dx[:, others])
    assert bool((got.dx[0, 1] == float("inf")).all())
    cols = [i for i in range(N) if i != 5]
    assert torch.equal(got.dweight[cols], want.dweight[cols])
    assert bool((~got.dweight[5].isfinite()).all()) and not bool(got.dweight[5].isnan().any())


@pytest.mark.parametrize("rows", [1, 3, 8, 16, 40])
def test_infinite_inputs_of_the_backward(tm, rows):
    """An infinity in weight makes its column of dx infinite, one in x its column of dweight, with the signs of dz,
    whether dz goes into the products as one number or as two."""
    K, N = 72, 136
    p = make(1, rows, K, N, "f32", "", 1, 41)
    p["weight"][7, 3] = float("inf")
    p["x"][0, rows - 1, 9] = float("-inf")
    d = tm.make_linear_desc(1, K, N, "none", "f32")
    gen = torch.Generator(device="cuda").manual_seed(42)
    dout = torch.randn((1, rows, N), generator=gen, device="cuda")
    dout[0, :, 7] += 0.1 * torch.sign(dout[0, :, 7])
    got = tm.tm_linear_bwd(d, p["x"], p["weight"], dout, dbias=False)
    assert torch.equal(got.dx[0, :, 3].float(), torch.sign(dout[0, :, 7]) * float("inf"))
    assert torch.equal(got.dweight[:, 9].float(), torch.sign(dout[0, rows - 1]) * float("-inf"))
    columns = torch.arange(K, device="cuda")
    assert bool(got.dx[..., columns != 3].isfinite().all()) and bool(got.dweight[:, columns != 9].isfinite().all())


def test_gradients_without_what_they_do_not_need(tm):
    p = make(1, 40, 72, 200, "bf16", "", 1, 4)
    d = tm.make_linear_desc(1, 72, 200)
    dout = torch.randn((1, 40, 200), device="cuda").to(torch.bfloat16)
    want = tm.tm_linear_bwd(d, p["x"], p["weight"], dout)
    assert torch.equal(tm.tm_linear_bwd(d, None, p["weight"], dout, dweight=False).dx, want.dx)
    assert torch.equal(tm.tm_linear_bwd(d, p["x"], None, dout, dx=False).dweight, want.dweight)
    for args in ((None, p["weight"]), (p["x"], None)):
        with pytest.raises(tm.TMError) as e:
            tm.tm_linear_bwd(d, *args, dout)
        assert e.value.status == tm.TM_E_ARG


@pytest.mark.parametrize("n,K,N,act,out,parts", [(700, 2056, 7688, "gelu", "bf16", "bz"), (2900, 1032, 5128, "silu", "f32", "bgr"),
                                                 (1500, 6000, 5000, "none", "f32", "br")])
def test_large_tiles(tm, n, K, N, act, out, parts):
    """Sizes that the 256-wide tiles take, several to a workgroup and some of them split, rows and columns that
    end inside tiles, each kind of epilogue; held to the bounds above, sizes in fp32 (1.01 for its roundings)."""
    p = make(1, n, K, N, out, parts, 5, n)
    g = group_rows(1, n, 5, 600, 20, "cuda")
    d = tm.make_linear_desc(1, K, N, act, out, 5, 600)
    pre = torch.empty((1, n, N), dtype=torch.bfloat16, device="cuda") if "z" in parts else None
    o = tm.tm_linear_fwd(d, p["x"], p["weight"], p["bias"], p["gate"], p["residual"], 20, pre=pre)
    o64, z64 = linear(as64(p), act, g)
    S = 1.01 * (p["x"].float().abs() @ p["weight"].float().abs().t() + p["bias"].abs()).double()
    zb = 2 * (K + 8) * U * S
    gate = p["gate"].double()[:, g] if p["gate"] is not None else torch.ones((), device="cuda", dtype=torch.float64)
    held(o, o64, gate.abs() * (1.13 * zb + 32 * U * z64.abs()) + 4 * U * (
        (gate * z64).abs() + (p["residual"].double().abs() if p["residual"] is not None else 0)), "o")
    if pre is not None:
        held(pre, z64, zb, "pre")
    near(o, o64, "o")


def test_offsets_past_32_bits(tm):
    """More than 2^31 elements of output and of dout: the last rows, and sums that reach over all of them."""
    n, K, N = 70000, 64, 32768
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, n, K), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((N, K), generator=g, device="cuda") / 8).to(torch.bfloat16)
    b = torch.randn((N,), generator=g, device="cuda")
    d = tm.make_linear_desc(1, K, N, "silu", "bf16")
    o = tm.tm_linear_fwd(d, x, w, b)
    rows = torch.tensor([0, 1, 65535, 65536, n - 300, n - 1], device="cuda")
    z = x[0, rows].double() @ w.double().t() + b.double()
    S = x[0, rows].double().abs() @ w.double().abs().t() + b.double().abs()
    held(o[0, rows], activate(z, "silu"), 1.13 * 2 * (K + 8) * U * S + 32 * U * z.abs(), "o")
    # dout = o: dx of these rows, and dweight's columns of ones times a known sum
    d = tm.make_linear_desc(1, K, N, "none", "bf16")
    got = tm.tm_linear_bwd(d, x, w, o)
    want = o[0, rows].double() @ w.double()
    held(got.dx[0, rows], want, 2 * (N + 8) * U * (o[0, rows].double().abs() @ w.double().abs()), "dx")
    cols = torch.tensor([0, 1, N - 1], device="cuda")
    oc = o[0][:, cols].double()
    held(got.dweight[cols], oc.t() @ x[0].double(), 2 * (n + 8) * U * (oc.abs().t() @ x[0].double().abs()), "dweight")
    held(got.dbias[cols], oc.sum(0), (n + 8) * U * oc.abs().sum(0), "dbias")


# Runs that begin and end inside groups: over the border of two groups of many more tokens than the run, over
# whole groups and parts of two, few rows on both sides of a border.
@pytest.mark.parametrize("B,n,K,N,groups,group,first", [(1, 300, 64, 520, 2, 4000, 3850), (1, 61, 136, 72, 2, 2 ** 28, 2 ** 28 - 1),
                                                        (2, 700, 72, 264, 3, 600, 500), (1, 12, 72, 1032, 2, 100, 97),
                                                        (1, 3, 72, 136, 2, 100, 98), (3, 1000, 64, 64, 4, 400, 250)])
def test_runs_that_cut_their_groups(tm, B, n, K, N, groups, group, first):
    test_forward_and_backward(tm, B, n, K, N, "silu", "f32", "bgrz", groups, group, first)


# (every kernel variant, by tests/block_sizes.py and the host's check of its plans)
KINDS = [("gelu", "bf16", "bz", 1, 0, 5), ("silu", "f32", "bgrz", 9, 900, 40), ("none", "f32", "bgrz", 1, 0, 0)]


@pytest.mark.parametrize("n,K,N", PRODUCTS)
def test_every_variant_of_the_products(tm, n, K, N):
    for kind in KINDS:
        test_forward_and_backward(tm, 1, n, K, N, *kind)


@pytest.mark.parametrize("n,K,N", FEW_ROWS)
def test_every_variant_of_few_rows(tm, n, K, N):
    for kind in KINDS:
        test_forward_and_backward(tm, 1, n, K, N, *kind)
