"""Norms around a block (tm_block_norm_*) against the definition in 64 bits.

Tolerances, in units u = 2^-24 (half an fp32 step, relative). A sum over a row of E <= 16384 is 20 terms in a
lane, a tree of 6 and at most 16 waves' sums: 42 roundings, so a mean is off by at most 42 u of the mean
magnitude, a mean of squares by 44 u of itself plus, for a layer norm, 2 * 42 u of (mean |v|)^2-sized terms, and
1 / sqrt of it by half of that and 3 u more. An element of a norm is then within 64 u of its own size and 64 u of
(largest |v|) / sigma, sigma the root. The affine steps add at most 8 u of the terms they add up. So a forward
output is held to 128 u times the sum of its terms' sizes with |n| replaced by |n| + max |v| / sigma, and half a
step (2^-8 relative) more where it is bf16; with a norm on both sides the first one's error passes through the
second, whose slope is at most 1 / sigma (times 2): another 128 u of the size of what r was made of.
The backward is a chain of the same sums: 512 u of the sum of its terms' sizes with means replaced by the
largest magnitudes. A sum over rows of R terms adds (R + 64) u of the sum of their sizes.
"""
import itertools

import pytest
import torch

from block_reference import as64, block_norm, group_rows, normed
from block_sizes import SUMS
from gpu_helpers import say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("x", "y", "gate", "post_weight", "pre_weight", "pre_bias", "scale", "shift")


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def make(B, n, E, stream, act, parts, groups, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, size=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * size).to(dtype)

    p = dict.fromkeys(NAMES)
    size = torch.exp(0.7 * normal((E,)))
    p["x"] = (normal((B, n, E)) * size + 0.3).to(DT[stream])
    if "y" in parts:
        p["y"] = normal((B, n, E), 1.0, DT[act])
    for name, key, mean in (("post_weight", "p", 1), ("pre_weight", "w", 1), ("pre_bias", "b", 0)):
        if key in parts:
            p[name] = mean + normal((E,), 0.2)
    if "g" in parts:
        p["gate"] = normal((B, groups, E), 0.5)
    if "m" in parts:
        p["scale"], p["shift"] = normal((B, groups, E), 0.3), normal((B, groups, E), 0.3)
    return p


def sizes(p, pre, post, g):
    """The sum of the sizes of the terms of r and of h, by the header's rules."""
    q = {k: None if v is None else v.abs() for k, v in p.items()}

    def spread(v, kind):
        if kind == "none":
            return v.abs()
        c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        sigma = torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
        return normed(v, kind, EPS).abs() + v.abs().amax(-1, keepdim=True) / sigma

    r, _ = block_norm(p, pre, post, EPS, g)
    rs = q["x"]
    if p["y"] is not None:
        z = spread(p["y"], post)
        z = z * q["post_weight"] if q["post_weight"] is not None else z
        rs = rs + (z * q["gate"][:, g] if q["gate"] is not None else z)
    if pre == "none":
        return rs, None
    c = r - r.mean(-1, keepdim=True) if pre == "layer" else r
    sigma = torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    m = spread(r, pre) + 2 * (rs + rs.mean(-1, keepdim=True)) / sigma
    m = m * q["pre_weight"] if q["pre_weight"] is not None else m
    m = m + q["pre_bias"] if q["pre_bias"] is not None else m
    if q["scale"] is not None:
        m = m * (1 + q["scale"][:, g]) + q["shift"][:, g]
    return rs, m


def held(got, want, bound, what):
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs()
    err = (got.double() - want).abs()
    worst = float((err / bound.clamp_min(1e-300)).max()) if err.numel() else 0.0
    say(f"  {what}: largest error / bound = {worst:.3f}")
    assert bool((err <= bound).all()), what


def run_forward(tm, p, pre, post, act, stream, groups, group, first, **kw):
    B, n, E = p["x"].shape
    d = tm.make_block_norm_desc(B, E, pre, post, act, stream, EPS, groups, group)
    return d, tm.tm_block_norm_fwd(d, p["x"], *[p[k] for k in NAMES[1:]], first, **kw)


SHAPES = [(1, 1, 8, 1, 0, 0), (2, 9, 128, 3, 4, 1), (3, 5, 136, 1, 0, 0), (1, 67, 256, 1, 0, 3), (2, 6, 264, 1, 0, 0),
          (2, 400, 264, 900, 1, 37), (2, 1500, 1032, 800, 2, 30), (1, 19000, 64, 600, 33, 100),
          (1, 1, 5120, 1, 0, 9), (2, 7, 64, 3, 4, 2), (3, 33, 1000, 5, 10, 7), (1, 130, 1024, 2, 100, 30),
          (2, 5, 2056, 9, 1, 3), (1, 3, 16384, 1, 0, 0), (1, 9, 16376, 4, 3, 1), (2, 3, 8200, 1, 0, 0), (1, 300, 264, 1, 4000, 11)]
SETS = [("layer", "none", "m"), ("layer", "none", "ygm"), ("rms", "rms", "ypw"), ("none", "layer", "ygp"),
        ("rms", "layer", "ygpwbm"), ("layer", "none", "wb"), ("layer", "rms", "yb"), ("none", "none", "yg")]


@pytest.mark.parametrize("B,n,E,groups,group,first", SHAPES)
@pytest.mark.parametrize("pre,post,parts", SETS)
def test_forward_and_backward(tm, B, n, E, groups, group, first, pre, post, parts):
    for stream, act in itertools.product(("f32", "bf16"), repeat=2):
        p = make(B, n, E, stream, act, parts, groups, E + n)
        g = group_rows(B, n, groups, group, first, "cuda")
        p64 = as64(p)
        rs, hs = sizes(p64, pre, post, g)
        d, (r, h) = run_forward(tm, p, pre, post, act, stream, groups, group, first)
        r64, h64 = block_norm(p64, pre, post, EPS, g)
        what = f"{stream} {act}"
        if "y" in parts:
            assert r.dtype == DT[stream]
            held(r, r64, 128 * U * rs, what + " r")
        else:
            assert r is None
        if pre != "none":
            assert h.dtype == DT[act]
            held(h, h64, 128 * U * hs, what + " h")
        else:
            assert h is None
        backward(tm, d, p, pre, post, act, stream, groups, g, first, r if r is not None else p["x"], what)


def gradients64(p, pre, post, g, r_in, dh, dr):
    """The gradients' formulas in 64 bits at the r that the call is given, and the sizes of their terms."""
    q = as64(p)
    out, size = {}, {}
    a, asz = (dr, dr.abs()) if dr is not None else (torch.zeros_like(r_in), torch.zeros_like(r_in))

    def sums(v):
        t = torch.zeros((v.shape[0], sums.groups, v.shape[2]), dtype=v.dtype, device=v.device)
        return t.index_add_(1, g, v)

    sums.groups = 1 if q["gate"] is None and q["scale"] is None else (q["gate"] if q["gate"] is not None else q["scale"]).shape[1]

    def slope(t, tsz, v, kind):
        """t times the Jacobian of the norm at v, and its size."""
        if kind == "none":
            return t, tsz
        c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        sigma = torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
        n = c / sigma
        big = n.abs() + v.abs().amax(-1, keepdim=True) / sigma
        res = (t - (t.mean(-1, keepdim=True) if kind == "layer" else 0) - n * (t * n).mean(-1, keepdim=True)) / sigma
        return res, (tsz + tsz.mean(-1, keepdim=True) + big * (tsz * big).mean(-1, keepdim=True)) / sigma

    def spread(v, kind):
        if kind == "none":
            return v.abs()
        c = v - v.mean(-1, keepdim=True) if kind == "layer" else v
        sigma = torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
        return (c / sigma).abs() + v.abs().amax(-1, keepdim=True) / sigma

    if pre != "none":
        n, nsz = normed(r_in, pre, EPS), spread(r_in, pre)
        t = dh
        if q["scale"] is not None:
            m, msz = n, nsz
            if q["pre_weight"] is not None:
                m, msz = m * q["pre_weight"], msz * q["pre_weight"].abs()
            if q["pre_bias"] is not None:
                m, msz = m + q["pre_bias"], msz + q["pre_bias"].abs()
            out["dscale"], size["dscale"] = sums(dh * m), sums(dh.abs() * msz)
            out["dshift"], size["dshift"] = sums(dh), sums(dh.abs())
            t = t * (1 + q["scale"][:, g])
        if q["pre_bias"] is not None:
            out["dpre_bias"], size["dpre_bias"] = t.sum((0, 1)), t.abs().sum((0, 1))
        if q["pre_weight"] is not None:
            out["dpre_weight"], size["dpre_weight"] = (t * n).sum((0, 1)), (t.abs() * nsz).sum((0, 1))
            t = t * q["pre_weight"]
        more, msz = slope(t, t.abs(), r_in, pre)
        a, asz = a + more, asz + msz
    out["dx"], size["dx"] = a, asz
    if q["y"] is not None:
        v, vsz = normed(q["y"], post, EPS), spread(q["y"], post)
        u, usz = a, asz
        if q["gate"] is not None:
            w = q["post_weight"] if q["post_weight"] is not None else 1.0
            out["dgate"] = sums(a * v * w)
            size["dgate"] = sums(asz * vsz * (w.abs() if q["post_weight"] is not None else 1.0))
            u, usz = u * q["gate"][:, g], usz * q["gate"][:, g].abs()
        if q["post_weight"] is not None:
            out["dpost_weight"], size["dpost_weight"] = (u * v).sum((0, 1)), (usz * vsz).sum((0, 1))
            u, usz = u * q["post_weight"], usz * q["post_weight"].abs()
        out["dy"], size["dy"] = slope(u, usz, q["y"], post)
    return out, size


def backward(tm, d, p, pre, post, act, stream, groups, g, first, r, what):
    B, n, E = r.shape
    gen = torch.Generator(device="cuda").manual_seed(5)
    dh = torch.randn(r.shape, generator=gen, device="cuda").to(DT[act]) if pre != "none" else None
    dr = torch.randn(r.shape, generator=gen, device="cuda").to(DT[stream])
    for with_dr in ((True, False) if pre != "none" else (True,)):
        got = tm.tm_block_norm_bwd(d, r if pre != "none" else None, dh, dr if with_dr else None,
                                   *[p[k] for k in NAMES[1:]], first)
        want, size = gradients64(p, pre, post, g, r.double(), None if dh is None else dh.double(),
                                 dr.double() if with_dr else None)
        for name, t in got._asdict().items():
            assert (t is None) == (name not in want), name
            if t is not None:
                terms = 512 if name in ("dx", "dy") else 512 + B * n + 64
                held(t, want[name].expand(t.shape), terms * U * size[name], f"{what} {name}")


def test_gradients_against_differences(tm):
    B, n, E, groups, group, first = 2, 21, 136, 4, 7, 3
    pre, post = "layer", "rms"
    p = make(B, n, E, "f32", "f32", "ygpwbm", groups, 1)
    g = group_rows(B, n, groups, group, first, "cuda")
    p64 = as64(p)
    gen = torch.Generator(device="cuda").manual_seed(2)
    ch, cr = (torch.randn((B, n, E), generator=gen, device="cuda") for _ in range(2))
    d, (r, h) = run_forward(tm, p, pre, post, "f32", "f32", groups, group, first)
    got = tm.tm_block_norm_bwd(d, r, ch, cr, *[p[k] for k in NAMES[1:]], first)

    def loss(q):
        r64, h64 = block_norm(q, pre, post, EPS, g)
        return float((h64 * ch.double()).sum() + (r64 * cr.double()).sum())

    for name in NAMES:
        v = torch.randn(p[name].shape, generator=gen, device="cuda", dtype=torch.float64)
        step = 1e-5
        diff = (loss({**p64, name: p64[name] + step * v}) - loss({**p64, name: p64[name] - step * v})) / (2 * step)
        grad = getattr(got, "d" + name).double()
        # differences: third derivatives times step^2 (1e-10), and the loss' own 2^-52 times its terms / step;
        # the gradient: within 2000 u of its terms' sizes, which are at most 100 times the largest element
        bound = float(grad.abs().max()) * float(v.abs().sum()) * (2000 * U + 1e-6) + 1e-5
        say(f"  d{name}: differences {diff:.8g}, gradient {float((grad * v).sum()):.8g}, bound {bound:.2g}")
        assert abs(diff - float((grad * v).sum())) <= bound


def test_in_place_and_given_outputs(tm):
    p = make(2, 50, 520, "f32", "bf16", "ygm", 6, 3)
    d, (r, h) = run_forward(tm, p, "layer", "none", "bf16", "f32", 6, 10, 5)
    x = p["x"].clone()
    h2 = torch.full_like(h, float("nan"))
    out = tm.tm_block_norm_fwd(d, x, p["y"], p["gate"], scale=p["scale"], shift=p["shift"], first_token=5, r=x, h=h2)
    assert out[0] is x and out[1] is h2
    assert torch.equal(x, r) and torch.equal(h2, h)
    dh, dr = torch.randn_like(h), torch.randn_like(r)
    args = (p["y"], p["gate"], None, None, None, p["scale"], p["shift"], 5)
    want = tm.tm_block_norm_bwd(d, r, dh, dr, *args)
    dr2, dh2 = dr.clone(), dh.clone()
    got = tm.tm_block_norm_bwd(d, r, dh2, dr2, *args, dx=dr2, dy=dh2)
    assert got.dx is dr2 and got.dy is dh2
    for a, b in zip(want, got):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    some = tm.tm_block_norm_bwd(d, r, dh, dr, *args, dgate=False, dscale=False)
    assert some.dgate is None and some.dscale is None and torch.equal(some.dshift, want.dshift)
    ws = torch.empty(tm.lib().tm_block_norm_bwd_workspace(d, 50, 5), dtype=torch.uint8, device="cuda")
    for a, b in zip(want, tm.tm_block_norm_bwd(d, r, dh, dr, *args, workspace=ws)):
        assert a is None or torch.equal(a, b)


def test_rows_keep_to_themselves(tm):
    """An infinity or a NaN in one row leaves the others' bits alone, and no row at all is a call too."""
    p = make(1, 40, 1024, "f32", "f32", "ygm", 4, 4)
    d, (r, h) = run_forward(tm, p, "layer", "rms", "f32", "f32", 4, 10, 0)
    q = dict(p, x=p["x"].clone(), y=p["y"].clone())
    q["x"][0, 7, 5], q["y"][0, 20, 1000] = float("nan"), float("inf")
    _, (r2, h2) = run_forward(tm, q, "layer", "rms", "f32", "f32", 4, 10, 0)
    rows = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(r[:, rows], r2[:, rows]) and torch.equal(h[:, rows], h2[:, rows])
    assert bool(h2[0, 7].isnan().all()) and bool(h2[0, 20].isnan().all())
    # a row of zeros: n = 0 / sqrt(eps)
    z = dict(p, x=torch.zeros_like(p["x"]), y=torch.zeros_like(p["y"]))
    _, (r3, h3) = run_forward(tm, z, "layer", "rms", "f32", "f32", 4, 10, 0)
    g = group_rows(1, 40, 4, 10, 0, "cuda")
    assert bool((r3 == 0).all()) and torch.equal(h3, p["shift"][:, g])
    e = {k: v[:, :0] if k in ("x", "y") else v for k, v in p.items()}
    d0, (r0, h0) = run_forward(tm, e, "layer", "rms", "f32", "f32", 4, 10, 0)
    assert r0.shape == h0.shape == (1, 0, 1024)
    got = tm.tm_block_norm_bwd(d0, r0, h0, r0, *[e[k] for k in NAMES[1:]], 0)
    assert all(bool((t == 0).all()) for t in got if t is not None) and got.dgate.shape == (1, 4, 1024)


def test_groups_without_a_token_get_zeros_and_runs_add_up(tm):
    """Two calls on the halves of a run give the rows of the whole, and gradients that add up to it."""
    B, n, E, groups, group, first = 1, 90, 512, 8, 20, 30
    p = make(B, n, E, "f32", "f32", "ygm", groups, 6)
    d, (r, h) = run_forward(tm, p, "layer", "none", "f32", "f32", groups, group, first)
    dh, dr = torch.randn_like(h), torch.randn_like(r)
    rest = (p["gate"], None, None, None, p["scale"], p["shift"])
    whole = tm.tm_block_norm_bwd(d, r, dh, dr, p["y"], *rest, first)
    assert bool((whole.dgate[:, 0] == 0).all()) and bool((whole.dscale[:, 6:] == 0).all())
    halves = []
    for t0, t1 in ((0, 37), (37, 90)):
        q = {k: v[:, t0:t1].contiguous() if k in ("x", "y") else v for k, v in p.items()}
        _, (rr, hh) = run_forward(tm, q, "layer", "none", "f32", "f32", groups, group, first + t0)
        assert torch.equal(rr, r[:, t0:t1]) and torch.equal(hh, h[:, t0:t1])
        halves.append(tm.tm_block_norm_bwd(d, rr, dh[:, t0:t1].contiguous(), dr[:, t0:t1].contiguous(), q["y"], *rest, first + t0))
    for name in ("dgate", "dscale", "dshift"):
        a, b = (getattr(x, name).double() for x in halves)
        w = getattr(whole, name).double()
        # sums of at most 20 terms of size below 5 * 5 * 5
        assert bool(((a + b - w).abs() <= 100 * U * 20 * 125).all()), name


def test_captured_calls_and_other_streams(tm):
    p = make(1, 700, 1024, "f32", "bf16", "ygm", 7, 8)
    d, (r, h) = run_forward(tm, p, "layer", "none", "bf16", "f32", 7, 100, 0)
    dh, dr = torch.randn_like(h), torch.randn_like(r)
    rest = (p["y"], p["gate"], None, None, None, p["scale"], p["shift"], 0)
    want = tm.tm_block_norm_bwd(d, r, dh, dr, *rest)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r2, h2 = tm.tm_block_norm_fwd(d, p["x"], p["y"], p["gate"], scale=p["scale"], shift=p["shift"])
        got = tm.tm_block_norm_bwd(d, r2, dh, dr, *rest)
    for _ in range(3):
        for t in (r2, h2, *got):
            if t is not None:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r2, r) and torch.equal(h2, h)
        for a, b in zip(want, got):
            assert a is None or torch.equal(a, b)
        tm.tm_block_norm_bwd(d, r, dh, dr, *rest)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with pytest.raises(tm.TMError) as e:
        tm.tm_block_norm_bwd(d, r, dh, dr, *rest, stream=side)
    assert e.value.status == tm.TM_E_ARG and "workspace" in str(e.value)
    ws = torch.empty(tm.lib().tm_block_norm_bwd_workspace(d, 700, 0), dtype=torch.uint8, device="cuda")
    outs = dict(dx=torch.empty_like(r), dy=torch.empty_like(p["y"]), dgate=torch.empty_like(p["gate"]),
                dscale=torch.empty_like(p["gate"]), dshift=torch.empty_like(p["gate"]))
    side.wait_stream(torch.cuda.current_stream())
    got = tm.tm_block_norm_bwd(d, r, dh, dr, *rest, workspace=ws, stream=side, **outs)
    side.synchronize()
    for a, b in zip(want, got):
        assert a is None or torch.equal(a, b)


def test_more_rows_than_one_launch_takes(tm):
    """Thread numbers are 32 bits: 2^25 rows of one wave each take a second launch."""
    n, E = 2 ** 25 + 1000, 8
    x = torch.randn((1000, E), device="cuda").repeat(n // 1000 + 1, 1)[:n].to(torch.bfloat16).view(1, n, E)
    d = tm.make_block_norm_desc(1, E, "layer", "none", "bf16", "bf16")
    _, h = tm.tm_block_norm_fwd(d, x)
    _, want = tm.tm_block_norm_fwd(d, x[:, :1000].contiguous())
    assert torch.equal(h[:, :1000], want)
    at = (2 ** 25 // 1000) * 1000  # a multiple of the period, below the second launch's first row
    assert torch.equal(h[:, at:at + 1000], want) and torch.equal(h[:, n - 500:], h[:, n - 500 - at:n - at])


def test_offsets_past_32_bits(tm):
    """More than 2^31 elements: the last rows, forward and backward."""
    n, E = 135000, 16000
    x = torch.randn((1000, E), device="cuda").to(torch.bfloat16).repeat(n // 1000, 1).view(1, n, E)
    d = tm.make_block_norm_desc(1, E, "rms", "none", "bf16", "bf16")
    w = 1 + 0.2 * torch.randn((E,), device="cuda")
    _, h = tm.tm_block_norm_fwd(d, x, pre_weight=w)
    _, want = tm.tm_block_norm_fwd(d, x[:, :1000].contiguous(), pre_weight=w)
    assert torch.equal(h[:, :1000], want) and torch.equal(h[:, -1000:], want)
    got = tm.tm_block_norm_bwd(d, x, h, pre_weight=w)
    part = tm.tm_block_norm_bwd(d, x[:, :1000].contiguous(), want, pre_weight=w)
    assert torch.equal(got.dx[:, -1000:], part.dx)
    # 135 times the period's sum, each within its terms' roundings
    n64 = normed(x[0, :1000].double(), "rms", EPS)
    t = want[0].double() * n64
    held(got.dpre_weight, 135 * t.sum(0), (512 + n + 64) * U * 135 * t.abs().sum(0), "dpre_weight")


@pytest.mark.parametrize("pre", ["none", "layer"])
@pytest.mark.parametrize("E", [136, 1032, 8200])
@pytest.mark.parametrize("act", ["f32", "bf16"])
def test_gradient_of_an_output_that_no_norm_takes_does_not_read_it(tm, E, act, pre):
    """Without a norm after the branch dy is gate * post_weight * dx: the same bits whatever y holds, an infinity or
    a NaN too, and the sums over rows of the other columns stay as they are."""
    B, n, groups, group = 1, 23, 3, 10
    p = make(B, n, E, "f32", act, "ygp", groups, E)
    d = tm.make_block_norm_desc(B, E, pre, "none", act, "f32", EPS, groups, group)
    gen = torch.Generator(device="cuda").manual_seed(7)
    dr = torch.randn((B, n, E), generator=gen, device="cuda")
    r, dh = (p["x"], torch.randn((B, n, E), generator=gen, device="cuda").to(DT[act])) if pre != "none" else (None, None)
    want = tm.tm_block_norm_bwd(d, r, dh, dr, p["y"], p["gate"], p["post_weight"])
    y = p["y"].clone()
    cols = [3, 64, E - 1]
    for row, col, v in zip((0, 11, n - 1), cols, ("inf", "-inf", "nan")):
        y[0, row, col] = float(v)
    got = tm.tm_block_norm_bwd(d, r, dh, dr, y, p["gate"], p["post_weight"])
    assert bool(want.dy.isfinite().all()) and torch.equal(got.dy, want.dy) and torch.equal(got.dx, want.dx)
    others = [c for c in range(E) if c not in cols]
    assert torch.equal(got.dgate[..., others], want.dgate[..., others])
    assert torch.equal(got.dpost_weight[others], want.dpost_weight[others])
    assert not bool(got.dpost_weight[cols].isfinite().any())


# Runs that begin and end inside groups: over the border of two groups of many more tokens than the run, with one
# token on either side, over several whole groups and parts of two, more groups than parts.
CUT = [(1, 300, 264, 2, 4000, 3850), (2, 200, 1024, 2, 3000, 2900), (1, 61, 5120, 2, 2 ** 28, 2 ** 28 - 1),
       (1, 61, 64, 2, 2 ** 28, 2 ** 28 - 60), (2, 700, 1000, 3, 600, 500), (1, 802, 8200, 3, 800, 799),
       (3, 1000, 136, 4, 400, 250), (2, 1500, 72, 400, 4, 3), (5, 1, 2056, 2, 30, 30)]


@pytest.mark.parametrize("B,n,E,groups,group,first", CUT)
def test_runs_that_cut_their_groups(tm, B, n, E, groups, group, first):
    test_forward_and_backward(tm, B, n, E, groups, group, first, "rms", "layer", "ygpwbm")


def test_infinite_modulations_of_a_cut_group(tm):
    """Infinities in the gate and the scale of a run's first and last group, of which it has a few tokens, make the
    weights' gradients infinite in their columns, not NaN, and leave the others' bits alone."""
    n, E, groups, group, first = 290, 264, 3, 200, 180
    p = make(1, n, E, "f32", "f32", "ygpwm", groups, 11)
    d = tm.make_block_norm_desc(1, E, "none", "none", "f32", "f32", EPS, groups, group)
    p["y"], dr = p["y"].abs() + 0.1, torch.rand((1, n, E), device="cuda") + 0.1
    want = tm.tm_block_norm_bwd(d, None, None, dr, p["y"], p["gate"], p["post_weight"], first_token=first)
    gate = p["gate"].clone()
    gate[0, 0, 5], gate[0, 2, 9] = float("inf"), float("-inf")
    got = tm.tm_block_norm_bwd(d, None, None, dr, p["y"], gate, p["post_weight"], first_token=first)
    assert float(got.dpost_weight[5]) == float("inf") and float(got.dpost_weight[9]) == float("-inf")
    others = [c for c in range(E) if c not in (5, 9)]
    assert torch.equal(got.dpost_weight[others], want.dpost_weight[others]) and torch.equal(got.dgate, want.dgate)
    d = tm.make_block_norm_desc(1, E, "layer", "none", "f32", "f32", EPS, groups, group)
    scale = p["scale"].clone()
    scale[0, 0, 5], scale[0, 2, 9] = float("inf"), float("inf")
    dh = dr  # (the sums are of dh, and of dh * n, without the scale)
    bias = torch.zeros((E,), device="cuda")
    got = tm.tm_block_norm_bwd(d, p["x"], dh, dr, pre_bias=bias, scale=scale, shift=p["shift"], first_token=first)
    assert bool((got.dpre_bias[[5, 9]] == float("inf")).all())
    assert bool(got.dpre_bias[others].isfinite().all()) and bool(got.dscale.isfinite().all())


@pytest.mark.parametrize("B,n,E,groups,group,first", SUMS)
def test_every_variant_of_the_sums(tm, B, n, E, groups, group, first):
    test_forward_and_backward(tm, B, n, E, groups, group, first, "layer", "rms", "ygpwbm")
