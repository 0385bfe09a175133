"""Tensors that the block norms and the linear layers refuse: outputs that overlap another tensor of the call, but for
the pairs that may be the same, tensors that are not contiguous, not aligned or too short for the call. A refused call
writes nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def refused(tm, message, fn, *tensors):
    """fn is refused with TM_E_ARG and this message, and the tensors keep their bits."""
    before = [t.clone() for t in tensors]
    with pytest.raises(tm.TMError) as e:
        fn()
    assert e.value.status == tm.TM_E_ARG and message in str(e.value), e.value
    torch.cuda.synchronize()
    for a, b in zip(before, tensors):
        assert torch.equal(a, b)


def shifted(shape, dtype, by=16):
    """Two tensors, the second one `by` bytes into the first."""
    n, more = 1, by // torch.empty((), dtype=dtype).element_size()
    for s in shape:
        n *= s
    flat = torch.randn((n + more,), device="cuda").to(dtype)
    return flat[:n].view(shape), flat[more:].view(shape)


B, n, E = 2, 24, 136
SHAPE = (B, n, E)


def norm_inputs(stream=F32, act=F32):
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda shape, dtype=F32: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    return dict(x=normal(SHAPE, stream), y=normal(SHAPE, act), gate=normal((B, 3, E)), post_weight=normal((E,)),
                pre_weight=normal((E,)), pre_bias=normal((E,)), scale=normal((B, 3, E)), shift=normal((B, 3, E)))


def test_forward_norm_outputs(tm):
    d = tm.make_block_norm_desc(B, E, "layer", "rms", "f32", "f32", 1e-6, 3, 10)
    p = norm_inputs()
    call = lambda **kw: tm.tm_block_norm_fwd(d, **{**p, **kw})  # noqa: E731
    r, h = call()
    refused(tm, "h overlaps", lambda: call(h=p["x"]), p["x"])
    refused(tm, "h overlaps", lambda: call(h=p["y"]), p["y"])
    refused(tm, "r overlaps y", lambda: call(r=p["y"]), p["y"])
    refused(tm, "r overlaps h", lambda: call(r=r, h=r), r)
    x, at = shifted(SHAPE, F32)
    refused(tm, "r overlaps x", lambda: call(x=x, r=at), x, at)
    refused(tm, "r overlaps x", lambda: call(x=at, r=x), x, at)
    a, b = shifted(SHAPE, F32, 4 * B * n * E - 16)  # the last 16 bytes of one are the first of the other
    refused(tm, "overlaps", lambda: call(r=a, h=b), a, b)
    for name in ("gate", "scale", "shift"):
        big = torch.zeros(SHAPE, device="cuda")
        small = big.view(-1)[-B * 3 * E:].view(B, 3, E)
        refused(tm, "h overlaps " + name, lambda: call(h=big, **{name: small}), big)
    for name in ("post_weight", "pre_weight", "pre_bias"):
        big = torch.zeros(SHAPE, device="cuda")
        refused(tm, "r overlaps " + name, lambda: call(r=big, **{name: big[1, 5]}), big)
    # r may be x itself, and tensors that only touch are apart
    x = p["x"].clone()
    flat = torch.empty((2 * B * n * E,), device="cuda")
    halves = flat[:B * n * E].view(SHAPE), flat[B * n * E:].view(SHAPE)
    for got in (call(x=x, r=x), call(r=halves[1], h=halves[0])):
        assert torch.equal(got[0], r) and torch.equal(got[1], h)


def test_backward_norm_outputs(tm):
    d = tm.make_block_norm_desc(B, E, "layer", "rms", "f32", "f32", 1e-6, 3, 10)
    p = norm_inputs()
    r, h = tm.tm_block_norm_fwd(d, **p)
    p.pop("x")
    dh, dr = torch.randn_like(h), torch.randn_like(r)
    call = lambda **kw: tm.tm_block_norm_bwd(d, **{**dict(p, r=r, dh=dh, dr=dr), **kw})  # noqa: E731
    want = call()

    def same(got):
        for a, b in zip(want, got):
            assert torch.equal(a, b)

    refused(tm, "dx overlaps r", lambda: call(dx=r), r)
    refused(tm, "dx overlaps dh", lambda: call(dx=dh), dh)
    refused(tm, "dx overlaps y", lambda: call(dx=p["y"]), p["y"])
    refused(tm, "dy overlaps r", lambda: call(dy=r), r)
    refused(tm, "dy overlaps dr", lambda: call(dy=dr), dr)
    out = torch.zeros(SHAPE, device="cuda")
    refused(tm, "overlaps", lambda: call(dx=out, dy=out), out)
    for of, into in (("dr", "dx"), ("y", "dy"), ("dh", "dy")):
        t, at = shifted(SHAPE, F32)
        refused(tm, f"{into} overlaps {of}", lambda: call(**{of: t, into: at}), t, at)
        refused(tm, f"{into} overlaps {of}", lambda: call(**{of: at, into: t}), t, at)
    for name in ("gate", "scale"):
        refused(tm, f"d{name} overlaps {name}", lambda: call(**{"d" + name: p[name]}), p[name])
    mod = torch.zeros((B, 3, E), device="cuda")
    refused(tm, "overlaps", lambda: call(dscale=mod, dshift=mod), mod)
    vec = torch.zeros((E,), device="cuda")
    refused(tm, "overlaps", lambda: call(dpre_weight=vec, dpre_bias=vec), vec)
    refused(tm, "overlaps", lambda: call(dpost_weight=p["pre_weight"]), p["pre_weight"])
    nbytes = tm.lib().tm_block_norm_bwd_workspace(d, n, 0)
    big = torch.zeros((max(nbytes // 4, B * n * E) + 64,), device="cuda")
    view = big[:B * n * E].view(SHAPE)
    refused(tm, "overlaps", lambda: call(workspace=big, dx=view), big)
    refused(tm, "overlaps", lambda: call(workspace=big, dr=view), big)
    refused(tm, "overlaps", lambda: call(workspace=big, gate=big[:B * 3 * E].view(B, 3, E)), big)
    refused(tm, "workspace is smaller", lambda: call(workspace=big[:nbytes // 4 - 1]), big)
    # the pairs that may be the same
    t = dr.clone()
    same(call(dr=t, dx=t))
    t = p["y"].clone()
    same(call(y=t, dy=t))
    t = dh.clone()
    same(call(dh=t, dy=t))


def test_linear_outputs(tm):
    K, N, rows = 20008, 776, 40  # long enough that tiles are split
    g = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda shape, dtype: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    d = tm.make_linear_desc(1, K, N, "none", "bf16", 4, 10)
    x, w, res = normal((1, rows, K), BF16), normal((N, K), BF16), normal((1, rows, N), BF16)
    bias, gate = normal((N,), F32), normal((1, 4, N), F32)
    call = lambda **kw: tm.tm_linear_fwd(d, **{**dict(x=x, weight=w, bias=bias, gate=gate, residual=res), **kw})  # noqa: E731
    pre = torch.zeros((1, rows, N), dtype=BF16, device="cuda")
    want = call(pre=pre)
    refused(tm, "o overlaps x", lambda: call(o=x.view(-1)[:rows * N].view(1, rows, N)), x)
    refused(tm, "o overlaps weight", lambda: call(o=w.view(-1)[:rows * N].view(1, rows, N)), w)
    refused(tm, "overlaps", lambda: call(o=pre, pre=pre), pre)
    refused(tm, "pre overlaps residual", lambda: call(pre=res), res)
    t, at = shifted((1, rows, N), BF16)
    refused(tm, "o overlaps residual", lambda: call(residual=t, o=at), t, at)
    refused(tm, "o overlaps residual", lambda: call(residual=at, o=t), t, at)
    big = torch.zeros((rows * N,), device="cuda")
    out = big.view(BF16)[:rows * N].view(1, rows, N)
    refused(tm, "o overlaps bias", lambda: call(o=out, bias=big[:N]), big)
    refused(tm, "o overlaps gate", lambda: call(o=out, gate=big[:4 * N].view(1, 4, N)), big)
    nbytes = tm.lib().tm_linear_fwd_workspace(d, rows)
    assert nbytes > 2 * rows * N
    ws = torch.zeros((nbytes // 2,), dtype=BF16, device="cuda")
    refused(tm, "overlaps", lambda: call(workspace=ws, o=ws[:rows * N].view(1, rows, N)), ws)
    refused(tm, "overlaps", lambda: call(workspace=ws, residual=ws[:rows * N].view(1, rows, N)), ws)
    refused(tm, "workspace is smaller", lambda: call(workspace=ws[:-1]), ws)
    t = res.clone()
    assert torch.equal(call(residual=t, o=t), want)

    dout = normal((1, rows, N), BF16)
    back = lambda **kw: tm.tm_linear_bwd(d, **{**dict(x=x, weight=w, dout=dout, gate=gate, pre=pre), **kw})  # noqa: E731
    refused(tm, "dx overlaps x", lambda: back(dx=x), x)
    refused(tm, "dweight overlaps weight", lambda: back(dweight=w), w)
    refused(tm, "overlaps", lambda: back(dx=w.view(-1)[:rows * K].view(1, rows, K)), w)
    refused(tm, "overlaps", lambda: back(dgate=gate), gate)
    refused(tm, "overlaps", lambda: back(dbias=gate.view(-1)[:N]), gate)
    big = torch.zeros((N * K,), dtype=BF16, device="cuda")
    refused(tm, "overlaps", lambda: back(dweight=big.view(N, K), dx=big[:rows * K].view(1, rows, K)), big)
    refused(tm, "overlaps", lambda: back(dweight=big.view(N, K), dout=big[-rows * N:].view(1, rows, N)), big)
    nbytes = tm.lib().tm_linear_bwd_workspace(d, rows, 0)
    ws = torch.zeros((max(nbytes // 2, rows * K),), dtype=BF16, device="cuda")
    refused(tm, "overlaps", lambda: back(workspace=ws, dx=ws[:rows * K].view(1, rows, K)), ws)
    refused(tm, "overlaps", lambda: back(workspace=ws, dout=ws[:rows * N].view(1, rows, N)), ws)
    refused(tm, "workspace is smaller", lambda: back(workspace=ws[:nbytes // 2 - 1]), ws)


def test_layouts_and_lengths(tm):
    d = tm.make_block_norm_desc(B, E, "layer", "rms", "f32", "f32", 1e-6, 3, 10)
    p = norm_inputs()
    call = lambda **kw: tm.tm_block_norm_fwd(d, **{**p, **kw})  # noqa: E731
    wide = torch.zeros((B, n, 2 * E), device="cuda")
    refused(tm, "not contiguous", lambda: call(x=wide[..., :E]))
    refused(tm, "not contiguous", lambda: call(h=wide[..., :E]), wide)
    refused(tm, "not contiguous", lambda: call(gate=torch.zeros((B, 6, E), device="cuda")[:, ::2]))
    flat = torch.zeros((B * n * E + 4,), device="cuda")
    refused(tm, "16-byte aligned", lambda: call(x=flat[1:-3].view(SHAPE)))
    refused(tm, "not on a GPU", lambda: call(y=p["y"].cpu()))
    # an address whose allocation ends too early
    lib = tm.lib()
    stream = torch.cuda.current_stream().cuda_stream
    addr = {k: t.data_ptr() for k, t in p.items()}
    big = tm.make_block_norm_desc(65535, 16384, "layer", "none", "f32", "f32")
    st = lib.tm_block_norm_fwd(big, 1000, 0, addr["x"], None, None, None, None, None, None, None, None, addr["y"], stream)
    assert st == tm.TM_E_ARG and "past the end" in tm.tm_last_error()
    dl = tm.make_linear_desc(1, 1 << 18, 1 << 18)
    st = lib.tm_linear_fwd(dl, 1, 0, addr["x"], addr["y"], None, None, None, None, addr["gate"], None, 0, stream)
    assert st == tm.TM_E_ARG and "past the end" in tm.tm_last_error()
