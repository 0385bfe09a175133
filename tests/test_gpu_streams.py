"""Calls on another stream than the current one that allocate their outputs: the outputs take no memory that the
current stream still uses, and their own memory is not handed out again while the current stream reads them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


@pytest.fixture(scope="module")
def wait():
    """Keeps the current stream at work for some 200 ms."""
    times = []
    for cycles in (1000, 1_000_000):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        torch.cuda._sleep(cycles)
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))

    def run():
        torch.cuda._sleep(int(1_000_000 * 200 / max(times[1], 0.1)))

    return run


@pytest.fixture(scope="module")
def side(wait):
    """A stream whose work does not queue behind the current one's (streams share a few queues of the hardware)."""
    for _ in range(8):
        stream = torch.cuda.Stream()
        wait()
        done = torch.cuda.current_stream().record_event()
        with torch.cuda.stream(stream):
            torch.zeros((64,), device="cuda")
        stream.synchronize()
        beside = not done.query()
        torch.cuda.synchronize()
        if beside:
            return stream
    raise AssertionError("every stream waits for the current one")


def calls(tm, seed):
    """name -> call(stream), which returns a tuple of new tensors, and the inputs' bytes stay alive in the closure."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    n, E, N = 700, 1024, 1032
    x, y, mod, dr, dh = normal(1, n, E), normal(1, n, E, dtype=BF16), normal(1, 1, E), normal(1, n, E), normal(1, n, E, dtype=BF16)
    dn = tm.make_block_norm_desc(1, E, "layer", "rms", "bf16", "f32")
    xb, w, dout = normal(1, n, E, dtype=BF16), normal(N, E, dtype=BF16), normal(1, n, N, dtype=BF16)
    dl = tm.make_linear_desc(1, E, N)
    ws = torch.empty(tm.lib().tm_block_norm_bwd_workspace(dn, n, 0) + 16, dtype=torch.uint8, device="cuda")
    ws_l = torch.empty(tm.lib().tm_linear_bwd_workspace(dl, n, 0), dtype=torch.uint8, device="cuda")
    q, k, v = (normal(1, 7 * 64, 2, 64, dtype=BF16) for _ in range(3))
    da = tm.make_desc(1, 2, 64, 64, 2, 1, 1, "bf16")
    rope = tm.make_rope_desc(64, 7, 8, 8)
    table = tm.tm_rope3d_table(rope)
    o, lse = torch.empty_like(q), torch.empty((1, 2, 7 * 64), device="cuda")
    tm.tm_sparse_causal_attn_fwd(da, q, -1, k=k, v=v, n_frames=7, o=o, lse=lse)
    return {
        "norm": lambda s: tm.tm_block_norm_fwd(dn, x, y, mod, scale=mod, shift=mod, stream=s),
        "norm backward": lambda s: tuple(t for t in tm.tm_block_norm_bwd(dn, x, dh, dr, y, mod, scale=mod, shift=mod, workspace=ws,
                                                                         stream=s) if t is not None),
        "linear": lambda s: (tm.tm_linear_fwd(dl, xb, w, stream=s),),
        "linear backward": lambda s: tuple(t for t in tm.tm_linear_bwd(dl, xb, w, dout, workspace=ws_l, stream=s) if t is not None),
        "attention": lambda s: (tm.tm_sparse_causal_attn_fwd(da, q, -1, k=k, v=v, n_frames=7, stream=s),
                                tm.tm_sparse_causal_attn_fwd_f32out(da, q, -1, k=k, v=v, n_frames=7, stream=s)),
        "attention backward": lambda s: tm.tm_sparse_causal_attn_bwd(da, 7, q, k, v, o, lse, o, stream=s),
        "rope": lambda s: tm.tm_rope3d_fwd(rope, table, q, k, stream=s),
        "table": lambda s: (tm.tm_rope3d_table(rope, stream=s),),
    }


NAMES = ["norm", "norm backward", "linear", "linear backward", "attention", "attention backward", "rope", "table"]


@pytest.mark.parametrize("name", NAMES)
def test_new_outputs_take_nothing_that_the_current_stream_uses(tm, wait, side, name):
    call = calls(tm, 1)[name]
    side.wait_stream(torch.cuda.current_stream())
    want = call(side)
    torch.cuda.synchronize()
    held = [torch.full_like(t, 3) for t in want]
    torch.cuda.synchronize()
    wait()
    kept = [t.clone() for t in held]  # behind the wait
    del held                          # their memory is the current stream's to hand out
    done = torch.cuda.current_stream().record_event()
    got = call(side)
    side.synchronize()
    assert not done.query()  # else this shows nothing
    torch.cuda.synchronize()
    assert all(bool((t == 3).all()) for t in kept)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_outputs_dropped_while_the_current_stream_reads_them(tm, wait, side, name):
    first, second = calls(tm, 1)[name], calls(tm, 2)[name]
    side.wait_stream(torch.cuda.current_stream())
    got = first(side)
    torch.cuda.current_stream().wait_stream(side)
    want = [t.clone() for t in got]
    torch.cuda.synchronize()
    wait()
    kept = [t.clone() for t in got]
    done = torch.cuda.current_stream().record_event()
    del got
    for _ in range(3):
        second(side)
    side.synchronize()
    assert not done.query()
    torch.cuda.synchronize()
    for a, b in zip(want, kept):
        assert torch.equal(a, b)


def test_the_default_stream_from_another_one(tm):
    both = calls(tm, 1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    default = torch.cuda.default_stream()
    with torch.cuda.stream(side):
        for given in (default, default.cuda_stream):
            for name in ("norm", "linear"):
                got = both[name](given)
                default.synchronize()
                want = both[name](None)
                side.synchronize()
                for a, b in zip(want, got):
                    # (on its own stream the linear layer may share its sums out: another order of a 1024-term sum)
                    assert torch.equal(a, b) if name == "norm" else float((a.double() - b.double()).norm() / a.double().norm()) < 2 ** -8
