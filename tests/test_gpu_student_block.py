"""A block of the student on the operators together (examples/student_block.py): its output and every gradient
against autograd over the same block in fp32, token rows by the few-rows forms, and a captured block."""
import importlib.util
import os

import pytest
import torch

from block_reference import activate, normed

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("student_block", os.path.join(ROOT, "examples", "student_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def turned(x, table, frames, grid):
    """The rotation of tm_rope3d over its own table, in fp32 (pairs are neighbours)."""
    n, T = x.shape[1], grid[0] * grid[1]
    p = torch.arange(n, device="cuda")
    at = torch.cat([table[:frames * 22].view(frames, 22, 2)[p // T],
                    table[frames * 22:][:grid[0] * 21].view(grid[0], 21, 2)[p % T // grid[1]],
                    table[frames * 22 + grid[0] * 21:].view(grid[1], 21, 2)[p % grid[1]]], 1)
    a, b = x[..., 0::2], x[..., 1::2]
    c, s = at[None, :, None, :, 0], at[None, :, None, :, 1]
    return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)


def reference(block, grid, x, mod, weights, biases):
    """The block in fp32 (attention's products per head, two-dimensional)."""
    n, T, H, D = x.shape[1], block.T, block.heads, 128
    g = torch.arange(n, device="cuda") // T

    def linear(name, h):
        return h @ weights[name].t().contiguous() + biases[name]

    def modulated(r, i):
        return normed(r, "layer", 1e-6) * (1 + mod[f"scale{i}"][:, g]) + mod[f"shift{i}"][:, g]

    h = modulated(x, 1)
    q, k, v = (linear(name, h).view(1, n, H, D) for name in "qkv")
    q, k = (turned(t, block.table, block.frames, grid) for t in (q, k))
    chunk = torch.tensor([0 if f < 1 else 1 + (f - 1) // 3 for f in range(block.frames)], device="cuda").repeat_interleave(T)
    allowed = (chunk[None] == 0) | ((chunk[None] >= chunk[:, None] - 1) & (chunk[None] <= chunk[:, None]))
    rows = []
    for i in range(H):
        s = (q[0, :, i] @ k[0, :, i].t().contiguous() / D ** 0.5).masked_fill(~allowed, float("-inf"))
        rows.append(torch.softmax(s, -1) @ v[0, :, i])
    a = torch.stack(rows, 1).reshape(1, n, H * D)
    r = x + mod["gate1"][:, g] * linear("o", a)
    u = activate(linear("up", modulated(r, 2)), "gelu")
    return r + mod["gate2"][:, g] * linear("down", u)


def close(got, want, what, bound=0.03):
    """bf16 activations, gradients and P at about ten places on the way, each within 2^-8 / sqrt(3) of its norm at
    random: 0.7%; gradients of q and k take differences of nearly equal numbers and lose another two digits."""
    rel = float((got.float() - want).norm() / want.norm())
    print(f"  {what}: {rel:.4f} of its norm", flush=True)
    assert rel < bound, what


def test_block_forward_and_backward(example):
    heads, grid, frames = 2, (5, 9), 7
    block = example.Block(heads, grid, frames, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    n = frames * block.T
    x = torch.randn((1, n, block.E), generator=g, device="cuda")
    t = torch.randn((1, frames, block.E), generator=g, device="cuda").bfloat16()
    mod = block.modulation(t)
    w32 = {k: w.float().requires_grad_() for k, w in block.weights.items()}
    b32 = {k: b.clone().requires_grad_() for k, b in block.biases.items()}
    with torch.no_grad():
        tt = activate(t.float() @ w32["time"].t().contiguous() + b32["time"], "silu")
        m = (tt @ w32["modulate"].t().contiguous() + b32["modulate"]).view(1, frames, 6, block.E)
    for i, name in enumerate(example.PARTS):
        close(mod[name], m[:, :, i], name, 0.01)
    out = block.forward(x, mod)
    leaf = {k: v.clone().requires_grad_() for k, v in mod.items()}
    x32 = x.clone().requires_grad_()
    want = reference(block, grid, x32, leaf, w32, b32)
    close(out, want.detach(), "out", 0.01)
    dout = torch.randn(out.shape, generator=g, device="cuda")
    dx, dmod = block.backward(dout)
    want.backward(dout)
    close(dx, x32.grad, "dx")
    for k in example.PARTS:
        close(dmod[k], leaf[k].grad, "d" + k)
    for k in ("q", "k", "v", "o", "up", "down"):
        close(block.grads[k], w32[k].grad, "dW " + k)
        if k != "k":  # (a softmax does not see k's bias but through the rotation: next to nothing is left of it)
            close(block.grads[k + " bias"], b32[k].grad, "dbias " + k)


def test_block_captured(example):
    block = example.Block(2, (4, 6), 4, seed=5)
    n = 4 * block.T
    x = torch.randn((1, n, block.E), device="cuda")
    mod = block.modulation(torch.randn((1, 4, block.E), device="cuda").bfloat16())
    dout = torch.randn_like(x)
    block.forward(x, mod)
    block.backward(dout)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.forward(x, mod)
        dx, dmod = block.backward(dout)
    results = None
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        now = [t.clone() for t in (out, dx, *dmod.values())]
        if results is not None:
            assert all(torch.equal(a, b) for a, b in zip(now, results))
        results = now
        eager = block.forward(x, mod)
        edx, edmod = block.backward(dout)
        # (under capture the forward has no workspace and orders its sums otherwise: the last digit of bf16)
        for a, b in zip(results, (eager, edx, *edmod.values())):
            assert float((a - b).norm() / b.norm()) < 0.01
