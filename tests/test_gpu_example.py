"""The example runs the new operators together as a program would."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("stream_8bit", os.path.join(ROOT, "examples", "stream_8bit.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (6, 2)])
def test_stream(example, heads, kv_heads):
    # rows of unit size: codes of K are off by 0.9% of a row's size, of V by as much, and with them
    # scores and output; the 16-bit path rounds keys and queries twice more: together below 5%
    differences, bytes8, bytes16 = example.stream(heads, kv_heads, (9, 11), 2, 3)
    assert len(differences) == 4 and max(differences) < 0.05
    # regions are whole blocks of 64 tokens here: 99 -> 128, 198 -> 256, and the 16-bit cache holds every head
    assert bytes8 < 0.7 * bytes16 * kv_heads / heads


def test_training_step(example):
    """dq and dk against autograd in fp32 over the same rotation and attention."""
    heads, grid, frames = 2, (5, 8), 7
    dq, dk, dv = example.train(heads, grid, frames)
    tm = example.tm
    D, T, n = 128, grid[0] * grid[1], frames * grid[0] * grid[1]
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, do = (example.draw((1, n, heads, D), g) for _ in range(4))
    q, k = example.normalise(q).float().requires_grad_(), example.normalise(k).float().requires_grad_()
    v = v.float().requires_grad_()
    rope = tm.make_rope_desc(D, frames, *grid, dtype="f32")
    table = tm.tm_rope3d_table(rope)
    chunk = torch.tensor([0 if f < 1 else 1 + (f - 1) // 3 for f in range(frames)], device="cuda").repeat_interleave(T)
    allowed = (chunk[None] == 0) | ((chunk[None] >= chunk[:, None] - 1) & (chunk[None] <= chunk[:, None]))
    p = torch.arange(n, device="cuda")
    at = torch.cat([table[:frames * 22].view(frames, 22, 2)[p // T],
                    table[frames * 22:][:grid[0] * 21].view(grid[0], 21, 2)[p % T // grid[1]],
                    table[frames * 22 + grid[0] * 21:].view(grid[1], 21, 2)[p % grid[1]]], 1)

    def turned(x):
        a, b = x[..., 0::2], x[..., 1::2]
        c, s = at[None, :, None, :, 0], at[None, :, None, :, 1]
        return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)

    rows = []
    for h in range(heads):
        x = turned(q)[0, :, h] @ turned(k)[0, :, h].T.contiguous() / D ** 0.5
        rows.append(torch.softmax(x.masked_fill(~allowed, float("-inf")), -1) @ v[0, :, h])
    torch.stack(rows, 1)[None].backward(do.float())
    for got, want in ((dq, q.grad), (dk, k.grad), (dv, v.grad)):
        # bf16 q, k, o, P and dS on the way: a few times 2^-8
        assert float((got.float() - want).norm() / want.norm()) < 0.02
