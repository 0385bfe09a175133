"""A streamed clip through the 8-bit cache, and a training step beside it.

One attention layer of the chunked student, with synthetic projections:

- serving: for every chunk, ``tm_qkv8_produce`` RMS-normalises the chunk's
  queries and keys, rotates them by their latent frame, row and column, and
  quantises keys and values into the 8-bit cache; ``tm_kv8_attn_fwd`` attends,
  for the whole chunk and for its last token's queries alone. The same stream through the
  16-bit cache says what the 8 bits cost;
- training: ``tm_rope3d_fwd``, the whole-sequence attention forward and backward,
  and ``tm_rope3d_bwd``.

    python examples/stream_8bit.py [--heads 40] [--grid 30 52] [--chunks 4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_03099_amd import tm  # noqa: E402

EPS = 1e-6


def draw(shape, g):
    return torch.randn(shape, generator=g, device="cuda").bfloat16()


def normalise(x):
    x = x.float()
    return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)).bfloat16()


def stream(heads, kv_heads, grid, chunk_frames, chunks, seed=0):
    """Streams a reference frame and ``chunks`` chunks; returns for each the relative difference of
    the 8-bit cache's attention to the 16-bit cache's, and the two caches' bytes."""
    D, T = 128, grid[0] * grid[1]
    desc = tm.make_desc(1, heads, D, T, chunk_frames, 1, 1, "bf16")
    rope = tm.make_rope_desc(D, 1 + chunk_frames * chunks, *grid)
    table = tm.tm_rope3d_table(rope)
    cache8, cache16 = tm.KV8Cache(desc, kv_heads), tm.KVCache(desc)
    g = torch.Generator(device="cuda").manual_seed(seed)
    first, differences = 0, []
    for t in range(chunks + 1):
        n = T if t == 0 else chunk_frames * T
        q, k, v = draw((1, n, heads, D), g), draw((1, n, kv_heads, D), g), draw((1, n, kv_heads, D), g)
        rotated = tm.tm_qkv8_produce(cache8, t, q, k, v, eps=EPS, rope=rope, table=table, first_token=first)
        o8 = tm.tm_kv8_attn_fwd(cache8, rotated, t)
        last = tm.tm_kv8_attn_fwd(cache8, rotated[:, -1:].contiguous(), t)  # one token's rows
        assert float((last.float() - o8[:, -1:].float()).norm() / last.float().norm()) < 0.01
        # the 16-bit cache: every head of queries has keys of its own there
        q16, k16 = tm.tm_rope3d_fwd(rope, table, normalise(q), normalise(k), first)
        share = heads // kv_heads
        tm.tm_kv_append(cache16, t, k16.repeat_interleave(share, 2), v.repeat_interleave(share, 2))
        o16 = tm.tm_sparse_causal_attn_fwd(desc, q16, t, cache=cache16)
        differences.append(float((o8.float() - o16.float()).norm() / o16.float().norm()))
        first += n
    return differences, cache8.pool.numel(), 2 * cache16.k_pool.numel() * 2


def train(heads, grid, frames, seed=1):
    """Gradients of a whole sequence's projections through rotation and attention."""
    D, T = 128, grid[0] * grid[1]
    desc = tm.make_desc(1, heads, D, T, 3, 1, 1, "bf16")
    rope = tm.make_rope_desc(D, frames, *grid)
    table = tm.tm_rope3d_table(rope)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = frames * T
    q, k, v, do = normalise(draw((1, n, heads, D), g)), normalise(draw((1, n, heads, D), g)), \
        draw((1, n, heads, D), g), draw((1, n, heads, D), g)
    lse = torch.empty((1, heads, n), dtype=torch.float32, device="cuda")
    qr, kr = tm.tm_rope3d_fwd(rope, table, q, k)
    o = tm.tm_sparse_causal_attn_fwd(desc, qr, -1, k=kr, v=v, n_frames=frames, lse=lse)
    dqr, dkr, dv = tm.tm_sparse_causal_attn_bwd(desc, frames, qr, kr, v, o, lse, do)
    dq, dk = tm.tm_rope3d_bwd(rope, table, dqr, dkr)
    return dq, dk, dv


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--heads", type=int, default=40)
    p.add_argument("--kv-heads", type=int, default=None)
    p.add_argument("--grid", type=int, nargs=2, default=(30, 52))
    p.add_argument("--chunk-frames", type=int, default=3)
    p.add_argument("--chunks", type=int, default=4)
    a = p.parse_args()
    differences, bytes8, bytes16 = stream(a.heads, a.kv_heads or a.heads, tuple(a.grid), a.chunk_frames, a.chunks)
    for t, d in enumerate(differences):
        print(f"chunk {t}: the 8-bit cache's attention differs from the 16-bit one's by {100 * d:.2f}%")
    print(f"cache: {bytes8 / 1e6:.1f} MB in 8 bits, {bytes16 / 1e6:.1f} MB in 16")
    for name, x in zip(("dq", "dk", "dv"), train(a.heads, tuple(a.grid), 1 + a.chunk_frames * 2)):
        print(f"{name}: {tuple(x.shape)}, root mean square {float(x.float().square().mean().sqrt()):.3e}")


if __name__ == "__main__":
    main()
