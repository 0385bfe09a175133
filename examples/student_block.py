"""A block of the student, forward and backward, on the library's operators.

The residual stream is in 32 bits, activations and weights in 16, the modulation is one row for each latent frame:

    modulation = linear(silu(linear(timestep)))                     a few rows
    h = (1 + scale1) norm(x) + shift1                               tm_block_norm
    q, k, v = linear(h), turned by position, attended to            tm_linear, tm_rope3d, tm_sparse_causal_attn
    r = x + gate1 linear(o);  h = (1 + scale2) norm(r) + shift2     tm_linear, tm_block_norm
    out = r + gate2 linear(gelu(linear(h)))                         tm_linear, twice

    python examples/student_block.py [--heads 8] [--grid 30 52] [--frames 7]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_03099_amd import tm  # noqa: E402

D, EPS = 128, 1e-6
PARTS = ("shift1", "scale1", "gate1", "shift2", "scale2", "gate2")


class Block:
    def __init__(self, heads, grid, frames, chunk_frames=3, hidden=4, seed=0):
        self.heads, self.frames, self.T = heads, frames, grid[0] * grid[1]
        E = self.E = heads * D
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k, size=1.0):
            return (torch.randn((n, k), generator=g, device="cuda") * size * k ** -0.5).bfloat16()

        self.weights = {"time": weight(E, E), "modulate": weight(6 * E, E, 0.3), "q": weight(E, E), "k": weight(E, E),
                        "v": weight(E, E), "o": weight(E, E), "up": weight(hidden * E, E),
                        "down": weight(E, hidden * E)}
        self.biases = {k: 0.1 * torch.randn(w.shape[0], generator=g, device="cuda") for k, w in self.weights.items()}
        by_frame = dict(groups=frames, group_tokens=self.T)
        self.norm = tm.make_block_norm_desc(1, E, "layer", "none", "bf16", "f32", EPS, **by_frame)
        act = {"time": "silu", "up": "gelu"}
        self.descs = {k: tm.make_linear_desc(1, w.shape[1], w.shape[0], act.get(k, "none"),
                                             "f32" if k in ("modulate", "down") else "bf16",
                                             **(by_frame if k == "down" else {})) for k, w in self.weights.items()}
        self.attn = tm.make_desc(1, heads, D, self.T, chunk_frames, 1, 1, "bf16")
        self.rope = tm.make_rope_desc(D, frames, *grid)
        self.table = tm.tm_rope3d_table(self.rope)

    def linear(self, name, x, **kw):
        return tm.tm_linear_fwd(self.descs[name], x, self.weights[name], self.biases[name], **kw)

    def linear_bwd(self, name, x, dout, **kw):
        g = tm.tm_linear_bwd(self.descs[name], x, self.weights[name], dout, **kw)
        self.grads[name], self.grads[name + " bias"] = g.dweight, g.dbias
        return g

    def pre(self, name, n):
        return torch.empty((1, n, self.weights[name].shape[0]), dtype=torch.bfloat16, device="cuda")

    def modulation(self, timesteps):
        """Six rows of E for each frame, from the frames' timestep vectors [1, frames, E]."""
        m = self.linear("modulate", self.linear("time", timesteps))
        return dict(zip(PARTS, (t.contiguous() for t in m.view(1, self.frames, 6, self.E).unbind(2))))

    def forward(self, x, mod):
        n = x.shape[1]
        heads = (1, n, self.heads, D)
        s = self.saved = {"x": x, "mod": mod}
        _, s["h1"] = tm.tm_block_norm_fwd(self.norm, x, scale=mod["scale1"], shift=mod["shift1"])
        q, k, v = (self.linear(name, s["h1"]).view(heads) for name in "qkv")
        s["q"], s["k"] = tm.tm_rope3d_fwd(self.rope, self.table, q, k)
        s["v"], s["lse"] = v, torch.empty((1, self.heads, n), dtype=torch.float32, device="cuda")
        s["a"] = tm.tm_sparse_causal_attn_fwd(self.attn, s["q"], -1, k=s["k"], v=v, n_frames=n // self.T, lse=s["lse"])
        s["y"] = self.linear("o", s["a"].view(1, n, self.E))
        s["r"], s["h2"] = tm.tm_block_norm_fwd(self.norm, x, s["y"], mod["gate1"], scale=mod["scale2"],
                                               shift=mod["shift2"])
        s["up"], s["down"] = self.pre("up", n), self.pre("down", n)
        s["u"] = self.linear("up", s["h2"], pre=s["up"])
        return self.linear("down", s["u"], gate=mod["gate2"], residual=s["r"], pre=s["down"])

    def backward(self, dout):
        """dx and the modulation's gradients; the weights' and biases' are left in ``grads``."""
        s, mod, n = self.saved, self.saved["mod"], dout.shape[1]
        self.grads, dmod = {}, {}
        g = self.linear_bwd("down", s["u"], dout, gate=mod["gate2"], pre=s["down"])
        dmod["gate2"] = g.dgate
        g = self.linear_bwd("up", s["h2"], g.dx, pre=s["up"])
        b = tm.tm_block_norm_bwd(self.norm, s["r"], g.dx, dout, s["y"], mod["gate1"], scale=mod["scale2"],
                                 shift=mod["shift2"])
        dmod["gate1"], dmod["scale2"], dmod["shift2"] = b.dgate, b.dscale, b.dshift
        da = self.linear_bwd("o", s["a"].view(1, n, self.E), b.dy).dx.view(s["a"].shape)
        dq, dk, dv = tm.tm_sparse_causal_attn_bwd(self.attn, n // self.T, s["q"], s["k"], s["v"], s["a"], s["lse"], da)
        dq, dk = tm.tm_rope3d_bwd(self.rope, self.table, dq, dk)
        dh = sum(self.linear_bwd(name, s["h1"], t.view(1, n, self.E)).dx.float() for name, t in zip("qkv", (dq, dk, dv)))
        b = tm.tm_block_norm_bwd(self.norm, s["x"], dh.bfloat16(), b.dx, scale=mod["scale1"], shift=mod["shift1"])
        dmod["scale1"], dmod["shift1"] = b.dscale, b.dshift
        return b.dx, dmod


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--heads", type=int, default=8)
    p.add_argument("--grid", type=int, nargs=2, default=(30, 52))
    p.add_argument("--frames", type=int, default=7)
    a = p.parse_args()
    block = Block(a.heads, tuple(a.grid), a.frames)
    g = torch.Generator(device="cuda").manual_seed(1)
    n = a.frames * block.T
    x = torch.randn((1, n, block.E), generator=g, device="cuda")
    mod = block.modulation(torch.randn((1, a.frames, block.E), generator=g, device="cuda").bfloat16())
    start, mid, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    for _ in range(3):
        start.record()
        out = block.forward(x, mod)
        mid.record()
        dx, dmod = block.backward(torch.ones_like(out))
        end.record()
    torch.cuda.synchronize()
    print(f"{n} tokens, {a.heads} heads: forward {start.elapsed_time(mid):.2f} ms, backward {mid.elapsed_time(end):.2f} ms")
    for name, t in {"out": out, "dx": dx, **dmod}.items():
        print(f"{name}: {tuple(t.shape)}, root mean square {float(t.float().square().mean().sqrt()):.3e}")


if __name__ == "__main__":
    main()
