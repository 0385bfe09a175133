"""The workloads that the norms around a block and the linear layers are timed on.

Each case is one call that a program makes through the binding
(``paper_2506_03099_amd.tm``), with ``own`` set, or the same computation in
elementary torch operations in 32 bits, without:

- ``norm``: a block's output added to the residual stream (normalised, scaled and
  gated on the way), and the stream normalised and modulated for the next block;
- ``norm_bwd``: the gradients of that;
- ``linear``: a matrix product with bias, activation, gate and residual;
- ``linear_bwd``: the gradients of that.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_GELU_C, _GELU_A = math.sqrt(2 / math.pi), 0.044715


# --------------------------------------------------------------------------- the cases


def _norm(name, direction, B, n, E, post, pre, stream, act, parts, group=0, groups=1, first=0):
    """`parts`: which of y (the block's output), gate, the weights and the modulation take part."""
    return {"name": name, "kind": "norm" if direction == "fwd" else "norm_bwd", "batch": B, "n": n, "width": E,
            "post": post, "pre": pre, "stream": stream, "dtype": act, "y": "y" in parts, "gate": "g" in parts,
            "post_weight": "p" in parts, "pre_weight": "w" in parts, "pre_bias": "b" in parts,
            "modulated": "m" in parts, "group": group, "groups": groups, "first": first}


def _linear(name, direction, B, n, K, N, act, out, parts, group=0, groups=1, first=0):
    """`parts`: which of bias, gate, residual and the kept pre-activation take part."""
    return {"name": name, "kind": "linear" if direction == "fwd" else "linear_bwd", "batch": B, "n": n, "in": K,
            "out": N, "act": act, "out_dtype": out, "bias": "b" in parts, "gate": "g" in parts,
            "residual": "r" in parts, "pre": "z" in parts, "group": group, "groups": groups, "first": first}


def listed():
    return [
        # one token's row before its first block of 40 heads of 128: launch latency
        _norm("norm_token", "fwd", 1, 1, 5120, "none", "layer", "f32", "bf16", "m"),
        # a 480x832 chunk between two blocks: gated into a 32-bit stream, normalised, modulated by frame
        _norm("norm_480p_chunk", "fwd", 1, 4680, 5120, "none", "layer", "f32", "bf16", "ygm", 1560, 7, 4680),
        # two 720x720 streams of 8 heads, norms on both sides of the block, a 16-bit stream, no modulation
        _norm("norm_720sq_both", "fwd", 2, 6075, 1024, "rms", "rms", "bf16", "bf16", "ypw"),
        # a training step on the 21-frame 480p clip: every frame has its own modulation
        _norm("norm_480p_clip_bwd", "bwd", 1, 32760, 5120, "none", "layer", "f32", "bf16", "ygm", 1560, 21),
        # three short ragged streams, all parts, activations in 32 bits
        _norm("norm_ragged_bwd", "bwd", 3, 333, 1000, "rms", "layer", "f32", "f32", "ygpwbm", 100, 5, 77),
        # one row through a projection with an activation, as the vectors that modulate are made
        _linear("linear_token", "fwd", 1, 1, 5120, 20480, "silu", "f32", "b"),
        # a few hundred ragged rows of a small layer, in a training step (the pre-activation is kept)
        _linear("linear_ragged", "fwd", 3, 111, 1000, 1352, "gelu", "bf16", "bz"),
        # the 480p chunk through the first matrix of its feed-forward layer
        _linear("linear_480p_up", "fwd", 1, 4680, 5120, 20480, "gelu", "bf16", "b"),
        # and the second, gated by frame into the 32-bit stream
        _linear("linear_480p_down", "fwd", 1, 4680, 20480, 5120, "none", "f32", "bgr", 1560, 7, 4680),
        # a hundred rows through a square projection: between the rows' and the matrix' bound
        _linear("linear_rows_130", "fwd", 2, 65, 5120, 5120, "none", "bf16", "br"),
        # a training step at 256 tokens a frame on 8 heads: the feed-forward layer's first matrix
        _linear("linear_256_bwd", "bwd", 1, 5376, 1024, 4096, "gelu", "bf16", "bz"),
        # the output projection of the 480p clip, gated by frame
        _linear("linear_480p_clip_bwd", "bwd", 1, 32760, 5120, 5120, "none", "f32", "bgz", 1560, 21),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: both operators in both directions, one row to a 21-frame clip, widths from 64 to 20480 in
    steps of 8, one to three streams, modulation of every token, of frames or of the whole run."""
    largest = listed()[-1]
    most = work(largest)
    while True:
        B, n = rng.choice([1, 1, 2, 3]), _log_int(rng, 1, 32760)
        first = rng.choice([0, rng.randint(0, 5000)])
        group = rng.choice([0, 0, _log_int(rng, 64, 3600), _log_int(rng, 64, 3600)])
        if n <= 512 and rng.random() < 0.15:
            group = 1
        groups = (first + n - 1) // group + 1 + rng.randint(0, 2) if group else 1
        direction = rng.choice(["fwd", "fwd", "bwd"])
        if rng.random() < 0.45:
            E = 8 * _log_int(rng, 8, 2048)
            post, pre = rng.choice(["none", "none", "layer", "rms"]), rng.choice(["layer", "layer", "rms", "none"])
            parts = "".join(p for p in "gpwbm" if rng.random() < 0.5)
            parts += "y" if post != "none" or pre == "none" or rng.random() < 0.7 else ""
            if "y" not in parts:
                parts = parts.replace("g", "").replace("p", "")
            if pre == "none":
                parts = "".join(p for p in parts if p not in "wbm")
            c = _norm("", direction, B, n, E, post, pre, rng.choice(["f32", "bf16"]),
                      rng.choice(["bf16", "bf16", "f32"]), parts, group, groups, first)
        else:
            K, N = 8 * _log_int(rng, 8, 2560), 8 * _log_int(rng, 8, 2560)
            act = rng.choice(["none", "none", "gelu", "silu"])
            parts = "".join(p for p in "bgr" if rng.random() < 0.5)
            if direction == "bwd":
                parts = parts.replace("r", "") + ("z" if act != "none" or "g" in parts else "")
            elif rng.random() < 0.3:
                parts += "z"
            c = _linear("", direction, B, n, K, N, act, rng.choice(["bf16", "bf16", "f32"]), parts, group, groups,
                        first)
        del c["name"]
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= 2.5e9:
            return c


# --------------------------------------------------------------------------- a pass's work


def _size(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    B, n = case["batch"], case["n"]
    rows = B * n
    if case["kind"] in ("norm", "norm_bwd"):
        E = case["width"]
        s, a, has_pre = _size(case["stream"]), _size(case["dtype"]), case["pre"] != "none"
        vectors = 4 * E * (B * case["groups"] * (case["gate"] + 2 * case["modulated"])
                           + case["post_weight"] + case["pre_weight"] + case["pre_bias"])
        if case["kind"] == "norm":
            # x and y in, r (where there is a y) and h out
            row = s + (a + s if case["y"] else 0) + (a if has_pre else 0)
            return {"bytes": rows * E * row + vectors, "flops": 12 * rows * E}
        # r, dr, y and dh in, dx and dy out; the vectors and their gradients
        row = 3 * s + (2 * a if case["y"] else 0) + (a if has_pre else 0)
        return {"bytes": rows * E * row + 2 * vectors, "flops": 24 * rows * E}
    K, N, o = case["in"], case["out"], _size(case["out_dtype"])
    gates = 4 * B * case["groups"] * N * case["gate"]
    if case["kind"] == "linear":
        total = 2 * (rows * K + N * K) + 4 * N * case["bias"] + gates
        total += rows * N * (o * (1 + case["residual"]) + 2 * case["pre"])
        return {"bytes": total, "flops": 2 * rows * N * K}
    # x, W, the output's gradient and the pre-activation in; dx, dW and the vectors' gradients out
    total = 2 * (2 * rows * K + 2 * N * K) + rows * N * (o + 2 * case["pre"]) + 4 * N * case["bias"] + 2 * gates
    return {"bytes": total, "flops": 4 * rows * N * K}


# --------------------------------------------------------------------------- inputs


def _normal(g, shape, dtype, size=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * size).to(dtype)


def _inputs(case, seed):
    """The tensors of a case, on the GPU: the same for both sides, and for exact()."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, n, G = case["batch"], case["n"], case["groups"]
    f32 = torch.float32
    s = {"case": case}
    if case["kind"] in ("norm", "norm_bwd"):
        E, st, dt = case["width"], _DT[case["stream"]], _DT[case["dtype"]]
        # some channels of a residual stream are far larger than the others
        size = torch.exp(0.7 * torch.randn(E, generator=g, device="cuda"))
        stream = (torch.randn((B, n, E), generator=g, device="cuda") * size).to(st)
        s["y"] = _normal(g, (B, n, E), dt) if case["y"] else None
        s["gate"] = _normal(g, (B, G, E), f32, 0.5) if case["gate"] else None
        s["post_weight"] = 1 + _normal(g, (E,), f32, 0.2) if case["post_weight"] else None
        s["pre_weight"] = 1 + _normal(g, (E,), f32, 0.2) if case["pre_weight"] else None
        s["pre_bias"] = _normal(g, (E,), f32, 0.1) if case["pre_bias"] else None
        s["scale"] = _normal(g, (B, G, E), f32, 0.3) if case["modulated"] else None
        s["shift"] = _normal(g, (B, G, E), f32, 0.3) if case["modulated"] else None
        if case["kind"] == "norm":
            s["x"] = stream
        else:
            s["r"] = stream
            s["dh"] = _normal(g, (B, n, E), dt, 1e-2) if case["pre"] != "none" else None
            s["dr"] = _normal(g, (B, n, E), st, 1e-2)
        return s
    K, N, od = case["in"], case["out"], _DT[case["out_dtype"]]
    s["x"] = _normal(g, (B, n, K), torch.bfloat16)
    s["weight"] = _normal(g, (N, K), torch.bfloat16, K ** -0.5)
    s["bias"] = _normal(g, (N,), f32, 0.1) if case["bias"] else None
    s["gate"] = _normal(g, (B, G, N), f32, 0.5) if case["gate"] else None
    if case["kind"] == "linear":
        s["residual"] = _normal(g, (B, n, N), od, 2.0) if case["residual"] else None
    else:
        s["pre"] = _normal(g, (B, n, N), torch.bfloat16) if case["pre"] else None
        s["dout"] = _normal(g, (B, n, N), od, 1e-2)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2506_03099_amd import tm
        s["tm"] = tm
        if case["kind"] in ("norm", "norm_bwd"):
            s["desc"] = tm.make_block_norm_desc(case["batch"], case["width"], case["pre"], case["post"],
                                                case["dtype"], case["stream"], EPS, case["groups"], case["group"])
        else:
            s["desc"] = tm.make_linear_desc(case["batch"], case["in"], case["out"], case["act"], case["out_dtype"],
                                            case["groups"], case["group"])
    return s


# --------------------------------------------------------------------------- the plain forms


def _groups(case):
    """The modulation row of each token."""
    i = case["first"] + torch.arange(case["n"], device="cuda")
    return i // case["group"] if case["group"] else torch.zeros_like(i)


def _of_tokens(case, t):
    """A modulation [B, G, E] as each token's row [B, n, E] (or [B, 1, E])."""
    return t if case["groups"] == 1 else t[:, _groups(case)]


def _of_groups(case, rows):
    """Rows [B, n, E] summed over the tokens of each group: [B, G, E]."""
    if case["groups"] == 1:
        return rows.sum(1, keepdim=True)
    out = torch.zeros((rows.shape[0], case["groups"], rows.shape[2]), device="cuda", dtype=rows.dtype)
    at, first, group = 0, case["first"], case["group"]
    while at < case["n"]:
        g = (first + at) // group
        end = min((g + 1) * group - first, case["n"])
        out[:, g] = rows[:, at:end].sum(1)
        at = end
    return out


def _normed(x, kind):
    """Normalised rows, and what they were multiplied by."""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    by = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * by, by


def _normed_bwd(t, normed, by, kind):
    if kind == "none":
        return t
    t = t - normed * (t * normed).mean(-1, keepdim=True) - (t.mean(-1, keepdim=True) if kind == "layer" else 0)
    return t * by


def _plain_norm(s):
    case = s["case"]
    r = s["x"].float()
    out = []
    if case["y"]:
        z, _ = _normed(s["y"].float(), case["post"])
        if case["post_weight"]:
            z = z * s["post_weight"]
        if case["gate"]:
            z = z * _of_tokens(case, s["gate"])
        r = r + z
        out.append(r.to(s["x"].dtype))
    if case["pre"] != "none":
        m, _ = _normed(r, case["pre"])
        if case["pre_weight"]:
            m = m * s["pre_weight"]
        if case["pre_bias"]:
            m = m + s["pre_bias"]
        if case["modulated"]:
            m = m * (1 + _of_tokens(case, s["scale"])) + _of_tokens(case, s["shift"])
        out.append(m.to(_DT[case["dtype"]]))
    return tuple(out)


def _plain_norm_bwd(s):
    case = s["case"]
    a = s["dr"].float()
    out = {}
    if case["pre"] != "none":
        n, by = _normed(s["r"].float(), case["pre"])
        dh = s["dh"].float()
        t = dh
        if case["modulated"]:
            m = n * s["pre_weight"] if case["pre_weight"] else n
            m = m + s["pre_bias"] if case["pre_bias"] else m
            out["dscale"], out["dshift"] = _of_groups(case, dh * m), _of_groups(case, dh)
            t = t * (1 + _of_tokens(case, s["scale"]))
        if case["pre_bias"]:
            out["dpre_bias"] = t.sum((0, 1))
        if case["pre_weight"]:
            out["dpre_weight"] = (t * n).sum((0, 1))
            t = t * s["pre_weight"]
        a = a + _normed_bwd(t, n, by, case["pre"])
    out["dx"] = a.to(s["r"].dtype)
    if case["y"]:
        v, by = _normed(s["y"].float(), case["post"])
        u = a
        if case["gate"]:
            z = v * s["post_weight"] if case["post_weight"] else v
            out["dgate"] = _of_groups(case, u * z)
            u = u * _of_tokens(case, s["gate"])
        if case["post_weight"]:
            out["dpost_weight"] = (u * v).sum((0, 1))
            u = u * s["post_weight"]
        out["dy"] = _normed_bwd(u, v, by, case["post"]).to(s["y"].dtype)
    return out


def _act(z, act):
    if act == "gelu":
        return z / (1 + torch.exp(-2 * _GELU_C * (z + _GELU_A * z * z * z)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_slope(z, act):
    if act == "gelu":
        s = 1 / (1 + torch.exp(-2 * _GELU_C * (z + _GELU_A * z * z * z)))
        return s + z * s * (1 - s) * (2 * _GELU_C * (1 + 3 * _GELU_A * z * z))
    s = 1 / (1 + torch.exp(-z))
    return s + z * s * (1 - s)


def _plain_linear(s):
    case = s["case"]
    z = s["x"].float() @ s["weight"].float().t()
    if case["bias"]:
        z = z + s["bias"]
    u = _act(z, case["act"])
    if case["gate"]:
        u = u * _of_tokens(case, s["gate"])
    if case["residual"]:
        u = u + s["residual"].float()
    o = u.to(_DT[case["out_dtype"]])
    return (o, z.to(torch.bfloat16)) if case["pre"] else o


def _plain_linear_bwd(s):
    case = s["case"]
    out = {}
    dz = s["dout"].float()
    if case["gate"]:
        out["dgate"] = _of_groups(case, dz * _act(s["pre"].float(), case["act"]))
        dz = dz * _of_tokens(case, s["gate"])
    if case["act"] != "none":
        dz = dz * _act_slope(s["pre"].float(), case["act"])
    if case["bias"]:
        out["dbias"] = dz.sum((0, 1))
    flat = dz.view(-1, case["out"])
    out["dx"] = (dz @ s["weight"].float()).to(torch.bfloat16)
    out["dweight"] = (flat.t() @ s["x"].float().view(-1, case["in"])).to(torch.bfloat16)
    return out


# --------------------------------------------------------------------------- a pass


def run(state):
    case, s = state["case"], state
    kind = case["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "linear": _plain_linear,
                "linear_bwd": _plain_linear_bwd}[kind](state)
    tm, first = s["tm"], case["first"]
    if kind == "norm":
        r, h = tm.tm_block_norm_fwd(s["desc"], s["x"], s["y"], s["gate"], s["post_weight"], s["pre_weight"],
                                    s["pre_bias"], s["scale"], s["shift"], first)
        return tuple(t for t, there in ((r, case["y"]), (h, case["pre"] != "none")) if there)
    if kind == "norm_bwd":
        g = tm.tm_block_norm_bwd(s["desc"], s["r"], s["dh"], s["dr"], s["y"], s["gate"], s["post_weight"],
                                 s["pre_weight"], s["pre_bias"], s["scale"], s["shift"], first)
        return {k: v for k, v in g._asdict().items() if v is not None}
    if kind == "linear":
        if not case["pre"]:
            return tm.tm_linear_fwd(s["desc"], s["x"], s["weight"], s["bias"], s["gate"], s["residual"], first)
        pre = torch.empty((case["batch"], case["n"], case["out"]), dtype=torch.bfloat16, device="cuda")
        return tm.tm_linear_fwd(s["desc"], s["x"], s["weight"], s["bias"], s["gate"], s["residual"], first,
                                pre=pre), pre
    g = tm.tm_linear_bwd(s["desc"], s["x"], s["weight"], s["dout"], s["gate"], s["pre"], first,
                         dbias=None if case["bias"] else False)
    return {k: v for k, v in g._asdict().items() if v is not None}


# --------------------------------------------------------------------------- the definitions in 64 bits


def _exact_mod(case, t):
    """[B, n, E] rows of a modulation [B, G, E], ones for none, token by token's group."""
    index = [(case["first"] + i) // case["group"] if case["group"] else 0 for i in range(case["n"])]
    return t.double()[:, torch.tensor(index, device="cuda")]


def _exact_sums(case, rows):
    index = [(case["first"] + i) // case["group"] if case["group"] else 0 for i in range(case["n"])]
    out = torch.zeros((rows.shape[0], case["groups"], rows.shape[2]), dtype=torch.float64, device="cuda")
    return out.index_add_(1, torch.tensor(index, device="cuda"), rows)


def _exact_norm(x, kind):
    if kind == "none":
        return x, torch.ones_like(x[..., :1])
    mean = x.sum(-1, keepdim=True) / x.shape[-1] if kind == "layer" else torch.zeros_like(x[..., :1])
    var = ((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1]
    return (x - mean) * torch.rsqrt(var + EPS), torch.rsqrt(var + EPS)


def _exact_norm_slope(grad, x, kind):
    """grad times the Jacobian of the norm at x."""
    if kind == "none":
        return grad
    E = x.shape[-1]
    n, inv = _exact_norm(x, kind)
    along = (grad * n).sum(-1, keepdim=True) / E
    flat = grad.sum(-1, keepdim=True) / E if kind == "layer" else 0.0
    return inv * (grad - flat - along * n)


def _vector(t):
    return 1.0 if t is None else t.double()


def exact(case, seed):
    s = _inputs(case, seed)
    B, n = case["batch"], case["n"]
    if case["kind"] == "norm":
        r = s["x"].double()
        out = []
        if case["y"]:
            z = _exact_norm(s["y"].double(), case["post"])[0] * _vector(s["post_weight"])
            r = r + (_exact_mod(case, s["gate"]) * z if case["gate"] else z)
            out.append(r)
        if case["pre"] != "none":
            h = _exact_norm(r, case["pre"])[0] * _vector(s["pre_weight"])
            h = h + s["pre_bias"].double() if case["pre_bias"] else h
            if case["modulated"]:
                h = h + h * _exact_mod(case, s["scale"]) + _exact_mod(case, s["shift"])
            out.append(h)
        return tuple(out)
    if case["kind"] == "norm_bwd":
        out = {}
        a = s["dr"].double()
        if case["pre"] != "none":
            r, dh = s["r"].double(), s["dh"].double()
            unit = _exact_norm(r, case["pre"])[0]
            dm = dh + dh * _exact_mod(case, s["scale"]) if case["modulated"] else dh
            if case["modulated"]:
                affine = unit * _vector(s["pre_weight"])
                affine = affine + s["pre_bias"].double() if case["pre_bias"] else affine
                out["dscale"], out["dshift"] = _exact_sums(case, dh * affine), _exact_sums(case, dh)
                del affine
            if case["pre_bias"]:
                out["dpre_bias"] = dm.reshape(B * n, -1).sum(0)
            if case["pre_weight"]:
                out["dpre_weight"] = (dm * unit).reshape(B * n, -1).sum(0)
            del unit
            a = a + _exact_norm_slope(dm * _vector(s["pre_weight"]), r, case["pre"])
        out["dx"] = a
        if case["y"]:
            y = s["y"].double()
            unit = _exact_norm(y, case["post"])[0]
            dz = a * _exact_mod(case, s["gate"]) if case["gate"] else a
            if case["gate"]:
                out["dgate"] = _exact_sums(case, a * unit * _vector(s["post_weight"]))
            if case["post_weight"]:
                out["dpost_weight"] = (dz * unit).reshape(B * n, -1).sum(0)
            del unit
            out["dy"] = _exact_norm_slope(dz * _vector(s["post_weight"]), y, case["post"])
        return out
    x, w = s["x"].double().view(B * n, -1), s["weight"].double()

    def sigmoid(v):
        return torch.special.expit(v)

    def act(z):
        if case["act"] == "silu":
            return z * sigmoid(z)
        if case["act"] == "gelu":
            return z * 0.5 * (1 + torch.tanh(_GELU_C * (z + _GELU_A * z ** 3)))
        return z

    if case["kind"] == "linear":
        z = (x @ w.t()).view(B, n, -1)
        if case["bias"]:
            z = z + s["bias"].double()
        o = act(z)
        if case["gate"]:
            o = o * _exact_mod(case, s["gate"])
        if case["residual"]:
            o = o + s["residual"].double()
        return (o, z) if case["pre"] else o
    out = {}
    dz = s["dout"].double()
    if case["gate"]:
        out["dgate"] = _exact_sums(case, dz * act(s["pre"].double()))
        dz = dz * _exact_mod(case, s["gate"])
    if case["act"] == "silu":
        z = s["pre"].double()
        dz = dz * (sigmoid(z) * (1 + z * (1 - sigmoid(z))))
    elif case["act"] == "gelu":
        z = s["pre"].double()
        t = torch.tanh(_GELU_C * (z + _GELU_A * z ** 3))
        dz = dz * (0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _GELU_C * (1 + 3 * _GELU_A * z ** 2))
    dz = dz.reshape(B * n, -1)
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    out["dx"] = (dz @ w).view(B, n, -1)
    out["dweight"] = dz.t() @ x
    return out
