"""The workloads that the rotary positions, the 8-bit cache and the attention
over that cache are timed on.

Each case is one call sequence that a program makes through the binding
(``paper_2506_03099_amd.tm``), with ``own`` set, or the same computation in
elementary torch operations in 32 bits, without:

- ``rope``: queries and keys rotated by their (frame, row, column) positions,
  forward or backward;
- ``write_read``: a chunk's keys and values into the 8-bit cache, and the values
  that the cache now stands for read back;
- ``produce``: the chunk's queries and keys RMS-normalised and rotated on the
  way into the 8-bit cache, the rotated queries and the cached values returned;
- ``attend``: query rows of the latest chunk over the 8-bit cache.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
THETA = 10000.0
BLOCK = 64           # tokens that share a scale
LEAST = 2.0 ** -60   # a block's scale is that of at least this magnitude
_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# --------------------------------------------------------------------------- the cases


def _rope(name, direction, dtype, B, heads, kv_heads, D, grid_h, grid_w, first, n, halves=False, pairs=None):
    return {"name": name, "kind": "rope", "direction": direction, "dtype": dtype, "batch": B, "heads": heads,
            "kv_heads": kv_heads, "head_dim": D, "grid_h": grid_h, "grid_w": grid_w, "first": first, "n": n,
            "halves": halves, "pairs_t": (pairs or _pairs(D))[0], "pairs_h": (pairs or _pairs(D))[1],
            "pairs_w": (pairs or _pairs(D))[2]}


def _pairs(D):
    third = D // 2 // 3
    return D // 2 - 2 * third, third, third


def _write(name, B, kv_heads, D, n, out="bf16"):
    return {"name": name, "kind": "write_read", "batch": B, "kv_heads": kv_heads, "head_dim": D, "n": n, "out": out}


def _produce(name, B, heads, kv_heads, D, grid_h, grid_w, first, n, gains, rotate=True, halves=False):
    p = _pairs(D)
    return {"name": name, "kind": "produce", "batch": B, "heads": heads, "kv_heads": kv_heads, "head_dim": D,
            "grid_h": grid_h, "grid_w": grid_w, "first": first, "n": n, "gains": gains, "rotate": rotate,
            "halves": halves, "pairs_t": p[0], "pairs_h": p[1], "pairs_w": p[2]}


def _attend(name, B, heads, kv_heads, D, ref, chunk, window, chunks, last, n_q, lse):
    """c_0 of `ref` tokens, then `chunks` chunks of `chunk` tokens, the latest of `last`; the cache holds
    c_0 and the last window + 1 of them."""
    return {"name": name, "kind": "attend", "batch": B, "heads": heads, "kv_heads": kv_heads, "head_dim": D,
            "ref": ref, "chunk": chunk, "window": window, "chunks": chunks, "last": last, "n_q": n_q, "lse": lse}


def listed():
    return [
        # one token's queries and keys, as a decoder that goes on token by token rotates them: launch latency
        _rope("rope_one_token", "fwd", "bf16", 1, 40, 40, 128, 30, 52, 9000, 1),
        # a training step on the 21-frame 480x832 clip: the gradients of rotated queries and keys
        _rope("rope_480p_clip_bwd", "bwd", "bf16", 1, 40, 40, 128, 30, 52, 0, 32760),
        # a 720x720 frame run (45x45 tokens, starting inside a frame) in 32 bits, pairs as halves, shared key heads
        _rope("rope_720sq_f32", "fwd", "f32", 2, 8, 2, 64, 45, 45, 1000, 6075, True, (8, 10, 10)),
        # a 480p chunk into the 8-bit cache, and back
        _write("write_read_480p", 1, 40, 128, 4680),
        # three streams of a short ragged chunk, two key heads
        _write("write_read_ragged", 3, 2, 64, 333, "f32"),
        # the steady state of the 480p stream: normalise, rotate and quantise a chunk
        _produce("produce_480p", 1, 40, 40, 128, 30, 52, 6240, 4680, True),
        # a 720x720 chunk with shared key heads, no gains
        _produce("produce_720sq_shared", 1, 40, 8, 128, 45, 45, 8100, 6075, False),
        # one query row over a long prompt, shared key heads, four streams: bound by the cache's bytes
        _attend("attend_token_long", 4, 40, 8, 128, 65536, 64, 3, 5, 17, 1, True),
        # one query row over the 480p cache, a head of keys for each head of queries
        _attend("attend_token_480p", 1, 40, 40, 128, 1560, 4680, 1, 2, 4680, 1, False),
        # 17 query rows over a small ragged cache at the narrow head width
        _attend("attend_rows_small", 2, 8, 8, 64, 130, 257, 1, 3, 100, 17, True),
        # a 720x720 chunk on 8 heads: nothing divides evenly
        _attend("attend_720sq_8heads", 1, 8, 8, 128, 2025, 6075, 1, 3, 6075, 6075, True),
        # the 480p chunk: 4680 queries, 10920 keys, 40 heads
        _attend("attend_480p_chunk", 1, 40, 40, 128, 1560, 4680, 1, 2, 4680, 4680, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every kind, one token to a 21-frame clip, frames of 16 to 3600 tokens, 1 to 40 heads, keys
    shared by 1 to 8 heads, both head widths, prompts up to 100000 tokens, ragged last chunks."""
    while True:
        kind = rng.choice(["rope", "rope", "write_read", "produce", "attend", "attend", "attend"])
        B = rng.choice([1, 1, 2, 3])
        kv = rng.choice([1, 2, 3, 5, 8, 10, 20, 40])
        heads = kv * rng.choice([g for g in (1, 1, 2, 3, 4, 5, 8) if kv * g <= 40])
        D = rng.choice([128, 128, 64])
        gh, gw = rng.randint(4, 45), rng.randint(4, 80)
        first = rng.randint(0, 20 * gh * gw)
        n = _log_int(rng, 1, 32760)
        if kind == "rope":
            a, b = rng.randint(0, D // 2), rng.randint(0, D // 2)
            pairs = rng.choice([_pairs(D), _pairs(D), (min(a, b), abs(a - b), (D // 2 - max(a, b)) // 2)])
            c = _rope("", rng.choice(["fwd", "bwd"]), rng.choice(["bf16", "bf16", "f32"]), B, heads, kv, D, gh, gw,
                      first, n, rng.random() < 0.4, pairs)
        elif kind == "write_read":
            c = _write("", B, kv, D, min(n, 12000), rng.choice(["bf16", "f32"]))
        elif kind == "produce":
            c = _produce("", B, heads, kv, D, gh, gw, first, min(n, 12000), rng.random() < 0.5, rng.random() < 0.8,
                         rng.random() < 0.4)
        else:
            ref, chunk = _log_int(rng, 1, 100000), _log_int(rng, 1, 8000)
            last = chunk if rng.random() < 0.5 else rng.randint(1, chunk)
            c = _attend("", B, heads, kv, D, ref, chunk, rng.choice([0, 1, 1, 2, 3]), rng.randint(0, 4), last,
                        rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 1, last)]), rng.random() < 0.5)
        del c["name"]
        w = work(c)
        scores = 0
        if kind == "attend":
            scores = B * heads * c["n_q"] * _keys(c)
            if c["n_q"] > last or (_keys(c) + (c["window"] + 1) * chunk) * B * kv * D > 2e8:
                continue
        if w["flops"] <= 1.0e12 and w["bytes"] <= 1.3e9 and scores <= 2.0e9:
            return c


def _lengths(case):
    """Tokens of every chunk that the case appends, c_0's first, and the index of the first chunk after c_0 that
    the latest one still sees."""
    n = [case["ref"]] + [case["chunk"]] * case["chunks"]
    if case["chunks"]:
        n[-1] = case["last"]
    return n, max(1, case["chunks"] - case["window"])


def _keys(case):
    n, lo = _lengths(case)
    return n[0] + sum(n[lo:])


# --------------------------------------------------------------------------- a pass's work


def work(case):
    B, D = case["batch"], case["head_dim"]
    kv = case["kv_heads"]
    if case["kind"] == "rope":
        elems = B * case["n"] * (case["heads"] + kv) * D
        return {"bytes": elems * 2 * (4 if case["dtype"] == "f32" else 2) + 8 * _table_rows(case),
                "flops": 3 * elems}
    if case["kind"] in ("write_read", "produce"):
        elems = 2 * B * case["n"] * kv * D
        scales = 4 * 2 * B * kv * -(-case["n"] // BLOCK)
        # values in, codes out, codes in, values out, and the scales out and in
        total = elems * (2 + 1 + 1 + (4 if case.get("out") == "f32" else 2)) + 2 * scales
        flops = 5 * elems
        if case["kind"] == "produce":
            total += 2 * 2 * B * case["n"] * case["heads"] * D
            flops += 8 * B * case["n"] * (case["heads"] + kv) * D
        return {"bytes": total, "flops": flops}
    rows = B * case["heads"] * case["n_q"]
    keys = _keys(case)
    total = rows * D * 4 + (rows * 4 if case["lse"] else 0) + B * kv * 2 * (keys * D + 4 * -(-keys // BLOCK))
    return {"bytes": total, "flops": 4 * D * rows * keys}


def _frames(case):
    return (case["first"] + case["n"] - 1) // (case["grid_h"] * case["grid_w"]) + 1


def _table_rows(case):
    return _frames(case) * case["pairs_t"] + case["grid_h"] * case["pairs_h"] + case["grid_w"] * case["pairs_w"]


# --------------------------------------------------------------------------- inputs


def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _unit_rows(g, shape):
    """Rows of unit root mean square, as normalised queries and keys are."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return (x * torch.rsqrt((x * x).mean(-1, keepdim=True))).to(torch.bfloat16)


def _projected(g, shape):
    """Projections before their normalisation: every row has a size of its own."""
    size = torch.exp(torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    return (torch.randn(shape, generator=g, device="cuda") * size).to(torch.bfloat16)


def _table(case):
    """(cos, sin) of every frame, row and column position and pair, in 64 bits, rounded to 32."""
    parts = [(_frames(case), case["pairs_t"]), (case["grid_h"], case["pairs_h"]), (case["grid_w"], case["pairs_w"])]
    angles = [torch.arange(n, device="cuda", dtype=torch.float64)[:, None]
              * THETA ** (-torch.arange(p, device="cuda", dtype=torch.float64) / max(p, 1)) for n, p in parts]
    flat = torch.cat([a.reshape(-1) for a in angles])
    return torch.stack([torch.cos(flat), torch.sin(flat)], -1).to(torch.float32).contiguous()


def _rope_desc(tm, case, dtype):
    return tm.make_rope_desc(case["head_dim"], _frames(case), case["grid_h"], case["grid_w"],
                             (case["pairs_t"], case["pairs_h"], case["pairs_w"]), THETA, case["halves"], dtype)


def _inputs(case, seed):
    """The tensors of a case, on the GPU: the same for both sides, and for exact()."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, D, kv = case["batch"], case["head_dim"], case["kv_heads"]
    if case["kind"] == "rope":
        dt = _DT[case["dtype"]]
        return {"q": _normal(g, (B, case["n"], case["heads"], D), dt),
                "k": _normal(g, (B, case["n"], kv, D), dt)}
    if case["kind"] == "write_read":
        return {"k": _unit_rows(g, (B, case["n"], kv, D)), "v": _projected(g, (B, case["n"], kv, D))}
    if case["kind"] == "produce":
        x = {"q": _projected(g, (B, case["n"], case["heads"], D)), "k": _projected(g, (B, case["n"], kv, D)),
             "v": _normal(g, (B, case["n"], kv, D)), "q_gain": None, "k_gain": None}
        if case["gains"]:
            x["q_gain"] = 1 + 0.2 * torch.randn((case["heads"], D), generator=g, device="cuda")
            x["k_gain"] = 1 + 0.2 * torch.randn((kv, D), generator=g, device="cuda")
        return x
    n, lo = _lengths(case)
    # every chunk of the stream in turn; those that the window has left are overwritten in the cache
    kv_of = [(_unit_rows(g, (B, t, kv, D)), _normal(g, (B, t, kv, D))) for t in n]
    return {"q": _unit_rows(g, (B, case["n_q"], case["heads"], D)), "chunks": kv_of, "seen_from": lo}


def _codes(x):
    """8-bit codes and 32-bit scales of one chunk's rows [B, n, H, D]: a scale for each 64 tokens and head."""
    B, n, H, D = x.shape
    blocks = -(-n // BLOCK)
    f = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, blocks * BLOCK - n)).view(B, blocks, BLOCK, H, D)
    scale = f.abs().amax((2, 4)).clamp(min=LEAST) * (1 / 127)
    code = torch.round(f * scale.reciprocal()[:, :, None, :, None]).to(torch.int8)
    return code.view(B, blocks * BLOCK, H, D)[:, :n], scale


def _values(code, scale):
    """What codes [B, n, H, D] and scales [B, blocks, H] stand for, in 32 bits."""
    return code.float() * scale.repeat_interleave(BLOCK, 1)[:, :code.shape[1], :, None]


def prepare(case, seed):
    x = _inputs(case, seed)
    s = {"case": case, **x}
    if case["kind"] in ("rope", "produce"):
        s["table"] = _table(case)
    if not own:
        if case["kind"] == "attend":
            seen = [x["chunks"][0]] + x["chunks"][x["seen_from"]:]
            s["cached"] = [(_codes(k), _codes(v)) for k, v in seen]
            del s["chunks"]
        return s
    from paper_2506_03099_amd import tm
    B, D, kv = case["batch"], case["head_dim"], case["kv_heads"]
    s["tm"] = tm
    if case["kind"] == "rope":
        s["rope"] = _rope_desc(tm, case, case["dtype"])
    elif case["kind"] == "attend":
        desc = tm.make_desc(B, case["heads"], D, 1, case["chunk"], case["ref"], case["window"], "bf16")
        s["cache"] = tm.KV8Cache(desc, kv)
        for i, (k, v) in enumerate(x["chunks"]):
            tm.tm_kv8_append(s["cache"], i, k, v)
        del s["chunks"]
    else:
        # the cache in mid-stream: a reference frame and a chunk before this one
        desc = tm.make_desc(B, case.get("heads", kv), D, 1, case["n"], 64, 1, "bf16")
        s["cache"] = tm.KV8Cache(desc, kv)
        for i in range(2):
            tm.tm_kv8_append(s["cache"], i, x["k"][:, :1].contiguous(), x["v"][:, :1].contiguous())
        if case["kind"] == "produce":
            s["rope"] = _rope_desc(tm, case, "bf16") if case["rotate"] else None
    return s


# --------------------------------------------------------------------------- the plain forms


def _positions(case):
    p = case["first"] + torch.arange(case["n"], device="cuda")
    j = p % (case["grid_h"] * case["grid_w"])
    return p // (case["grid_h"] * case["grid_w"]), j // case["grid_w"], j % case["grid_w"]


def _cos_sin(case, table):
    """[n, D / 2] cosines and sines of the case's tokens (1 and 0 of the pairs that no axis turns)."""
    f, y, x = _positions(case)
    pt, ph, pw = case["pairs_t"], case["pairs_h"], case["pairs_w"]
    at = _frames(case) * pt
    rows = [table[:at].view(-1, pt, 2)[f], table[at:at + case["grid_h"] * ph].view(-1, ph, 2)[y],
            table[at + case["grid_h"] * ph:].view(-1, pw, 2)[x]]
    still = torch.zeros((case["n"], case["head_dim"] // 2 - pt - ph - pw, 2), device="cuda")
    still[..., 0] = 1
    cs = torch.cat(rows + [still], 1)
    return cs[..., 0], cs[..., 1]


def _turn(x, cos, sin, halves):
    """Rotates the pairs of x [B, n, H, D] in 32 bits."""
    c, s = cos[None, :, None], sin[None, :, None]
    if halves:
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, a * s + b * c], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)


def _plain_rope(s):
    case = s["case"]
    cos, sin = _cos_sin(case, s["table"])
    if case["direction"] == "bwd":
        sin = -sin
    return tuple(_turn(s[n].float(), cos, sin, case["halves"]).to(s[n].dtype) for n in "qk")


def _plain_write_read(s):
    dt = _DT[s["case"]["out"]]
    return tuple(_values(*_codes(s[n])).to(dt) for n in "kv")


def _plain_produce(s):
    case = s["case"]
    cos, sin = _cos_sin(case, s["table"]) if case["rotate"] else (None, None)

    def normed(x, gain):
        x = x.float()
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        x = x if gain is None else x * gain
        return _turn(x, cos, sin, case["halves"]) if case["rotate"] else x

    q, k = normed(s["q"], s["q_gain"]), normed(s["k"], s["k_gain"])
    return (q.to(torch.bfloat16), _values(*_codes(k)).to(torch.bfloat16),
            _values(*_codes(s["v"])).to(torch.bfloat16))


def _plain_attend(s):
    case = s["case"]
    B, H, kv, D, n = case["batch"], case["heads"], case["kv_heads"], case["head_dim"], case["n_q"]
    k = torch.cat([_values(*kc) for kc, _ in s["cached"]], 1).permute(0, 2, 3, 1).contiguous()  # [B, kv, D, N]
    v = torch.cat([_values(*vc) for _, vc in s["cached"]], 1).transpose(1, 2).contiguous()      # [B, kv, N, D]
    # the rows of the query heads that share a key head together
    q = s["q"].float().view(B, n, kv, H // kv, D).transpose(1, 2).reshape(B * kv, n * (H // kv), D)
    x = torch.bmm(q, k.view(B * kv, D, -1)) * (1.0 / math.sqrt(D))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p, v.view(B * kv, -1, D)) / total
    o = o.view(B, kv, n, H // kv, D).transpose(1, 2).reshape(B, n, H, D).to(torch.bfloat16)
    if not case["lse"]:
        return o
    lse = (top + torch.log(total)).view(B, kv, n, H // kv).transpose(2, 3).reshape(B, H, n)
    return o, lse.contiguous()


# --------------------------------------------------------------------------- a pass


def run(state):
    case = state["case"]
    if not own:
        return {"rope": _plain_rope, "write_read": _plain_write_read, "produce": _plain_produce,
                "attend": _plain_attend}[case["kind"]](state)
    tm = state["tm"]
    if case["kind"] == "rope":
        turn = tm.tm_rope3d_fwd if case["direction"] == "fwd" else tm.tm_rope3d_bwd
        return turn(state["rope"], state["table"], state["q"], state["k"], case["first"])
    if case["kind"] == "write_read":
        tm.tm_kv8_append(state["cache"], 2, state["k"], state["v"])
        return tm.tm_kv8_read(state["cache"], 2, _DT[case["out"]])
    if case["kind"] == "produce":
        q = tm.tm_qkv8_produce(state["cache"], 2, state["q"], state["k"], state["v"], state["q_gain"],
                               state["k_gain"], EPS, state["rope"], state["table"], case["first"])
        return (q,) + tuple(tm.tm_kv8_read(state["cache"], 2))
    if not case["lse"]:
        return tm.tm_kv8_attn_fwd(state["cache"], state["q"], case["chunks"])
    lse = torch.empty((case["batch"], case["heads"], case["n_q"]), dtype=torch.float32, device="cuda")
    return tm.tm_kv8_attn_fwd(state["cache"], state["q"], case["chunks"], lse=lse), lse


# --------------------------------------------------------------------------- the definitions in 64 bits


def _exact_spin(case):
    """exp(i angle) of every token and pair, from the positions."""
    out = torch.ones((case["n"], case["head_dim"] // 2), dtype=torch.complex128, device="cuda")
    at = 0
    for pos, p in zip(_positions(case), (case["pairs_t"], case["pairs_h"], case["pairs_w"])):
        for i in range(p):
            angle = pos.double() * math.exp(-math.log(THETA) * i / p)
            out[:, at + i] = torch.polar(torch.ones_like(angle), angle)
        at += p
    return out


def _exact_turn(case, x, spin):
    if case["halves"]:
        h = case["head_dim"] // 2
        z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * spin[None, :, None]
        return torch.cat([z.real, z.imag], -1)
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], -1, 2)) * spin[None, :, None]
    return torch.view_as_real(z).flatten(-2)


def _exact_held(x):
    """What the cache stands for after x [B, n, H, D] (64 bits) went into it, block by block."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[1], BLOCK):
        b = x[:, at:at + BLOCK]
        step = b.abs().amax((1, 3), keepdim=True).clamp(min=LEAST) / 127
        out[:, at:at + BLOCK] = torch.round(b / step) * step
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] == "rope":
        spin = _exact_spin(case)
        if case["direction"] == "bwd":
            spin = spin.conj().resolve_conj()
        return tuple(_exact_turn(case, x[n].double(), spin) for n in "qk")
    if case["kind"] == "write_read":
        return tuple(_exact_held(x[n].double()) for n in "kv")
    if case["kind"] == "produce":
        spin = _exact_spin(case)
        out = []
        for n in "qk":
            y = x[n].double()
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
            if x[n + "_gain"] is not None:
                y = y * x[n + "_gain"].double()
            out.append(_exact_turn(case, y, spin) if case["rotate"] else y)
        return out[0], _exact_held(out[1]), _exact_held(x["v"].double())
    B, H, kv, D, n = case["batch"], case["heads"], case["kv_heads"], case["head_dim"], case["n_q"]
    seen = [x["chunks"][0]] + x["chunks"][x["seen_from"]:]
    k = torch.cat([_exact_held(c[0].double()) for c in seen], 1)
    v = torch.cat([_exact_held(c[1].double()) for c in seen], 1)
    o = torch.empty((B, n, H, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, H, n), dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(H):
            logits = (x["q"][b, :, h].double() @ k[b, :, h * kv // H].T.contiguous()) / math.sqrt(D)
            lse[b, h] = torch.logsumexp(logits, -1)
            o[b, :, h] = torch.softmax(logits, -1) @ v[b, :, h * kv // H].contiguous()
    return (o, lse) if case["lse"] else o
