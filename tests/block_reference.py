"""The norms around a block and the linear layers in 64 bits, from their definitions, for the tests."""
from __future__ import annotations

import math

import torch

F64 = torch.float64


def group_rows(B, n, groups, group_tokens, first, device):
    """The modulation row of each token."""
    i = first + torch.arange(n, device=device)
    return i // group_tokens if group_tokens else torch.zeros_like(i)


def of_tokens(t, g):
    return t[:, g]


def normed(x, kind, eps):
    if kind == "none":
        return x
    c = x - x.mean(-1, keepdim=True) if kind == "layer" else x
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + eps)


def block_norm(p, pre, post, eps, g):
    """(r, h) of a dict of 64-bit tensors x, y, gate, ... (None: not there)."""
    r = p["x"]
    if p["y"] is not None:
        z = normed(p["y"], post, eps)
        if p["post_weight"] is not None:
            z = z * p["post_weight"]
        if p["gate"] is not None:
            z = z * of_tokens(p["gate"], g)
        r = r + z
    if pre == "none":
        return r, None
    m = normed(r, pre, eps)
    if p["pre_weight"] is not None:
        m = m * p["pre_weight"]
    if p["pre_bias"] is not None:
        m = m + p["pre_bias"]
    if p["scale"] is not None:
        m = m * (1 + of_tokens(p["scale"], g)) + of_tokens(p["shift"], g)
    return r, m


def activate(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def linear(p, act, g):
    """(o, z) of a dict of 64-bit tensors x, weight, bias, gate, residual."""
    z = p["x"] @ p["weight"].t()
    if p["bias"] is not None:
        z = z + p["bias"]
    o = activate(z, act)
    if p["gate"] is not None:
        o = o * of_tokens(p["gate"], g)
    if p["residual"] is not None:
        o = o + p["residual"]
    return o, z


def as64(p):
    return {k: None if v is None else v.to(F64) for k, v in p.items()}
