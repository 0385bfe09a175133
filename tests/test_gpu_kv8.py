"""The 8-bit cache: tm_kv8_append, tm_qkv8_produce, tm_kv8_read and tm_kv8_attn_fwd.

- A written chunk reads back, bit for bit, as the definition in include/tm.h says
  (numpy, fp32 operation by operation).
- The producer's cached values and queries are held to the definition in 64 bits.
  Normalising and rotating in fp32 costs below 1e-5 of a row's largest element
  (some twenty operations of 2^-24 each); coding adds half a scale; the queries'
  bf16 half an ulp.
- Attention, in its fp32 output, is held to the softmax in 64 bits of the values
  that the cache reads back as. Rounding P to fp16 is off by at most 2^-11 of
  each weight, so the output by 2^-11 sum_j p_j |v_j|. Scores are fp32 sums of D
  products and one fma: for |score| < 30 (all but the cases that say otherwise)
  they are off by less than 128 * 2^-24 * 30 / 2 < 2^-12.9 in all, P by as much
  again: 2^-12. The bound is (2^-11 + 2^-12) sum_j p_j |v_j|. The bf16 output is the
  fp32 output rounded, bit for bit. The log-sum-exp is fp32 throughout: 1e-4, as
  for the 16-bit cache.
"""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import assert_rounds_to, say

pytestmark = pytest.mark.gpu

BLOCK = 64


def in_tiles(B, Hk, rows, lengths, D):
    """Whether a call's rows go in tiles of 256 (and not of 32): the library's rule on the call's
    sizes, which the cases below are there to straddle."""
    blocks = sum(-(-n // BLOCK) for n in lengths)
    tiles, rounds = -(-rows // 32) * B * Hk, -(-(-(-rows // 256) * B * Hk) // 256)
    if D == 64:
        most, little, few_us, tile_us = 64, 22000 if blocks > 80 else 50000, 0.0045 + 0.00066 * blocks, 8 + 1.05 * blocks
    else:
        most, little, few_us, tile_us = 32, 8000 if blocks > 40 else 24000, 0.0105 + 0.0011 * blocks, 9 + 1.4 * blocks
    sooner = tiles <= 512 or 5 + tiles * few_us < rounds * tile_us
    return rows > most and (tiles * blocks > little or not sooner)


@pytest.fixture(scope="module")
def tm():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def held32(x):
    """What the cache stands for after the rows x [B, n, H, D] (fp32 numpy) went into it."""
    f = np.float32
    y = np.empty_like(x)
    for at in range(0, x.shape[1], BLOCK):
        b = x[:, at:at + BLOCK]
        top = np.abs(b).max((1, 3), keepdims=True)
        with np.errstate(all="ignore"):
            scale = np.where(np.isfinite(top), np.maximum(top, f(2.0 ** -60)) * f(1.0 / 127.0), f(np.nan))
            y[:, at:at + BLOCK] = np.rint(b * (f(1.0) / scale)) * scale
        assert scale.dtype == np.float32
    return y


def bf16(t):
    return t.to(torch.bfloat16)


def make(tm, B, H, Hk, D, ref, chunk, window, scale=0.0):
    desc = tm.make_desc(B, H, D, 1, chunk, ref, window, "bf16", scale)
    return tm.KV8Cache(desc, Hk)


def reference(q, k, v, scale):
    """Softmax attention in 64 bits: q [B, n, H, D], k, v [B, N, Hk, D] (GPU tensors); also
    sum_j p_j |v_j| and the log-sum-exp [B, H, n]."""
    B, n, H, D = q.shape
    Hk = k.shape[2]
    o = torch.empty((B, n, H, D), dtype=torch.float64, device=q.device)
    size = torch.empty_like(o)
    lse = torch.empty((B, H, n), dtype=torch.float64, device=q.device)
    for b in range(B):
        for h in range(H):
            kk, vv = k[b, :, h * Hk // H].double().contiguous(), v[b, :, h * Hk // H].double().contiguous()
            x = q[b, :, h].double() @ kk.T.contiguous() * scale
            p = torch.softmax(x, -1)
            o[b, :, h], size[b, :, h] = p @ vv, p @ vv.abs()
            lse[b, h] = torch.logsumexp(x, -1)
    return o, size, lse


def seen(tm, cache, window):
    """The keys and values that the latest chunk's queries see, as the cache stands for them."""
    t = cache.latest()
    parts = [tm.tm_kv8_read(cache, c, torch.float32) for c in [0] + list(range(max(1, t - window), t + 1))]
    return torch.cat([p[0] for p in parts], 1), torch.cat([p[1] for p in parts], 1)


BOUND = 2.0 ** -11 + 2.0 ** -12


def check_attention(tm, cache, window, q, what, scale=None):
    D = q.shape[3]
    t = cache.latest()
    k, v = seen(tm, cache, window)
    want, size, want_lse = reference(q, k, v, scale or 1.0 / math.sqrt(D))
    lse = torch.empty(want_lse.shape, dtype=torch.float32, device="cuda")
    o32 = tm.tm_kv8_attn_fwd(cache, q, t, o_f32=True, lse=lse)
    o = tm.tm_kv8_attn_fwd(cache, q, t)
    assert torch.isfinite(o32).all(), what
    worst = float(((o32.double() - want).abs() / (BOUND * size + 1e-30)).max())
    off = float((lse.double() - want_lse).abs().max())
    say(f"  {what}: largest error / bound = {worst:.3f}, lse off by {off:.1e}")
    assert worst <= 1.0, what
    assert off <= 1e-4, what
    assert_rounds_to(o, o32, what)
    return o32, lse


# --------------------------------------------------------------------------- writing and reading


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hk,n", [(1, 1, 1), (2, 3, 63), (1, 2, 64), (3, 1, 65), (1, 5, 200), (1, 40, 1000)])
def test_a_chunk_reads_back_as_the_definition_says(tm, D, B, Hk, n):
    g = torch.Generator().manual_seed(n)
    size = torch.exp(2 * torch.randn((B, n, Hk, 1), generator=g))
    k, v = bf16(torch.randn((B, n, Hk, D), generator=g)), bf16(torch.randn((B, n, Hk, D), generator=g) * size)
    cache = make(tm, B, Hk, Hk, D, n, n, 1)
    cache.pool.fill_(0xFF)  # (what was there before must not show)
    tm.tm_kv8_append(cache, 0, k.cuda(), v.cuda())
    for dtype in (torch.float32, torch.bfloat16):
        for x, y in zip((k, v), tm.tm_kv8_read(cache, 0, dtype)):
            want = torch.from_numpy(held32(x.float().numpy()))
            assert y.dtype == dtype and torch.equal(y.cpu(), want.to(dtype)), (dtype,)
            assert float((want - x.float()).abs().max()) <= 0.5001 / 127 * float(x.float().abs().max())


def test_blocks_of_zeros_tiny_huge_and_not_finite_values(tm):
    D, n = 64, 5 * BLOCK
    g = torch.Generator().manual_seed(1)
    x = torch.randn((1, n, 2, D), generator=g)
    x[:, :64] = 0
    x[:, 64:128] *= 1e-30                   # below the least magnitude: reads back as zeros
    x[:, 128:192] *= 3e37
    x[:, 200, 0, 5] = float("inf")          # only head 0's block
    x[:, 260, 1, 63] = float("nan")         # only head 1's block
    x = bf16(x)
    cache = make(tm, 1, 2, 2, D, n, 1, 0)
    tm.tm_kv8_append(cache, 0, x.cuda(), x.cuda())
    want = held32(x.float().numpy())
    for y in tm.tm_kv8_read(cache, 0, torch.float32):
        y = y.cpu().numpy()
        assert np.array_equal(y, want, equal_nan=True)
        assert np.all(y[:, :128] == 0)
        assert np.all(np.isnan(y[:, 192:256, 0])) and np.all(np.isfinite(y[:, 192:256, 1]))
        assert np.all(np.isnan(y[:, 256:, 1])) and np.all(np.isfinite(y[:, 256:, 0]))


def test_eviction_replacement_and_locate(tm):
    D, window, chunk, ref = 64, 1, 70, 5
    cache = make(tm, 2, 2, 1, D, ref, chunk, window)
    g = torch.Generator().manual_seed(5)
    rows = {}

    def put(c, n):
        rows[c] = [bf16(torch.randn((2, n, 1, D), generator=g)) for _ in range(2)]
        tm.tm_kv8_append(cache, c, rows[c][0].cuda(), rows[c][1].cuda())

    for c in range(5):
        put(c, ref if c == 0 else chunk - c)
    put(4, 3)  # the latest chunk again, shorter
    assert cache.latest() == 4 and cache.capacity == 64 + 2 * 128
    assert cache.locate(0) == (0, ref) and cache.locate(3) == (64, chunk - 3) and cache.locate(4) == (192, 3)
    for c in (0, 3, 4):
        for x, y in zip(rows[c], tm.tm_kv8_read(cache, c, torch.float32)):
            assert np.array_equal(y.cpu().numpy(), held32(x.float().numpy()))
    for c in (1, 2, 5, -1):
        with pytest.raises(tm.TMError) as e:
            tm.tm_kv8_read(cache, c)
        assert e.value.status == tm.TM_E_ORDER
    cache.reset()
    assert cache.latest() == -1


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("B,H,Hk,n,first,gains,turn", [(1, 1, 1, 1, 0, False, True), (2, 6, 2, 77, 50, True, True),
                                                       (1, 8, 8, 300, 9, True, False), (1, 10, 5, 129, 0, False, True)])
def test_producer(tm, D, halves, B, H, Hk, n, first, gains, turn):
    from test_gpu_rope import rotate64
    gh, gw, eps = 5, 9, 1e-6
    frames = (first + n - 1) // (gh * gw) + 1
    pairs = (D // 2 - 2 * (D // 6), D // 6, D // 6)
    rope = tm.make_rope_desc(D, frames, gh, gw, pairs, 10000.0, halves)
    table = tm.tm_rope3d_table(rope)
    g = torch.Generator().manual_seed(n)
    x = {"q": (H, None), "k": (Hk, None), "v": (Hk, None)}
    t = {}
    for name, (heads, _) in x.items():
        size = torch.exp(torch.randn((B, n, heads, 1), generator=g))
        t[name] = bf16(torch.randn((B, n, heads, D), generator=g) * size)
    gain = {name: 1 + 0.3 * torch.randn((x[name][0], D), generator=g) if gains else None for name in "qk"}
    cache = make(tm, B, H, Hk, D, n, 1, 0)
    q_out = tm.tm_qkv8_produce(cache, 0, t["q"].cuda(), t["k"].cuda(), t["v"].cuda(),
                               *(None if gain[m] is None else gain[m].cuda() for m in "qk"), eps,
                               rope if turn else None, table, first)
    k_out, v_out = tm.tm_kv8_read(cache, 0, torch.float32)
    want = {}
    for name in "qk":
        y = t[name].double().numpy()
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps)
        if gain[name] is not None:
            y = y * gain[name].double().numpy()
        want[name] = rotate64(y, first, gh, gw, frames, pairs, 10000.0, halves) if turn else y
    top = np.abs(want["q"]).max(-1, keepdims=True)
    err = np.abs(q_out.double().cpu().numpy() - want["q"])
    # half a bf16 ulp at |y|: 8 significant bits, so 2^(floor(log2 |y|) - 8) (an ulp at a binade's end)
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want["q"]) + 1e-5 * top, 1e-300))) - 8)
    assert np.all(err <= half + 1e-5 * top)
    kd = k_out.double().cpu().numpy()
    for at in range(0, n, BLOCK):
        w = want["k"][:, at:at + BLOCK]
        m = np.abs(w).max((1, 3), keepdims=True)
        assert np.all(np.abs(kd[:, at:at + BLOCK] - w) <= m * (0.5 / 127 + 2e-5))
    assert np.array_equal(v_out.cpu().numpy(), held32(t["v"].float().numpy()))
    # in place, and again on the same chunk: the same bits
    q2 = t["q"].cuda()
    tm.tm_qkv8_produce(cache, 0, q2, t["k"].cuda(), t["v"].cuda(),
                       *(None if gain[m] is None else gain[m].cuda() for m in "qk"), eps,
                       rope if turn else None, table, first, q_out=q2)
    assert torch.equal(q2, q_out)


# --------------------------------------------------------------------------- attention


def fill(tm, cache, lengths, g, ks=1.0, vs=1.0):
    B, D, Hk = cache.desc.batch, cache.desc.head_dim, cache.kv_heads
    for c, n in enumerate(lengths):
        k = torch.randn((B, n, Hk, D), generator=g)
        k = k / k.square().mean(-1, keepdim=True).sqrt() * ks
        tm.tm_kv8_append(cache, c, bf16(k).cuda(), bf16(torch.randn((B, n, Hk, D), generator=g) * vs).cuda())


def queries(B, n, H, D, g):
    q = torch.randn((B, n, H, D), generator=g)
    return bf16(q / q.square().mean(-1, keepdim=True).sqrt()).cuda()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,Hk,lengths,window,n_q", [
    (1, 1, 1, [1], 0, 1),                           # one key
    (1, 2, 2, [63], 0, 3),
    (2, 4, 1, [64], 1, 8),                          # 32 rows of shared heads
    (1, 4, 2, [65, 1], 1, 17),                      # 34 rows: a tile of two blocks
    (1, 3, 3, [5, 70, 70, 70, 9], 1, 9),            # eviction, ragged regions
    (1, 2, 1, [100, 200, 130], 3, 130),
    (2, 2, 2, [130, 257, 257, 100], 2, 257),        # more rows than a tile
    (1, 1, 1, [4000, 300], 1, 1),                   # a split single row
    (1, 8, 1, [3000, 64, 64, 64], 3, 4),
    (1, 2, 2, [2000, 1000], 1, 300),                # split tiles
    (3, 10, 5, [700, 320, 320], 0, 40),
    # in tiles of 256 rows
    (1, 47, 47, [1800, 40, 1800], 1, 1000),         # 188 tiles: each cut in two
    (3, 90, 90, [1300, 130, 65], 1, 250),           # 270 tiles, the last 14 split
    (4, 64, 64, [2000, 100, 1000, 290], 0, 193),    # whole rounds only; tiles of seven blocks
    (1, 64, 64, [8000, 64], 1, 65),                 # split tiles of three blocks
    (2, 100, 25, [3000, 700, 321], 1, 129),         # shared heads: 516 rows, three tiles a head
    (1, 5, 5, [6000, 3000, 3000], 1, 2500),         # 50 tiles of many parts
    (1, 1, 1, [70000, 64], 0, 700),                 # three tiles of more than 16 parts
])
def test_attention(tm, D, B, H, Hk, lengths, window, n_q):
    g = torch.Generator().manual_seed(n_q)
    if H * n_q > 4000:
        now = [lengths[0]] + lengths[max(1, len(lengths) - 1 - window):]
        assert in_tiles(B, Hk, n_q * (H // Hk), now, D)
    cache = make(tm, B, H, Hk, D, lengths[0], max(lengths[1:] + [1]), window)
    fill(tm, cache, lengths, g)
    q = queries(B, n_q, H, D, g)
    o1, l1 = check_attention(tm, cache, window, q, f"{lengths} {n_q}")
    o2, l2 = check_attention(tm, cache, window, q, "again")
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


@pytest.mark.parametrize("n_q", [1, 40, 3000])
def test_without_a_workspace(tm, n_q):
    """The parts in one workgroup: other sums, within twice the bound of the first."""
    import ctypes
    D, B, H = 128, 1, 2
    g = torch.Generator().manual_seed(2)
    cache = make(tm, B, H, H, D, 3000, 100, 1)
    fill(tm, cache, [3000, 100], g)
    q = queries(B, n_q, H, D, g)
    assert tm.lib().tm_kv8_attn_workspace(cache.handle, 1, n_q) > 0
    o1, _ = check_attention(tm, cache, 1, q, "with")
    o2 = torch.empty_like(o1)
    assert tm.lib().tm_kv8_attn_fwd(cache.handle, q.data_ptr(), 1, n_q, o2.data_ptr(), 1, None, None, 0,
                                    torch.cuda.current_stream().cuda_stream) == 0
    k, v = seen(tm, cache, 1)
    _, size, _ = reference(q, k, v, 1 / math.sqrt(D))
    assert bool(((o1 - o2).abs() <= 2 * BOUND * size).all())


@pytest.mark.parametrize("n_q,H", [(1, 2), (300, 2), (300, 170)])
@pytest.mark.parametrize("scale", [0.0, 0.7])
def test_scores_that_rise_late_and_fall(tm, n_q, H, scale):
    """Keys that grow from block to block raise the running maximum again and again; then they
    shrink. The sizes keep |score| below 30."""
    D, n = 128, 1000
    g = torch.Generator().manual_seed(7)
    cache = make(tm, 1, H, H, D, n, 1, 0, scale)
    assert in_tiles(1, H, n_q, [n], D) == (H > 2)
    k = torch.randn((1, n, H, D), generator=g)
    k = k / k.square().mean(-1, keepdim=True).sqrt()
    ramp = torch.cat([torch.linspace(0.01, 1, n // 2), torch.linspace(1, 0.01, n - n // 2)])
    size = 5.0 if scale == 0 else 0.6
    q = queries(1, n_q, H, D, g)
    # a common direction, so that scores grow with the ramp
    k = bf16((0.8 * q[:, :1].float().cpu() + 0.6 * k) * ramp[None, :, None, None] * size * 0.4)
    tm.tm_kv8_append(cache, 0, k.cuda(), bf16(torch.randn((1, n, H, D), generator=g)).cuda())
    check_attention(tm, cache, 0, q, "ramp", scale or None)


@pytest.mark.parametrize("n_q,H", [(1, 1), (257, 1), (512, 120)])
def test_blocks_whose_values_differ_by_orders(tm, n_q, H):
    """V blocks from 1e-9 to 1e6, one of zeros: the scale goes into P, so nothing over- or
    underflows, and the row sums count every key."""
    D, n = 64, 8 * BLOCK
    g = torch.Generator().manual_seed(8)
    cache = make(tm, 1, H, H, D, n, 1, 0)
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    k = torch.randn((1, n, H, D), generator=g)
    v = torch.randn((1, n, H, D), generator=g)
    for i, s in enumerate((1.0, 1e6, 1e-9, 0.0, 3e-4, 1e3, 1e-2, 1.0)):
        v[:, 64 * i:64 * i + 64] *= s
    tm.tm_kv8_append(cache, 0, bf16(k).cuda(), bf16(v).cuda())
    check_attention(tm, cache, 0, queries(1, n_q, H, D, g), "orders")


@pytest.mark.parametrize("n_q,H", [(3, 1), (300, 1), (300, 250)])
@pytest.mark.parametrize("size", [1e-35, 1e-12, 1e6])
def test_queries_of_any_size(tm, n_q, H, size):
    """Rows of q far from 1 (keys the other way round keep the scores below 30)."""
    D, n = 128, 300
    g = torch.Generator().manual_seed(11)
    cache = make(tm, 1, H, H, D, n, 1, 0)
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    fill(tm, cache, [n], g, ks=1.0 if size < 1 else 1.0 / size)
    q = bf16(queries(1, n_q, H, D, g).float() * size)
    q[:, 0] = 0  # a row of zeros sees the mean
    check_attention(tm, cache, 0, q, f"q * {size}")


@pytest.mark.parametrize("n_q,H", [(3, 1), (300, 1), (300, 250)])
@pytest.mark.parametrize("size", [1e2, 1e5, 1e8, 1e20, 1e36])
@pytest.mark.parametrize("at", [5, 170, 299])
def test_scores_of_any_size(tm, n_q, H, size, at):
    """One key's score is above the others' by 9 times `size` and more: its value is the output. (Its
    P is a power of two and the others' are 0, so the quotient by the row sum is off by a few 2^-24.)"""
    D, n = 128, 300
    g = torch.Generator().manual_seed(17)
    cache = make(tm, 1, H, H, D, n, 1, 0)
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    k = torch.randn((1, n, H, D), generator=g).clamp(-2, 2)
    k[:, at] = 4.0
    tm.tm_kv8_append(cache, 0, bf16(k).cuda(), bf16(torch.randn((1, n, H, D), generator=g)).cuda())
    # (rows of one sign)
    q = bf16(torch.randn((1, n_q, H, D), generator=g).abs().clamp(0.1, 4) * size).cuda()
    o = tm.tm_kv8_attn_fwd(cache, q, 0, o_f32=True)
    want = tm.tm_kv8_read(cache, 0, torch.float32)[1][:, at:at + 1]
    assert bool(((o - want).abs() <= 2.0 ** -20 * want.abs()).all())


@pytest.mark.parametrize("n_q,H", [(2, 1), (100, 40)])
def test_one_key_that_outweighs_a_long_cache(tm, n_q, H):
    """10000 keys at 2^-24 of the largest weight still count for their share: the fp16 weights
    keep 8 bits below the largest."""
    D, n = 64, 10000
    g = torch.Generator().manual_seed(12)
    cache = make(tm, 1, H, H, D, n, 1, 0)
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    k = torch.zeros((1, n, H, D))
    k[:, 77, :, 0] = 1.0
    v = torch.ones((1, n, H, D))
    v[:, 77] = 0
    q = torch.zeros((1, n_q, H, D))
    q[..., 0] = 24 * math.log(2) * math.sqrt(D)  # exactly one score of 24 log 2, bf16 rounding aside
    tm.tm_kv8_append(cache, 0, bf16(k).cuda(), bf16(v).cuda())
    # every one of the small weights may lose a whole unit of the last place of fp16's subnormal
    # range: 2^-24 of 2^8 times their weight's unit, i.e. relative 2^-24-8+24 = 2^-8
    kk, vv = seen(tm, cache, 0)
    want, size, _ = reference(bf16(q).cuda(), kk, vv, 1 / math.sqrt(D))
    o = tm.tm_kv8_attn_fwd(cache, bf16(q).cuda(), 0, o_f32=True)
    assert float(((o.double() - want).abs() / (2.0 ** -8 * size)).max()) <= 1.0


@pytest.mark.parametrize("n_q,H", [(4, 1), (60, 1), (510, 60)])
def test_rows_and_blocks_that_are_not_finite(tm, n_q, H):
    D, n = 64, 200
    g = torch.Generator().manual_seed(13)
    cache = make(tm, 2, H, H, D, n, 1, 0)
    assert in_tiles(2, H, n_q, [n], D) == (H > 1)
    k, v = bf16(torch.randn((2, n, H, D), generator=g)), bf16(torch.randn((2, n, H, D), generator=g))
    tm.tm_kv8_append(cache, 0, k.cuda(), v.cuda())
    q = queries(2, n_q, H, D, g)
    clean = tm.tm_kv8_attn_fwd(cache, q, 0)
    bad = q.clone()
    bad[0, 1, 0, 3] = float("nan")
    bad[1, 2, 0, 60] = float("inf")
    o = tm.tm_kv8_attn_fwd(cache, bad, 0)
    rows = torch.zeros((2, n_q, H), dtype=torch.bool, device="cuda")
    rows[0, 1, 0] = rows[1, 2, 0] = True
    assert bool(torch.isnan(o[rows]).all()) and torch.equal(o[~rows], clean[~rows])
    # a block without a scale makes its stream's and head's rows NaN, no other's
    v[1, 150, 0, 0] = float("-inf")
    tm.tm_kv8_append(cache, 0, k.cuda(), v.cuda())
    o = tm.tm_kv8_attn_fwd(cache, q, 0)
    assert bool(torch.isnan(o[1, :, 0]).all()) and torch.equal(o[0], clean[0])
    assert torch.equal(o[1, :, 1:], clean[1, :, 1:])


@pytest.mark.parametrize("D,H", [(64, 1), (128, 1), (64, 250), (128, 200)])
def test_a_row_does_not_depend_on_the_rows_beside_it(tm, D, H):
    """A row whose maximum is raised again and again, beside rows whose maximum is not: theirs keep
    their bits."""
    n, n_q = 640, 256
    g = torch.Generator().manual_seed(21)
    cache = make(tm, 1, H, H, D, n, 1, 0)
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    k = torch.randn((1, n, H, D), generator=g)
    tm.tm_kv8_append(cache, 0, bf16(k).cuda(), bf16(torch.randn((1, n, H, D), generator=g)).cuda())
    q = queries(1, n_q, H, D, g)
    want = tm.tm_kv8_attn_fwd(cache, q, 0, o_f32=True)
    other = q.clone()
    other[0, 5::32] = 40 * k[0, n - 1].cuda()
    got = tm.tm_kv8_attn_fwd(cache, other, 0, o_f32=True)
    keep = torch.ones(n_q, dtype=torch.bool, device="cuda")
    keep[5::32] = False
    assert torch.equal(got[0, keep], want[0, keep])


def test_in_place_other_stream_and_capture(tm):
    D = 128
    g = torch.Generator().manual_seed(14)
    cache = make(tm, 1, 4, 2, D, 9000, 200, 1)
    fill(tm, cache, [9000, 200], g)
    assert in_tiles(1, 2, 2 * 1000, [9000, 200], D)
    for n_q in (1, 1000):
        q = queries(1, n_q, 4, D, g)
        want = tm.tm_kv8_attn_fwd(cache, q, 1)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            other = tm.tm_kv8_attn_fwd(cache, q, 1)
        s.synchronize()
        assert torch.equal(want, other)
        out = torch.empty_like(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            tm.tm_kv8_attn_fwd(cache, q, 1, o=out)  # (under capture: without a workspace)
        for i in range(4):
            q.copy_(queries(1, n_q, 4, D, g))
            eager = torch.empty_like(q)
            assert tm.lib().tm_kv8_attn_fwd(cache.handle, q.data_ptr(), 1, n_q, eager.data_ptr(), 0, None, None, 0,
                                            torch.cuda.current_stream().cuda_stream) == 0
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
        want = tm.tm_kv8_attn_fwd(cache, q, 1)
        tm.tm_kv8_attn_fwd(cache, q, 1, o=q)
        assert torch.equal(q, want)


def test_codes_past_2_to_the_32(tm):
    """A cache whose codes pass 4 GiB: three keys far apart that alone count."""
    D, n = 128, (1 << 25) + 200
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GiB of free device memory")
    cache = make(tm, 1, 1, 1, D, n, 1, 0)
    k = torch.zeros((1, n, 1, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((1, n, 1, D), dtype=torch.bfloat16, device="cuda")
    at = [5, (1 << 24) + 77, n - 1]
    for i, t in enumerate(at):
        k[0, t, 0, 0] = 8.0
        v[0, t, 0] = float(i + 1)
    tm.tm_kv8_append(cache, 0, k, v)
    q = torch.zeros((1, 1, 1, D), dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 64.0  # score 45: the other 2^25 keys weigh 2^25 e^-45 < 1e-12 together
    o = tm.tm_kv8_attn_fwd(cache, q, 0, o_f32=True)
    assert float((o - 2.0).abs().max()) <= 2.0 ** -10
    kr, vr = tm.tm_kv8_read(cache, 0)
    assert torch.equal(kr, k) and torch.equal(vr, v)
    rows = q.expand(1, 64, 1, D).contiguous()
    assert in_tiles(1, 1, 64, [n], D)
    assert float((tm.tm_kv8_attn_fwd(cache, rows, 0, o_f32=True) - 2.0).abs().max()) <= 2.0 ** -10


def test_the_reference_call_agrees_with_the_16_bit_cache(tm):
    """The same chunks in both caches: the outputs differ by what coding K and V costs."""
    B, H, D, T = 1, 4, 128, 100
    desc = tm.make_desc(B, H, D, T, 2, 1, 1, "bf16")
    c16, c8 = tm.KVCache(desc), tm.KV8Cache(desc)
    g = torch.Generator().manual_seed(15)
    for t in range(4):
        n = T if t == 0 else 2 * T
        q = queries(B, n, H, D, g)
        k, v = queries(B, n, H, D, g), bf16(torch.randn((B, n, H, D), generator=g)).cuda()
        tm.tm_kv_append(c16, t, k, v)
        tm.tm_kv8_append(c8, t, k, v)
        a = tm.tm_sparse_causal_attn_fwd_f32out(desc, q, t, cache=c16)
        b = tm.tm_kv8_attn_fwd(c8, q, t, o_f32=True)
        # scores differ by ~0.009 (K's rms error over a row of unit size), V by ~0.012: together
        # under 5% of the output's size
        assert float((a - b).norm() / a.norm()) <= 0.05


def test_refusals(tm):
    D = 64
    cache = make(tm, 1, 4, 2, D, 10, 20, 1)
    k = torch.zeros((1, 10, 2, D), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 10, 4, D), dtype=torch.bfloat16, device="cuda")

    def refused(status, fn):
        with pytest.raises(tm.TMError) as e:
            fn()
        assert e.value.status == status, e.value

    refused(tm.TM_E_ORDER, lambda: tm.tm_kv8_attn_fwd(cache, q, 0))         # empty
    refused(tm.TM_E_ORDER, lambda: tm.tm_kv8_append(cache, 1, k, k))
    tm.tm_kv8_append(cache, 0, k, k)
    refused(tm.TM_E_ORDER, lambda: tm.tm_kv8_attn_fwd(cache, q, 1))
    refused(tm.TM_E_ORDER, lambda: tm.tm_kv8_append(cache, 2, k, k))
    big = torch.zeros((1, 21, 2, D), dtype=torch.bfloat16, device="cuda")
    refused(tm.TM_E_CAPACITY, lambda: tm.tm_kv8_append(cache, 1, big, big))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_append(cache, 1, k[:, :0], k[:, :0]))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_append(cache, 0, q, q))        # four heads
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_append(cache, 0, k.float(), k.float()))
    refused(tm.TM_E_ARG, lambda: tm.tm_kv8_append(cache, 0, k.transpose(1, 2).contiguous().transpose(1, 2), k))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_attn_fwd(cache, k, 0))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_attn_fwd(cache, q, 0, o=q, o_f32=True))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_kv8_attn_fwd(cache, q, 0, lse=torch.zeros((1, 4, 9), device="cuda")))
    rope = tm.make_rope_desc(128, 4, 2, 5)
    table = tm.tm_rope3d_table(rope)
    refused(tm.TM_E_ARG, lambda: tm.tm_qkv8_produce(cache, 0, q, k, k, eps=float("nan")))
    refused(tm.TM_E_ARG, lambda: tm.tm_qkv8_produce(cache, 0, q, k, k, rope=rope, table=table))  # head_dim
    refused(tm.TM_E_SHAPE, lambda: tm.tm_qkv8_produce(cache, 0, q, k, k, k_gain=torch.ones((4, D), device="cuda")))
    rope = tm.make_rope_desc(D, 1, 2, 5)
    table = tm.tm_rope3d_table(rope)
    refused(tm.TM_E_SHAPE, lambda: tm.tm_qkv8_produce(cache, 0, q, k, k, rope=rope, table=table, first_token=1))
    refused(tm.TM_E_ARG, lambda: tm.tm_qkv8_produce(cache, 0, q, k, k, rope=rope))
    assert cache.latest() == 0 and cache.locate(0) == (0, 10)
    assert tm.tm_kv8_attn_fwd(cache, q[:, :0], 0).shape == (1, 0, 4, D)


def test_the_producer_refuses_outputs_over_its_inputs(tm):
    D, n = 64, 32
    cache = make(tm, 1, 2, 2, D, n, n, 1)
    q = torch.zeros((1, n, 2, D), dtype=torch.bfloat16, device="cuda")
    gain = torch.ones((2, D), device="cuda")
    rope = tm.make_rope_desc(D, 1, 4, 8)
    table = tm.tm_rope3d_table(rope)
    out = torch.empty((1, n, 2, D), dtype=torch.bfloat16, device="cuda")
    in_out = out.view(-1)[:4 * D].view(torch.float32).view(2, D)
    in_pool = cache.pool[:8 * D].view(torch.float32).view(2, D)
    size = table.numel() * 4
    for more in ({"q_gain": in_out}, {"k_gain": in_out}, {"q_gain": in_pool}, {"k_gain": in_pool},
                 {"rope": rope, "table": cache.pool[:size].view(torch.float32).view(-1, 2)},
                 {"rope": rope, "table": out.view(-1)[:size // 2].view(torch.float32).view(-1, 2)}):
        with pytest.raises(tm.TMError) as e:
            tm.tm_qkv8_produce(cache, 0, q, q.clone(), q.clone(), q_out=out, **more)
        assert e.value.status == tm.TM_E_ARG, more
    assert cache.latest() == -1
    tm.tm_qkv8_produce(cache, 0, q, q.clone(), q.clone(), gain, gain, 1e-6, rope, table, q_out=out)
    assert cache.latest() == 0
