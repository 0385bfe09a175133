"""The 8-bit cache and the attention over it where sizes differ widely: blocks of V
of any finite size, K with a channel far above the others, rows of q with a common
part, scores of one row far above its neighbours', and the largest finite values.

The bounds are those of test_gpu_kv8.py's header, which hold for any such input:
P is off by 2^-11 of each weight that fp16 holds as a normal number, whatever its
block's scale (include/tm.h: to 2^-60 of the largest), so the output of every
dimension by 2^-11 sum_j p_j |v_j| of that dimension. The weights here are above
2^-14 of their row's largest, whose P is 2^8 times the quotient of two blocks' shares of
their units, 2^-4 at least: 2^8 * 2^-14 * 2^-4 = 2^-10, a normal fp16 number. Scores are
below 30 and the sums behind them are either of products whose sizes add up to less
than 30 as well, or exact (said where); with the share of 2^-12 for them the bound is
(2^-11 + 2^-12) sum_j p_j |v_j| again. The log-sum-exp: 1e-4.
"""
import pytest
import torch

from test_gpu_kv8 import BLOCK, bf16, check_attention, held32, in_tiles, make, queries, tm  # noqa: F401

pytestmark = pytest.mark.gpu

# query rows, heads, blocks of keys, whether in tiles of 256 rows (test_kv8_plan.py holds the layouts)
FORMS = [
    (1, 1, 8, False),        # one workgroup
    (3, 2, 50, False),       # keys split over workgroups
    (257, 1, 8, False),
    (512, 120, 8, True),     # whole tiles
    (1300, 9, 100, True),    # split ones
    (500, 75, 90, True),     # each cut in two
]


def put(tm, D, H, k, v):  # noqa: F811
    cache = make(tm, 1, H, H, D, k.shape[1], 1, 0)
    tm.tm_kv8_append(cache, 0, bf16(k).cuda(), bf16(v).cuda())
    return cache


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,blocks,tiles", FORMS)
@pytest.mark.parametrize("sizes", [
    (0.0, 2.0 ** 68),
    (2.0 ** 68, 0.0),
    (2.0 ** 76, 0.0, 1.0, 2.0 ** 76, 0.0),
    (1.0, 2.0 ** 100, 1e-9, 0.0, 2.0 ** 40, 2.0 ** 124, 1e-30, 1e6),
    (2.0 ** -55, 2.0 ** 10, 0.0, 2.0 ** 124, 0.0),
])
def test_row_sums_count_every_key_beside_values_of_any_size(tm, D, n_q, H, blocks, tiles, sizes):  # noqa: F811
    """Scores of a few units, V blocks of these sizes in turn: each key has its share of the row sum."""
    n = blocks * BLOCK
    assert in_tiles(1, H, n_q, [n], D) == tiles
    g = torch.Generator().manual_seed(31)
    k, v = torch.randn((1, n, H, D), generator=g), torch.randn((1, n, H, D), generator=g)
    for i in range(blocks):
        v[:, BLOCK * i:BLOCK * (i + 1)] *= sizes[i % len(sizes)]
    check_attention(tm, put(tm, D, H, k, v), 0, queries(1, n_q, H, D, g), f"{sizes}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,blocks,tiles", FORMS)
@pytest.mark.parametrize("large,small", [(1e6, 1e-2), (1e6, 1e-9), (2.0 ** 40, 2.0 ** -18), (3e38, 1e30)])
@pytest.mark.parametrize("at", [0, 5])
def test_dimensions_that_only_blocks_of_small_values_have(tm, D, n_q, H, blocks, tiles, large, small, at):  # noqa: F811
    """Every eighth block of V is large in dimension 0 and zero elsewhere; the other dimensions are
    held to the bound of the small values alone."""
    n = blocks * BLOCK
    assert in_tiles(1, H, n_q, [n], D) == tiles
    g = torch.Generator().manual_seed(32)
    k, v = torch.randn((1, n, H, D), generator=g), torch.randn((1, n, H, D), generator=g) * small / 4
    for i in range(at, blocks, 8):
        v[:, BLOCK * i:BLOCK * (i + 1)] = 0
        v[:, BLOCK * i:BLOCK * (i + 1), :, 0] = large
    check_attention(tm, put(tm, D, H, k, v), 0, queries(1, n_q, H, D, g), f"{large} {small}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,blocks,tiles", FORMS)
@pytest.mark.parametrize("outlier", [1, 30, 300, 3000])
def test_a_channel_of_k_far_above_the_others(tm, D, n_q, H, blocks, tiles, outlier):  # noqa: F811
    """Rows of q with a mean of their own and nothing in that channel: codes of the others are small, and
    so are the scores (the sizes of a score's products add up to about 1.2 * 0.8 sqrt(D), below 30)."""
    n = blocks * BLOCK
    assert in_tiles(1, H, n_q, [n], D) == tiles
    g = torch.Generator().manual_seed(33)
    k, v = torch.randn((1, n, H, D), generator=g), torch.randn((1, n, H, D), generator=g)
    k[..., 5] *= outlier
    q = 1 + torch.randn((1, n_q, H, D), generator=g)
    q[..., 5] = 0
    check_attention(tm, put(tm, D, H, k, v), 0, bf16(q).cuda(), f"outlier {outlier}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,blocks,tiles", FORMS)
@pytest.mark.parametrize("common", [40, 200])
def test_rows_of_q_with_a_common_part(tm, D, n_q, H, blocks, tiles, common):  # noqa: F811
    """q is whole numbers below 256, so its products with codes are whole and their sums below 2^24:
    exact, whatever their sizes. K's rows have a mean near zero, for scores of a few units."""
    n = blocks * BLOCK
    assert in_tiles(1, H, n_q, [n], D) == tiles
    g = torch.Generator().manual_seed(34)
    k, v = torch.randn((1, n, H, D), generator=g), torch.randn((1, n, H, D), generator=g)
    k = (k - k.mean(-1, keepdim=True)) * 0.3
    q = torch.round(common + torch.randn((1, n_q, H, D), generator=g))
    check_attention(tm, put(tm, D, H, k, v), 0, bf16(q).cuda(), f"common {common}")


@pytest.mark.parametrize("D,H", [(64, 1), (128, 1), (64, 250), (128, 200)])
def test_a_row_does_not_depend_on_far_larger_scores_beside_it(tm, D, H):  # noqa: F811
    """Scores of some thousand units in one row of 32: the others keep their bits."""
    n, n_q = 640, 256
    assert in_tiles(1, H, n_q, [n], D) == (H > 1)
    g = torch.Generator().manual_seed(35)
    k, v = torch.randn((1, n, H, D), generator=g), torch.randn((1, n, H, D), generator=g)
    cache = put(tm, D, H, k, v)
    q = queries(1, n_q, H, D, g)
    want = tm.tm_kv8_attn_fwd(cache, q, 0, o_f32=True)
    other = q.clone()
    other[0, 5::32] = 400 * bf16(k)[0, n - 1].cuda()
    got = tm.tm_kv8_attn_fwd(cache, other, 0, o_f32=True)
    keep = torch.ones(n_q, dtype=torch.bool, device="cuda")
    keep[5::32] = False
    assert torch.equal(got[0, keep], want[0, keep])
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,blocks,tiles", FORMS)
def test_large_rows_whose_products_are_zero(tm, D, n_q, H, blocks, tiles):  # noqa: F811
    """q and K of 1e30 in dimensions apart from each other's: every score is exactly zero."""
    n = blocks * BLOCK
    assert in_tiles(1, H, n_q, [n], D) == tiles
    g = torch.Generator().manual_seed(37)
    k, v = torch.randn((1, n, H, D), generator=g) * 1e30, torch.randn((1, n, H, D), generator=g)
    k[..., ::2] = 0
    q = torch.randn((1, n_q, H, D), generator=g) * 1e30
    q[..., 1::2] = 0
    check_attention(tm, put(tm, D, H, k, v), 0, bf16(q).cuda(), "zero products")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_finite_values_read_back(tm, D, dtype):  # noqa: F811
    n = 3 * BLOCK
    top = float(torch.finfo(torch.bfloat16).max)
    g = torch.Generator().manual_seed(36)
    x = bf16((2 * torch.rand((1, n, 2, D), generator=g) - 1) * top)
    x[:, 0, :, 0], x[:, BLOCK, :, 0] = top, -top
    assert torch.isfinite(x).all()
    cache = make(tm, 1, 2, 2, D, n, 1, 0)
    tm.tm_kv8_append(cache, 0, x.cuda(), x.cuda())
    want = torch.from_numpy(held32(x.float().numpy())).to(dtype)
    for y in tm.tm_kv8_read(cache, 0, dtype):
        assert torch.equal(y.cpu(), want)
