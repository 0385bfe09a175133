"""Host side of the block norms and linear layers, on a machine without a GPU: the sanitizer build of their
checks, parts and shares (tests/sanitize/host_block_driver.cpp), and what the binding refuses before the
library is called.
"""
import pytest
import torch

import test_host_sanitize as sanitize
from block_sizes import FEW_ROWS, PRODUCTS, SUMS

DRIVER = sanitize.DRIVER.replace("host_abi_driver", "host_block_driver")


@pytest.fixture(scope="module")
def tm():
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def refused(tm, status, fn):
    with pytest.raises(tm.TMError) as e:
        fn()
    assert e.value.status == status, e.value


def test_host_checks_parts_and_shares_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(sanitize, "DRIVER", DRIVER)
    sanitize._run()


def test_block_norm_refuses_host_tensors_and_wrong_shapes(tm):
    bf16 = torch.bfloat16
    d = tm.make_block_norm_desc(2, 64, "layer", "rms", "bf16", "f32", 1e-6, 3, 10)
    assert (d.pre, d.post, d.dtype, d.stream_dtype, d.groups, d.group_tokens) == (1, 2, tm.TM_BF16, tm.TM_F32, 3, 10)
    x, y, mod = torch.zeros((2, 5, 64)), torch.zeros((2, 5, 64), dtype=bf16), torch.zeros((2, 3, 64))
    refused(tm, tm.TM_E_ARG, lambda: tm.tm_block_norm_fwd(d, x, y))  # host memory
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_block_norm_fwd(d, x.to(bf16), y))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_block_norm_fwd(d, x[:1], y))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_block_norm_fwd(d, x[0], y))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_block_norm_bwd(d, x[..., :56], y, x, y))
    refused(tm, tm.TM_E_ARG, lambda: tm.tm_block_norm_bwd(d, None, y, x, y))
    refused(tm, tm.TM_E_ARG, lambda: tm.tm_block_norm_bwd(d, x, y, x, y, scale=mod))
    plain = tm.make_block_norm_desc(2, 64, "none", "none", "bf16", "f32")
    refused(tm, tm.TM_E_ARG, lambda: tm.tm_block_norm_bwd(plain, x, None, None, y))


def test_linear_refuses_host_tensors_and_wrong_shapes(tm):
    bf16 = torch.bfloat16
    d = tm.make_linear_desc(2, 64, 72, "gelu", "f32", 3, 10)
    assert (d.act, d.out_dtype, d.groups, d.group_tokens) == (tm.TM_ACT_GELU, tm.TM_F32, 3, 10)
    x, w, o = torch.zeros((2, 5, 64), dtype=bf16), torch.zeros((72, 64), dtype=bf16), torch.zeros((2, 5, 72))
    refused(tm, tm.TM_E_ARG, lambda: tm.tm_linear_fwd(d, x, w))  # host memory
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_linear_fwd(d, x.float(), w))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_linear_fwd(d, x[:, :, :56], w))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_linear_bwd(d, x, w, o.to(bf16)))
    refused(tm, tm.TM_E_SHAPE, lambda: tm.tm_linear_bwd(d, x, w, o[:, :, :64]))


def test_workspace_sizes(tm):
    lib = tm.lib()
    # a run of 21 groups of 1560: about a part for each CU, three sums each
    d = tm.make_block_norm_desc(1, 5120, groups=21, group_tokens=1560)
    n = lib.tm_block_norm_bwd_workspace(d, 32760, 0)
    assert n % (3 * 5120 * 4) == 0 and 200 <= n // (3 * 5120 * 4) <= 1024
    assert lib.tm_block_norm_bwd_workspace(d, 32761, 0) == 0
    # dz in bf16 at least, and room for a round of split tiles beside it
    d = tm.make_linear_desc(1, 5120, 5120, "none", "f32", 21, 1560)
    assert 32760 * 5120 * 2 <= lib.tm_linear_bwd_workspace(d, 32760, 0) < 32760 * 5120 * 2 + (200 << 20)
    assert lib.tm_linear_fwd_workspace(tm.make_linear_desc(1, 64, 64), 1) == 0


def test_plans_as_the_kernels_number_them_under_asan_and_ubsan(monkeypatch):
    """And that the sizes of the GPU tests take every kernel variant between them."""
    monkeypatch.setattr(sanitize, "DRIVER", DRIVER.replace("host_block_driver", "host_block_plan_driver"))
    args = []
    for kind, sizes in (("product", PRODUCTS + FEW_ROWS), ("sums", SUMS)):
        for size in sizes:
            args += [kind, ",".join(map(str, size))]
    sanitize._run(*args)


def test_refusals_by_their_messages_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(sanitize, "DRIVER", DRIVER.replace("host_block_driver", "host_block_refusal_driver"))
    sanitize._run()
