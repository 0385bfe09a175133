"""Host side of the rotary and 8-bit-cache calls, on a machine without a GPU: the
sanitizer build of their checks, sizes and layouts (tests/sanitize/host_kv8_driver.cpp),
and what the binding refuses before the library is called.
"""
import pytest
import torch

import test_host_sanitize as sanitize

DRIVER = sanitize.DRIVER.replace("host_abi_driver", "host_kv8_driver")


@pytest.fixture(scope="module")
def tm():
    from paper_2506_03099_amd import tm as binding
    binding.lib()
    return binding


def test_host_checks_and_layouts_under_asan_and_ubsan(monkeypatch):
    monkeypatch.setattr(sanitize, "DRIVER", DRIVER)
    sanitize._run()


def test_sizes(tm):
    # c_0 and each slot are whole blocks of 64: 1560 -> 1600, 4680 -> 4736
    d = tm.make_desc(1, 40, 128, 1560, 3, 1, 1, "bf16")
    assert tm.tm_kv8_cache_tokens(d) == 1600 + 2 * 4736
    assert tm.tm_kv8_cache_bytes(d, 40) == 2 * 40 * 11072 * 128 + 2 * 40 * 173 * 4
    assert tm.tm_kv8_cache_bytes(d, 40) / (2 * tm.tm_kv_cache_bytes(d)) < 0.51
    assert tm.tm_kv8_cache_bytes(d, 7) == 0
    assert tm.tm_kv8_cache_bytes(tm.make_desc(1, 40, 128, 1560, 3, 1, 1, "f32"), 40) == 0


def test_default_axes_of_the_rotary_descriptor(tm):
    d = tm.make_rope_desc(128, 21, 30, 52)
    assert (d.pairs_t, d.pairs_h, d.pairs_w) == (22, 21, 21)
    d = tm.make_rope_desc(64, 21, 30, 52, dtype=torch.float32, split_half=True)
    assert (d.pairs_t, d.pairs_h, d.pairs_w, d.split_half, d.dtype) == (12, 10, 10, 1, tm.TM_F32)


def test_binding_refuses_host_tensors_and_wrong_shapes(tm):
    q = torch.zeros((1, 8, 2, 128), dtype=torch.bfloat16)
    d = tm.make_rope_desc(128, 1, 2, 4)
    table = torch.zeros((22 + 2 * 21 + 4 * 21, 2))

    def refused(status, fn):
        with pytest.raises(tm.TMError) as e:
            fn()
        assert e.value.status == status, e.value

    refused(tm.TM_E_ARG, lambda: tm.tm_rope3d_fwd(d, table, q))              # host memory
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(d, table[1:], q))        # another descriptor's table
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(d, table, q[..., :64]))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_bwd(d, table, q, q[:, :7]))
    refused(tm.TM_E_SHAPE, lambda: tm.tm_rope3d_fwd(d, table, q, q_out=q.float()))
    refused(tm.TM_E_SHAPE, lambda: tm.KV8Cache(tm.make_desc(1, 4, 128, 8, 1, 1, 1, "bf16"), kv_heads=3))
    refused(tm.TM_E_DTYPE, lambda: tm.KV8Cache(tm.make_desc(1, 4, 128, 8, 1, 1, 1, "f32")))
    refused(tm.TM_E_ARG, lambda: tm.KV8Cache(tm.make_desc(1, 4, 128, 8, 1, 1, 1, "bf16"),
                                             pool=torch.zeros(100, dtype=torch.uint8)))
