"""Tensors of the 8-bit cache's producer that lie where the call writes."""
import pytest
import torch

from test_gpu_kv8 import make, tm  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("at", [0, 4096])
def test_the_producer_refuses_queries_in_the_pool(tm, at):  # noqa: F811
    D, n = 64, 32
    cache = make(tm, 1, 2, 2, D, n, n, 1)
    k, out = (torch.zeros((1, n, 2, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = cache.pool[at:at + 2 * k.numel()].view(torch.bfloat16).view(k.shape)
    for q_out in (out, q):
        with pytest.raises(tm.TMError) as e:
            tm.tm_qkv8_produce(cache, 0, q, k, k.clone(), q_out=q_out)
        assert e.value.status == tm.TM_E_ARG
    assert cache.latest() == -1
    tm.tm_qkv8_produce(cache, 0, k.clone(), k, k.clone(), q_out=out)
    assert cache.latest() == 0
