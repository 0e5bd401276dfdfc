"""The torch binding's own checks (no GPU is touched)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2410_14740_amd import attention, m2c


@pytest.mark.parametrize("args,name", [
    ((1 << 32,), "keep"), (((1 << 32) + 9, 1, 2), "keep"), ((1 << 31,), "keep"), ((-1,), "keep"),
    ((9, 1 << 32, 0), "first"), ((9, 0, -(1 << 32)), "recent"),
])
def test_evict_refuses_what_32_bits_do_not_hold(args, name):
    """A `keep` of 2^32, for no limit, must not become 0, which drops all."""
    c = object.__new__(attention.KVCache)
    c.n_seqs, c.device, c.desc = 1, torch.device("cuda", 0), None
    c._lib = SimpleNamespace(m2c_kv_evict=lambda *a: m2c.M2C_OK)
    with pytest.raises(m2c.M2CError) as e:
        c.evict(*args, stream=0)
    assert e.value.status == m2c.M2C_ERR_INVALID_ARG and str(e.value).count(f"{name} ")
    c.evict((1 << 31) - 1, 0, 5, stream=0)


def test_a_cache_in_host_memory_is_refused():
    codes = torch.zeros((4, 64, 64), dtype=torch.int8)
    for kw in (dict(tensors={"k_codes": codes}), dict(tensors={}), dict(tensors={"k_codes": codes[0]}), dict(device="cpu")):
        with pytest.raises(m2c.M2CError) as e:
            attention.KVCache(1, 2, 64, 2, **kw)
        assert e.value.status == m2c.M2C_ERR_INVALID_ARG
