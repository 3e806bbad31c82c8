"""Batches that no launch holds (a grid has fewer than 2^32 threads) are refused by the argument checks, before any HIP
call: no GPU is needed.  Addresses are dummies that nothing reads."""
import ctypes
import os

import pytest

lrqat = pytest.importorskip("paper_2406_06385_amd.lrqat")

from test_abi_operators_cpu import EUNSUPPORTED, _attn, _kv_io, _kv_structs


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lrqat.LIB_PATH):
        pytest.skip("liblrqat.so not built")
    return lrqat._lib()


@pytest.mark.parametrize("fn", ["lrqat_kv_write", "lrqat_kv_read"])
@pytest.mark.parametrize("cache", [
    dict(scale_tokens=1),                               # 2^25 waves' spans of 32 tokens, K and V
    dict(scale_tokens=64),                              # a block of 64 tokens for four waves
])
def test_cache_batches_past_a_grid(lib, fn, cache):
    assert _kv_io(lib, fn, cache, dict(sequences=1 << 15, max_new=1 << 16, table_width=1 << 12)) == EUNSUPPORTED
    assert "one launch" in lib.lrqat_last_error().decode()


@pytest.mark.parametrize("batch,hq", [
    (dict(sequences=65535, max_new=1, max_cached=600), 300),        # a block of 256 threads for each of them and head
    (dict(sequences=65535, max_new=1, max_cached=600), 4096),
])
def test_attention_batches_past_a_grid(lib, batch, hq):
    cache = dict(kv_heads=hq, head_dim=64)
    batch = dict(batch, table_width=1 << 12)
    assert _attn(lib, cache, batch, hq=hq, qs=hq * 64, os_=hq * 64) == EUNSUPPORTED
    assert "one launch" in lib.lrqat_last_error().decode()
    c, b = _kv_structs(cache, batch)
    assert lib.lrqat_kv_attention_workspace_size(ctypes.byref(c), ctypes.byref(b), hq) == 0
