"""GPU checks of what writes leave in the paged int8 KV cache for numbers that are none, and at its ends."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kv_cache import SHAPES, Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_06385_amd import lrqat
    lrqat.load_library()
    return lrqat


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,d,page,block", SHAPES)
def test_blocks_with_nans_of_every_kind_get_codes_of_zero(lr, heads, d, page, block, dtype):
    """NaNs of either sign and with any payload: scale NaN and codes 0, of the block's earlier tokens too."""
    S = Setup(lr, heads, d, page, block, [70])
    K, V = S.tokens(70, torch.float32, fused=False)
    rng = np.random.RandomState(5)
    for x in (K, V):
        bits = x.view(torch.int32)
        for p in (3, 21, 40, 69):
            for _ in range(4):
                at = p, rng.randint(heads), rng.randint(d)
                nan = 0x7f800000 | int(rng.randint(1, 1 << 23)) | (0x400000 if rng.randint(2) else 1)
                bits[at] = nan - (1 << 31) if rng.randint(2) else nan
    K, V = K.to(dtype), V.to(dtype)
    S.write([20], [0], K[:20], V[:20])
    S.write([50], [20], K[20:], V[20:])
    S.check([70])


@pytest.mark.parametrize("new,cached", [(40, 0), (33, 300), (300, 20)])
def test_a_sequence_that_ends_past_the_batch_is_cut_there(lr, new, cached):
    """The rows that the batch has are written, read and attended as if the sequence ended with them."""
    hq, hkv, d, page = 8, 2, 64, 32
    g = torch.Generator(device="cuda").manual_seed(81)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    width = (cached + new + 100) // page + 1
    table = torch.randperm(2 * width, device="cuda", generator=g).to(torch.int32).view(2, width)
    x = torch.randn((new + 3, hq + 2 * hkv, d), device="cuda", generator=g).to(torch.bfloat16)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    start = torch.randn((2, cached, hkv, d), device="cuda", generator=g).to(torch.bfloat16)
    outs = []
    for end in (new + 3, new + 90):
        cache = lr.lrqat_kv_cache(lr.KVCacheSpec(hkv, d, 2 * width, page, 16))
        for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            t.zero_()
        if cached:
            lr.lrqat_kv_write(cache, lr.KVBatch(dev([0, 0, cached]), dev([0, 0]), table, cached, cached, 0), *start)
        batch = lr.KVBatch(dev([0, 3, end]), dev([0, cached]), table, new + 3, new + 90, cached)
        lr.lrqat_kv_write(cache, batch, k, v)
        K, V = lr.lrqat_kv_read(cache, batch, torch.full_like(k, 7.0), torch.full_like(v, 7.0))
        outs.append([cache.k, cache.v, cache.k_scale, cache.v_scale, K, V]
                    + [lr.lrqat_kv_attention(cache, batch, q, causal=c, O=torch.full_like(q, 7.0)) for c in (True, False)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert (outs[0][4][3:].float() - k[3:].float()).abs().max() < 0.1 and not (outs[0][6] == 7).all(2).any()
