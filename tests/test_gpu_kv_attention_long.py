"""GPU checks of attention over the int8 cache on sequences that are long, longer than was planned, or grow from one
split into the next, against float64 evaluations of the definition.  The bound is the one derived in
test_gpu_kv_attention: 2^-8 |o| + 2^-10 sum p |v|."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_06385_amd import lrqat
    lrqat.load_library()
    return lrqat


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


def test_the_last_positions_of_a_full_table(lr):
    """2^31 - 2^16 positions, of which only the first page and the last two are in the cache."""
    page, d = 256, 16
    width = (2 ** 31 - 2 ** 16) // page
    cache = lr.lrqat_kv_cache(lr.KVCacheSpec(1, d, 3, page, 1))
    g = torch.Generator(device="cuda").manual_seed(61)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(-127, 128, t.shape, device="cuda", generator=g, dtype=torch.int8))
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(0.01)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -2], table[0, -1] = 2, 0, 1
    batch = lr.KVBatch(_dev([0, 1]), _dev([width * page - 1]), table, 1, 1, width * page - 1)
    q = torch.randn((1, 1, d), device="cuda", generator=g).to(torch.bfloat16)
    ws = lr.workspace(lr.lrqat_kv_attention_workspace_size(cache, batch, 1)).fill_(0xff)     # NaNs, if they were read
    O = lr.lrqat_kv_attention(cache, batch, q, ws=ws)
    k, v = (t[[2, 0, 1], 0].double().reshape(-1, d) * 0.01 for t in (cache.k, cache.v))
    p = torch.softmax(k @ q[0, 0].double() * d ** -0.5, 0)
    assert ((O[0, 0].double() - p @ v).abs() <= 2.0 ** -8 * (p @ v).abs() + 2.0 ** -10 * (p @ v.abs())).all()
