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
