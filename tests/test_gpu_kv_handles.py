"""The cache's and the batch's handles follow the memory of the tensors that they hold."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

HKV, D, PAGE = 2, 64, 16


@pytest.fixture(scope="module")
def lr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_06385_amd import lrqat
    lrqat.load_library()
    return lrqat


def _dev(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _make(lr):
    cache = lr.lrqat_kv_cache(lr.KVCacheSpec(HKV, D, 6, PAGE, 1))
    batch = lr.KVBatch(_dev([0, 20]), _dev([0]), _dev([[2, 0, 5]]), 20, 20, 0)
    x = torch.randn((20, 4 + 2 * HKV, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)).to(torch.bfloat16)
    lr.lrqat_kv_write(cache, batch, x[:, 4:4 + HKV], x[:, 4 + HKV:])
    return cache, batch, x


@pytest.mark.parametrize("how", ["set_", "data"])
def test_memory_that_is_exchanged(lr, how):
    """As a program does that takes a cache off the GPU and back: the old memory is kept here, and is not used."""
    cache, batch, x = _make(lr)
    want = lr.lrqat_kv_attention(cache, batch, x[:, :4])
    held = []
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, batch.first, batch.cached, batch.page_table):
        held.append(t.view_as(t))               # shares the old memory
        new = t.clone()
        if how == "set_":
            t.set_(new)
        else:
            t.data = new
    for t in held[:2]:
        t.zero_()
    assert torch.equal(lr.lrqat_kv_attention(cache, batch, x[:, :4]), want)
    codes = cache.k.clone()
    lr.lrqat_kv_write(cache, batch, -x[:, 4:4 + HKV], x[:, 4 + HKV:])
    assert not held[0].any() and torch.equal(cache.k[2], -codes[2])
    held[6].fill_(0)
    K, _ = lr.lrqat_kv_read(cache, batch)
    assert (K.float() + x[:, 4:4 + HKV].float()).abs().max() < 0.1


def test_memory_of_another_size_is_refused(lr):
    cache, batch, x = _make(lr)
    cache.k_scale.data = torch.empty((6, HKV, PAGE - 1), device="cuda")
    with pytest.raises(ValueError, match="k_scale"):
        lr.lrqat_kv_attention(cache, batch, x[:, :4])
    cache, batch, x = _make(lr)
    cache.v.data = cache.v.cpu()
    with pytest.raises(ValueError, match="v"):
        lr.lrqat_kv_write(cache, batch, x[:, 4:4 + HKV], x[:, 4 + HKV:])
    cache, batch, x = _make(lr)
    batch.cached.data = _dev([0, 0])
    with pytest.raises(ValueError, match="cached"):
        lr.lrqat_kv_read(cache, batch)


def test_a_wider_page_table(lr):
    cache, batch, x = _make(lr)
    table = torch.full((1, 40), -1, dtype=torch.int32, device="cuda")
    table[0, :3] = batch.page_table[0]
    want = lr.lrqat_kv_attention(cache, batch, x[:, :4])
    batch.page_table.data = table
    assert torch.equal(lr.lrqat_kv_attention(cache, batch, x[:, :4]), want)


def test_copies_do_not_share_the_struct(lr):
    import copy
    cache, batch, x = _make(lr)
    want = lr.lrqat_kv_attention(cache, batch, x[:, :4])
    other = copy.deepcopy(cache)
    cache.k.zero_()
    assert torch.equal(lr.lrqat_kv_attention(other, batch, x[:, :4]), want)
