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


from test_gpu_kv_attention import Setup


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


# hq, hkv, d, page, block, new, cached, and the bound that the batch gives in place of the largest cached
OVER = {
    "one token, no splits": (32, 8, 128, 64, 1, [1], [700], 300),
    "one token, one key more": (32, 8, 128, 64, 1, [1, 1], [512, 3], 511),
    "one token, splits": (8, 2, 64, 64, 16, [1, 1], [9000, 40], 3000),
    "one token, nothing planned": (4, 4, 80, 16, 1, [1, 1, 1], [5000, 0, 700], 0),
    "128 rows, no splits": (8, 8, 80, 16, 1, [33] * 40, [5] * 20 + [900] * 20, 5),
    "128 rows, splits": (32, 8, 112, 64, 1, [450], [2000], 400),
    "256 rows, splits": (32, 8, 128, 64, 16, [300, 7], [6000, 20], 2750),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name", list(OVER))
def test_sequences_longer_than_planned(lr, name, causal):
    """max_cached below what the device holds: attended in full, and nothing is written past the workspace."""
    *shape, bound = OVER[name]
    S = Setup(lr, *shape, seed=62)
    plain = S.batch()
    S.batch = lambda: lr.KVBatch(plain.first, plain.cached, plain.page_table, S.tokens, max(S.new), bound)
    need = lr.lrqat_kv_attention_workspace_size(S.cache, S.batch(), S.hq)
    assert (need > 256) == ("no" not in name and "one key" not in name)
    room = torch.full((need + (64 << 20),), 0x5a, dtype=torch.uint8, device="cuda")     # a canary behind the workspace
    O = S.run(causal, ws=room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 0x5a).all()
    ref, err = S.reference(causal)
    assert ((O.double() - ref).abs() <= err).all()


@pytest.mark.parametrize("block", [1, 16])
@pytest.mark.parametrize("hq,hkv,seqs,new", [(8, 8, 64, 1), (64, 4, 1, 1040)], ids=["one token", "256 rows"])
def test_many_keys_whose_values_are_zeros(lr, hq, hkv, seqs, new, block):
    """512000 keys with values of zeros (scales of 2^-100, as a write leaves them) ahead of ordinary ones, in one split:
    they count in the denominator, whose float32 sum in a lane would be 2^15 times 2^114 with one token a sequence and
    more with many.  One page holds all of the zeros, and one key."""
    d, page, zeros, own = 16, 64, 8000, 2 + -(-new // 64)
    cache = lr.lrqat_kv_cache(lr.KVCacheSpec(hkv, d, own + 1, page, block))
    g = torch.Generator(device="cuda").manual_seed(63)
    for t in (cache.k, cache.v):
        t.copy_(torch.randint(-127, 128, t.shape, device="cuda", generator=g, dtype=torch.int8))
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(0.01)
    lr.lrqat_kv_write(cache, lr.KVBatch(_dev([0, page]), _dev([0]), _dev([[0]]), page, page, 0),
                      torch.randn((1, hkv, d), device="cuda", generator=g).repeat(page, 1, 1), torch.zeros((page, hkv, d), device="cuda"))
    assert (cache.v_scale[0] == 2.0 ** -100).all()
    total = (zeros + own) * page - 5
    row = [0] * zeros + list(range(1, own + 1))
    batch = lr.KVBatch(_dev(np.arange(seqs + 1) * new), _dev([total - new] * seqs), _dev([row] * seqs), seqs * new, new,
                       total - new)
    q = torch.randn((seqs * new, hq, d), device="cuda", generator=g).to(torch.bfloat16)
    assert lr.lrqat_kv_attention_workspace_size(cache, batch, hq) == 256
    O = lr.lrqat_kv_attention(cache, batch, q)
    pages = torch.tensor(row, device="cuda")
    rows = torch.arange(0, seqs * new, 13, device="cuda")
    last = total - new + rows % new
    for h in range(0, hq, 3):
        k, v = (c[pages, h * hkv // hq].double().reshape(-1, d)[:total]
                * s[pages, h * hkv // hq].double().repeat_interleave(block, 1).reshape(-1, 1)[:total]
                for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        z = q[rows, h].double() @ k.t().contiguous() * d ** -0.5
        p = torch.softmax(z.masked_fill(torch.arange(total, device="cuda") > last[:, None], -math.inf), 1)
        # the smallest weights, as in test_gpu_kv_attention: 2^-39 of the largest p b, on codes of at most 127
        err = 2.0 ** -8 * (p @ v).abs() + 2.0 ** -10 * (p @ v.abs()) + 2.0 ** -39 * 127 * own * page * 0.01 * p.amax(1, keepdim=True)
        assert ((O[rows, h].double() - p @ v).abs() <= err).all()
        assert (O[rows, h] != 0).any()


def test_a_recorded_step_that_grows_from_one_split_into_the_next(lr):
    """Write and attention recorded once and replayed as the sequence grows, past the end of the first split and past
    max_cached: the bits of the calls made one by one, and float64's values."""
    S = Setup(lr, 8, 2, 64, 64, 16, [1], [1400], seed=64)
    first, cached, table = _dev([0, 1]), _dev([0]), _dev(S.table)
    batch = lr.KVBatch(first, cached, table, 1, 1, 1200)
    need = lr.lrqat_kv_attention_workspace_size(S.cache, batch, S.hq)
    assert need > 256                                       # split (after 512 keys)
    ws, out = lr.workspace(need), torch.empty((1, S.hq, S.d), dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((1, S.hq + 2 * S.hkv, S.d), dtype=torch.bfloat16, device="cuda")

    def step():
        lr.lrqat_kv_write(S.cache, batch, x[:, S.hq:S.hq + S.hkv], x[:, S.hq + S.hkv:])
        return lr.lrqat_kv_attention(S.cache, batch, x[:, :S.hq], O=out, ws=ws)

    parts = (S.cache.k, S.cache.v, S.cache.k_scale, S.cache.v_scale)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator(device="cuda").manual_seed(65)
    S.q = x[:, :S.hq]
    for n in [*range(505, 520), 640, *range(1020, 1028), 1199, 1200, 1201, 1300, 3, 511, 512, 1400]:
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        cached.fill_(n)
        before = [t.clone() for t in parts]
        graph.replay()
        torch.cuda.synchronize()
        got, after = out.clone(), [t.clone() for t in parts]
        for t, b in zip(parts, before):
            t.copy_(b)
        ws.fill_(0xff)
        want = step().clone()
        torch.cuda.synchronize()
        assert torch.equal(got, want), n
        assert all(torch.equal(a.view(torch.uint8), t.view(torch.uint8)) for a, t in zip(after, parts))
        S.cached = [n]
        ref, err = S.reference(True)
        assert ((got.double() - ref).abs() <= err).all(), n


@pytest.mark.parametrize("shape", [(4, 1, 128, 64, 1, [1], [9000]), (32, 8, 128, 64, 1, [300], [2750])],
                         ids=["one token", "256 rows"])
def test_splits_on_a_stream_of_their_own(lr, shape):
    S = Setup(lr, *shape, seed=66)
    q = S.q.contiguous()
    want, batch = lr.lrqat_kv_attention(S.cache, S.batch(), q), S.batch()
    O = torch.zeros_like(q)
    ws = lr.workspace(lr.lrqat_kv_attention_workspace_size(S.cache, batch, S.hq)).fill_(0xff)
    later = torch.zeros_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = torch.randn(2048, 2048, device="cuda")
        for _ in range(8):                                  # what the call has to wait for
            a = (a @ a).tanh_()
        later.copy_(q)
    lr.lrqat_kv_attention(S.cache, batch, later, O=O, ws=ws, stream=side)   # the current stream is another one
    side.synchronize()
    assert torch.equal(O, want)
