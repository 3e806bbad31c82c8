"""GPU checks of attention over the int8 cache at the sizes where a block owns
128 or 256 rows (prompts and chunks), against the float64 evaluation and the
bound of test_gpu_kv_attention.  Which tile a shape gets is the plan's choice
from the sizes; test_kv_plan_rows asserts on the host that the shapes here
still get the tiles that they are listed under."""
import math

import pytest

torch = pytest.importorskip("torch")

from test_gpu_kv_attention import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_06385_amd import lrqat
    lrqat.load_library()
    return lrqat


# rows of a tile and the heads' padded width, a scale a token or a block, whether the keys are split:
#   hq, hkv, d, page, block, new, cached
SHAPES = {
    (128, 64, "token", False): (8, 8, 64, 16, 1, [33] * 30 + [1, 0, 7], [5] * 30 + [40, 3, 0]),
    (128, 64, "block", False): (16, 16, 48, 32, 16, [40] * 12 + [3], [70] * 12 + [0]),
    (128, 64, "token", True): (32, 8, 64, 64, 1, [301], [299]),
    (128, 64, "block", True): (24, 8, 64, 256, 64, [400, 31], [650, 500]),
    (256, 64, "token", False): (64, 4, 64, 64, 1, [1040], [2100]),
    (256, 64, "block", False): (64, 4, 32, 128, 32, [1040], [2100]),
    (256, 64, "token", True): (32, 8, 64, 64, 1, [300, 5], [2750, 90]),
    (256, 64, "block", True): (30, 6, 64, 64, 64, [301], [2750]),
    (128, 128, "token", False): (8, 8, 80, 16, 1, [33] * 40, [5] * 20 + [0, 1, 2, 15, 16] * 4),
    (128, 128, "block", False): (16, 16, 128, 64, 16, [40] * 13, [7] * 6 + [80] * 7),
    (128, 128, "token", True): (32, 8, 112, 64, 1, [450], [400]),
    (128, 128, "block", True): (32, 8, 128, 32, 32, [300, 200], [1100, 700]),
    (256, 128, "token", False): (64, 4, 128, 64, 1, [1040], [2100]),
    (256, 128, "block", False): (64, 4, 96, 64, 64, [1040], [2100]),
    (256, 128, "token", True): (32, 8, 128, 64, 1, [300], [2750]),
    (256, 128, "block", True): (32, 2, 112, 128, 128, [200, 9], [3000, 600]),
    (128, 256, "token", False): (16, 4, 256, 64, 1, [200, 333], [50, 10]),
    (128, 256, "block", False): (16, 16, 144, 32, 16, [40] * 12, [9] * 12),
    (128, 256, "token", True): (32, 4, 208, 64, 1, [200], [3000]),
    (128, 256, "block", True): (32, 4, 256, 256, 256, [100, 40], [2600, 500]),
}
IDS = [f"{r}x{w}-{s}{'-split' if x else ''}" for r, w, s, x in SHAPES]
SOME = [(128, 128, "token", False), (256, 128, "token", True), (128, 64, "block", True), (128, 256, "token", True)]
SOME_IDS = [IDS[list(SHAPES).index(k)] for k in SOME]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("key", list(SHAPES), ids=IDS)
def test_against_float64(lr, key, causal):
    S = Setup(lr, *SHAPES[key], seed=51)
    assert (lr.lrqat_kv_attention_workspace_size(S.cache, S.batch(), S.hq) > 256) == key[3]
    O = S.check(causal)
    assert torch.equal(O, S.run(causal))    # a second run gives the same bits


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_scales_far_apart_and_peaked_scores(lr, key):
    S = Setup(lr, *SHAPES[key], seed=52, spread=6.0)
    S.check()
    S = Setup(lr, *SHAPES[key], seed=53)
    S.scale = 3.0
    S.check()


FEW = {"one token": (4, 2, 64, 64, 1, [1, 1], [300, 90]), "one token, split": (4, 1, 128, 64, 1, [1], [3000])}


@pytest.mark.parametrize("key", list(FEW) + SOME, ids=list(FEW) + SOME_IDS)
def test_scores_that_float32_holds_in_steps(lr, key):
    """Scores of 2^20 to 2^60: what a row sees of the largest code has all the weight, in equal parts, and no weight
    leaves half precision.  The scores of one code are the same float32, those of two are a 2^7-th apart at least; the
    average is of exact values, rounded to bfloat16."""
    S = Setup(lr, *(FEW[key] if key in FEW else SHAPES[key]), seed=59)
    hot = 0
    for t in (S.cache.k, S.cache.v_scale):
        t.zero_()
    S.cache.v_scale.fill_(1.0)
    S.cache.k[..., hot] = torch.arange(S.page, device="cuda").remainder(100).to(torch.int8)
    q = torch.zeros_like(S.q)
    q[..., hot] = 1.0
    ref = torch.empty(S.q.shape, dtype=torch.float64, device="cuda")
    for i, (a, c) in enumerate(zip(S.new, S.cached)):
        for h in range(S.hkv):
            v = S.cache.v[torch.from_numpy(S.table[i, :-(-(a + c) // S.page)]).long().cuda(), h].double().reshape(-1, S.d)
            code = torch.arange(len(v), device="cuda") % S.page % 100
            for r in range(a):
                best = code[:c + r + 1] == code[:c + r + 1].max()
                group = S.hq // S.hkv
                ref[int(S.first[i]) + r, h * group:(h + 1) * group] = v[:c + r + 1][best].mean(0)
    for exponent in (20, 23, 24, 24.5, 25, 25.3, 26, 27.7, 28, 31, 40, 60):
        S.cache.k_scale.fill_(2.0 ** exponent / 64)
        O = lr.lrqat_kv_attention(S.cache, S.batch(), q, scale=1.0)
        assert ((O.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -10 * 127).all(), exponent


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_scores_that_rise_and_fall_along_the_keys(lr, key):
    """Every row's largest score moves up by a little at a time, and down again: one step's maximum is within, at and
    past twice the weight of the one before."""
    S = Setup(lr, *SHAPES[key], seed=54)
    S.q.abs_()
    for up in (True, False):
        for i, n in enumerate(a + b for a, b in zip(S.new, S.cached)):
            at = torch.arange(-(-n // S.page), device="cuda").float() / 4
            for p, x in zip(S.table[i], (at if up else at.flip(0)).tolist()):
                S.cache.k[int(p)].abs_()
                S.cache.k_scale[int(p)] = 0.002 * (1 + x)
        for i, n in enumerate(a + b for a, b in zip(S.new, S.cached)):
            if n % S.page:  # past the sequence's end: as before, nothing that a row may see
                S.cache.k_scale[int(S.table[i, n // S.page]), :, -(-(n % S.page) // S.block):] = math.nan
        S.check()


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_rows_without_keys_give_zeros(lr, key):
    """Pages that lie outside the cache hold nothing: rows that see only such pages are empty."""
    S = Setup(lr, *SHAPES[key], seed=55)
    S.table[0, 0] = -1
    S.table[0, 2] = 2 ** 31 - 1
    S.table[-1, 1] = S.spec.pages
    for causal in (True, False):
        O = S.check(causal)
        if causal and S.cached[0] < S.page:
            assert not O[:S.page - S.cached[0]].any()
    S.table[0, :] = S.spec.pages                    # a sequence with no pages at all
    for causal in (True, False):
        assert not S.check(causal)[:S.new[0]].any()


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_a_nan_reaches_only_the_rows_that_see_it(lr, key):
    S = Setup(lr, *SHAPES[key], seed=56)
    group, head, at = S.hq // S.hkv, S.hkv - 1, S.cached[0] + S.new[0] // 2
    page, slot = int(S.table[0, at // S.page]), at % S.page
    first = at // S.block * S.block
    rows = (torch.arange(S.new[0], device="cuda") + S.cached[0] >= first)[:, None].expand(-1, group)
    for code, scale in ((S.cache.v, S.cache.v_scale), (S.cache.k, S.cache.k_scale)):
        was = scale[page, head, slot // S.block].clone()
        scale[page, head, slot // S.block] = math.nan
        code[page, head, slot // S.block * S.block:slot // S.block * S.block + S.block] = 0
        bad = S.run().isnan()
        assert torch.equal(bad.all(2), bad.any(2))
        bad = bad.all(2)
        assert torch.equal(bad[:S.new[0], head * group:(head + 1) * group], rows)
        assert int(bad.sum()) == int(rows.sum())
        scale[page, head, slot // S.block] = was
    q = S.q.clone()
    q[S.new[0] // 3, 1, 5] = math.nan
    O = lr.lrqat_kv_attention(S.cache, S.batch(), q)
    assert O[S.new[0] // 3, 1].isnan().all() and int(O.isnan().any(2).sum()) == 1


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_blocks_of_zeros(lr, key):
    """Scales of 0 (a cache that another program quantised) count in the denominator and add nothing."""
    S = Setup(lr, *SHAPES[key], seed=57)
    for p in (0, 2):
        for t in (S.cache.k_scale, S.cache.v_scale):
            t[int(S.table[0, p])] = 0.0
    S.check()


@pytest.mark.parametrize("key", SOME, ids=SOME_IDS)
def test_strides_and_in_place(lr, key):
    S = Setup(lr, *SHAPES[key], seed=58)
    ref = S.run()
    dense = S.q.contiguous()
    assert torch.equal(lr.lrqat_kv_attention(S.cache, S.batch(), dense, scale=S.scale), ref)
    wide = torch.full((S.tokens, S.hq + 3, S.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lr.lrqat_kv_attention(S.cache, S.batch(), S.q, scale=S.scale, O=wide[:, 2:S.hq + 2])
    assert torch.equal(wide[:, 2:S.hq + 2], ref) and (wide[:, :2] == 7).all() and (wide[:, S.hq + 2] == 7).all()
    lr.lrqat_kv_attention(S.cache, S.batch(), dense, scale=S.scale, O=dense)
    assert torch.equal(dense, ref)


@pytest.mark.parametrize("key", list(FEW) + SOME, ids=list(FEW) + SOME_IDS)
def test_values_near_the_end_of_bfloat16(lr, key):
    S = Setup(lr, *(FEW[key] if key in FEW else SHAPES[key]), seed=60)
    S.cache.v_scale.mul_(2.0 ** 115)
    S.check()
