"""GPU checks of the RMS norm's codes at the ends of the number range: what is no number shows in the scale, and rows
of very small values keep their codes.  Bounds as in test_gpu_norm."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_norm import EPS, TOL, _inputs, _near, _reference

pytestmark = pytest.mark.gpu

WIDTHS = [1, 100, 512, 4096, 16385, 40001]


@pytest.fixture(scope="module")
def lr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2406_06385_amd import lrqat
    lrqat.load_library()
    return lrqat


def _codes(lr, x, g, r=None):
    q = lr.int8_tokens(*x.shape)
    lr.lrqat_rmsnorm_forward(x, g, EPS, R=r, codes=q)
    torch.cuda.synchronize()
    return q


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", WIDTHS)
def test_what_a_gain_of_zero_hides_shows_in_the_scale(lr, n, dtype):
    x, _, g = _inputs(6, n, dtype, False, seed=71)
    at = n // 2
    g[at] = 0.0
    x[1, at] = float("inf")
    x[2, at] = float("-inf")
    x[4, at] = float("nan")
    q = _codes(lr, x, g)
    assert q.sx.isnan().tolist() == [False, True, True, False, True, False]
    # infinities that only the residual's addition makes
    x[1], x[2], x[4] = x[0], x[3], x[5]
    big = torch.finfo(dtype).max
    r = torch.zeros_like(x)
    x[3, at], r[3, at] = big, big
    q = _codes(lr, x, g, r)
    assert q.sx.isnan().tolist() == [False, False, False, True, False, False]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", WIDTHS)
def test_a_gain_that_is_no_number(lr, n, bad):
    x, _, g = _inputs(5, n, torch.bfloat16, False, seed=72)
    g[n - 1] = bad
    x[2, n - 1] = 0.0           # 0 times it: a NaN as well
    assert _codes(lr, x, g).sx.isnan().all()


@pytest.mark.parametrize("n", WIDTHS)
def test_squares_past_float32(lr, n):
    """1 / sqrt of an infinite sum would be 0, and the row one of zeros."""
    x, _, g = _inputs(4, n, torch.float32, False, seed=73)
    x[1, 0] = 1e25
    x[2, n - 1] = -3e38
    assert _codes(lr, x, g).sx.isnan().tolist() == [False, True, True, False]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", WIDTHS)
def test_rows_of_the_smallest_values(lr, n, dtype):
    """Down to subnormal values: with the squares beside eps, y is h g / sqrt(eps), and its codes are those of h g.
    Powers of 2 times whole numbers, so that h g and its quotients are exact; the scale of the smallest rows is itself
    subnormal, its last place 2^-149."""
    whole = torch.randint(-100, 101, (7, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(74))
    whole[:, 0] = 100
    whole[6, 1:] = 0
    exponents = torch.tensor([-90, -110, -118, -121, -126, -132, -126], device="cuda")
    x = (whole.double() * torch.exp2(exponents.double())[:, None]).to(dtype)
    assert torch.equal(x.double(), whole.double() * torch.exp2(exponents.double())[:, None])
    g = torch.ones(n, device="cuda")
    q = _codes(lr, x, g)
    u = whole.double() * 127 / 100
    assert not (((u - torch.floor(u)) - 0.5).abs() < 1e-4)[whole.abs() != 50].any()
    off = (q.codes[:, :n].double() - torch.round(u)).abs()
    assert not off[whole.abs() != 50].any() and off.max() <= 1         # 63.5: either side
    assert not q.codes[:, n:].any()
    assert torch.equal(q.nsum, q.codes.sum(1, dtype=torch.int32))
    s = 100 * torch.exp2(exponents.double()) / EPS ** 0.5 / 127
    assert ((q.sx.double() - s).abs() <= 2e-6 * s + 2.0 ** -148).all()
