"""Norms of rows whose spread is small beside their mean, or nothing at all, by every kernel plan, against 64 bits.  Large columns are made before the
offset is added: what the mean's rounding leaves is far more than half a step of the spread."""
import math

import pytest
import torch

import layer_reference as ref
from layer_inputs import Rows
from test_gpu_layer_norm import BF16, F16, F32, TYPES, Case

pytestmark = pytest.mark.gpu

# pieces of 16 bytes that a row has at most, one number for every plan of a row in registers, and rows that registers do not hold
PIECES = [1, 13, 50, 100, 150, 250, 350, 450, 700, 900, 1400, 2000, 2500]


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def width_of(pieces, dtype, less=1):
    return pieces * (4 if dtype == F32 else 8) - less


@pytest.mark.parametrize("offset", [1000.0, 3000.0, -1e4, 1e6])
@pytest.mark.parametrize("pieces", PIECES[2:])
def test_a_small_spread_beside_a_large_mean(B, pieces, offset):
    c = Case(B, F32, 2, 6, width_of(pieces, F32), masked=False, seed=21)
    x = torch.randn(c.total, c.d, generator=c.g)
    x[:, ::97] *= 8
    c.x = Rows(x + offset)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("pieces", PIECES[2:])
def test_a_spread_of_a_few_steps(B, dtype, pieces):
    """16-bit numbers a few of their own steps apart."""
    c = Case(B, dtype, 2, 5, width_of(pieces, dtype, 3), seed=22)
    x = 3000 + 20 * torch.randn(c.total, c.d, generator=c.g)
    x[~c.on] = math.nan
    c.x = Rows(x.to(dtype))
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


def forward(c, eps):
    y = Rows.empty(c.total, c.d, c.dtype)
    c.B.dbw_layer_norm(c.shape, c.x.arg, c.params, y.arg, eps=eps, stats_out=c.stats, **c.at)
    return y.result(), c.stats.cpu().view(-1, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pieces", PIECES)
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_rows_of_equal_numbers(B, dtype, pieces, eps):
    """y is the bias and mu the number itself, exactly: every difference from the mean is zero.  rho is 1 / sqrt(eps) to the roundings of a sum, a root and a
    quotient.  Also numbers whose sum passes the largest of fp32."""
    c = Case(B, dtype, 1, 24, width_of(pieces, dtype), masked=False, seed=23)
    size = torch.exp2(torch.rand(c.total, generator=c.g) * (15 if dtype == F16 else 32))
    size[::3] *= -1
    if dtype != F16:
        size[-4:] = torch.tensor([2e36, -4e37, 123760328.0, 1060113152.0])
    x = size.to(dtype)
    c.x = Rows(x[:, None].expand(-1, c.d).contiguous())
    y, stats = forward(c, eps)
    assert torch.equal(y, c.b.expand(c.total, -1).to(dtype))
    assert torch.equal(stats[:, 0], x.float())
    rho = 1 / math.sqrt(torch.tensor(eps).double().item())
    assert ((stats[:, 1].double() - rho).abs() <= 4 * ref.U * rho).all()
    # backwards: u is zero, dx = rho (g - mean of g), which may pass fp16's largest number
    dx, grads = c.backward()
    dy = c.dy.values.double()
    want, _, _ = ref.norm_grad(dy, x.double()[:, None].expand(-1, c.d), c.rows_w, x.double()[:, None], stats[:, 1:].double())
    bound = ref.norm_grad_bound(dy, x.double()[:, None].expand(-1, c.d), c.rows_w, x.double()[:, None], stats[:, 1:].double())
    got = dx.result()
    fits = want.abs() + 2 * bound < torch.finfo(dtype).max
    assert not torch.isnan(got).any()
    ref.close(torch.where(fits, got.double(), 0.0), torch.where(fits, want, 0.0), bound, "dx", dtype)
    assert (grads[:, 3:3 + c.d] == 0).all()
    db = grads[:, 4 + c.d:4 + 2 * c.d].cpu()
    ref.close(db, dy.sum(0, keepdim=True), dy.abs().sum(0, keepdim=True) * ref.U * (c.total + 20), "db")


@pytest.mark.parametrize("width", [982, 881, 124320])
def test_equal_numbers_that_gave_no_variance(B, width):
    c = Case(B, F32, 1, 3, width, masked=False, seed=24)
    c.x = Rows(torch.tensor([123760328.0, 1060113152.0, 104726992.0])[:, None].expand(-1, width).contiguous())
    y, stats = forward(c, 1e-5)
    assert torch.equal(y, c.b.expand(3, -1)) and torch.isfinite(stats).all()
    assert torch.isfinite(c.backward()[1][:, 3:3 + width]).all()


@pytest.mark.parametrize("at", [0, 1, -1])
@pytest.mark.parametrize("pieces", PIECES[1:])
def test_one_number_apart(B, pieces, at):
    """The first one, which is as any other; one whose distance is a step of the others, or a million of them."""
    c = Case(B, F32, 1, 4, width_of(pieces, F32), masked=False, seed=25)
    x = torch.full((4, c.d), 2.0 ** 20)
    x[:, at] += torch.tensor([0.125, -0.125, 2.0 ** 17, -2.0 ** 40])
    c.x = Rows(x)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("pieces", PIECES)
def test_infinities_and_nan_are_not_held_back(B, pieces):
    """Wherever in a row: all of it is NaN, mu what the formula gives, and its neighbours are as they were."""
    c = Case(B, F32, 1, 8, width_of(pieces, F32), masked=False, seed=26)
    plain = c.forward().result()
    x = c.x.values.clone()
    for r, (at, v) in {0: (0, math.nan), 2: (0, math.inf), 3: (-1, math.inf), 5: (-1, math.nan), 6: (c.d // 2, -math.inf)}.items():
        x[r, at] = v
    c.x = Rows(x)
    y, stats = c.forward().result(), c.stats.cpu().view(-1, 2)
    for r in range(8):
        assert torch.equal(y[r], plain[r]) if r in (1, 4, 7) else torch.isnan(y[r]).all() and torch.isnan(stats[r, 1]), r


@pytest.mark.parametrize("size", [1e20, 1e35])
@pytest.mark.parametrize("pieces", PIECES)
def test_squares_beyond_fp32(B, pieces, size):
    """Where they pass it, rho is 0 and y the bias; sums of numbers this large are still numbers."""
    c = Case(B, F32, 1, 3, width_of(pieces, F32), masked=False, seed=28)
    x = torch.randn(3, c.d, generator=c.g) * size
    c.x = Rows(x)
    y, stats = forward(c, 1e-5)
    far = ((x.double() - x.double().mean(1, keepdim=True)) ** 2).sum(1) > 4e38
    assert far.any()
    assert torch.equal(y[far], c.b.expand(3, -1)[far]) and (stats[far, 1] == 0).all()
    mu, off = x.double().mean(1), (ref.depth(c.d) + 4) * ref.U * x.double().abs().mean(1)
    ref.close(stats[:, 0], mu, off + ref.U * x[:, 0].double().abs(), "mu")


@pytest.mark.parametrize("width", [3, 13, 16, 33, 50, 64])
@pytest.mark.parametrize("loud", [10.0, 1e4])
@pytest.mark.parametrize("at", [0, -1])
def test_one_centre_for_all_lanes_of_a_row(B, width, loud, at):
    """Rows by 16 lanes, one number far from the others.  u = (x - mu) rho: a difference from the one centre (U |u|), without the rest, a sum of 4 products and 4 additions
    (9 U of the differences' mean magnitude), times rho (the variance's 9 U and two products by half, a sum, a root, a quotient) and rounded (U)."""
    c = Case(B, F32, 1, 200, width, masked=False, weight=False, bias=False, seed=29)
    x = torch.randn(c.total, width, generator=c.g)
    x[:, at] *= loud
    c.x = Rows(x)
    y = c.forward().result()
    eps = torch.tensor(1e-5).double().item()
    one, none = torch.ones(c.total, width, dtype=torch.float64), torch.zeros(c.total, width, dtype=torch.float64)
    u = ref.norm(x.double(), one, none, eps)[0]
    ref.close(y, u, ref.U * ((1 + 5.5 + 3 + 1) * u.abs() + (9 + 1) * u.abs().mean(1, keepdim=True)), "u")


@pytest.mark.parametrize("offset", [1000.0, -1e4, 1e6])
@pytest.mark.parametrize("width", [3, 13, 16, 33, 64])
def test_a_small_spread_beside_a_large_mean_by_16_lanes(B, width, offset):
    c = Case(B, F32, 2, 50, width, masked=False, seed=30)
    c.x = Rows(torch.randn(c.total, width, generator=c.g) + offset)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())
