"""The sums of a layer norm as its kernels take them, in fp32 on the CPU (pieces, lanes and waves in their order), for rows whose spread is nothing or little
beside their mean: many more rows than go to the GPU."""
import numpy as np
import pytest
import torch

import layer_reference as ref

f = np.float32
# threads that take a row and pieces of 16 bytes of each: the first with as many pieces as the row has
PLANS = [(16, 1), (64, 1), (64, 2), (64, 3), (64, 4), (128, 3), (256, 2), (256, 3), (512, 2), (512, 3), (512, 4)]
WIDTHS = [3, 17, 65, 100, 200, 257, 511, 700, 982, 1500, 2049, 3001, 5000, 8001, 20000]


def fma(a, b, c):
    return (np.float64(a) * np.float64(b) + np.float64(c)).astype(f)      # (a product of two fp32 numbers is exact in 64 bits)


def over_lanes(p, t):
    """[rows, T] summed over lanes, then waves."""
    n = p.shape[0]
    if t == 16:
        for s in (1, 2, 4, 8):
            p = p + np.roll(p, s, 1)
        return p[:, 0]
    w = p.reshape(n, t // 64, 4, 16)
    for s in (1, 2, 4, 8):
        moved = np.zeros_like(w)
        moved[..., s:] = w[..., :-s]
        w = w + moved
    ends = w[..., 15]
    ends = ends[..., 3] + ends[..., 2] + (ends[..., 1] + ends[..., 0])
    total = ends[:, 0]
    for k in range(1, t // 64):
        total = total + ends[:, k]
    return total


def norm(x, eps, size):
    """mu, rho, the variance and the differences from the mean [rows, width] of fp32 numbers of which a piece of 16 bytes holds 16 / size."""
    n, width = x.shape
    each = 16 // size
    t, turns = next(((t, c) for t, c in PLANS if width * size <= 16 * t * c), (1024, -(-width // (1024 * each))))
    inverse, first = f(1) / f(width), x[:, :1]
    cut = lambda v: v.reshape(n, turns, t, each)
    row = np.repeat(first, turns * t * each, 1)
    row[:, :width] = x
    there = np.zeros_like(row, dtype=bool)
    there[:, :width] = True
    pieces = cut(row)
    total = np.zeros((n, t), f)
    for i in range(turns):
        p = [pieces[:, i, :, j] for j in range(each)]
        while len(p) > 1:
            p = [p[k] + p[k + 1] for k in range(0, len(p), 2)]
        total = fma(p[0] - f(each) * first, inverse, total)
    mean = first[:, 0] + over_lanes(total, t)
    v = np.where(cut(there), pieces - mean[:, None, None, None], f(0))
    rest, squares = np.zeros((n, t), f), np.zeros((n, t), f)
    for i in range(turns):
        for j in range(each):
            rest, squares = fma(v[:, i, :, j], inverse, rest), fma(v[:, i, :, j], v[:, i, :, j], squares)
    rest, squares = over_lanes(rest, t), over_lanes(squares, t)
    variance = fma(-rest, rest, squares * inverse)
    rho = f(1) / np.sqrt(variance + f(eps))
    return mean + rest, rho, variance, fma(v, rho[:, None, None, None], (-rest * rho)[:, None, None, None]).reshape(n, -1)[:, :width]


@pytest.mark.parametrize("size", [4, 2])
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_rows_of_equal_numbers(size, eps):
    g = np.random.default_rng(1)
    for width in WIDTHS:
        x = np.exp2(g.uniform(-10, 120, 60)).astype(f) * g.choice([-1, 1], 60).astype(f)
        mu, rho, variance, u = norm(np.repeat(x[:, None], width, 1), eps, size)
        assert (mu == x).all() and (variance == 0).all() and (u == 0).all()
        assert np.abs(rho * np.sqrt(float(f(eps))) - 1).max() <= 4 * ref.U


@pytest.mark.parametrize("size", [4, 2])
def test_a_few_numbers_are_a_step_or_two_off(size):
    """The variance never loses more than some bits: it stays positive and near."""
    g = np.random.default_rng(2)
    for width in WIDTHS[1:]:
        for share in (0.001, 0.05, 0.3, 0.5):
            for base in (2.0 ** 20, 1.99 * 2 ** 20, 3e8):
                step = 2.0 ** (np.floor(np.log2(base)) - 23)
                x = (float(f(base)) + step * (g.random((20, width)) < share) * g.integers(1, 4, (20, 1))).astype(f)
                want = x.astype(np.float64).var(1)
                _, _, variance, _ = norm(x, 1e-12, size)
                assert (variance >= 0).all() and (np.abs(variance - want) <= 1e-5 * want).all(), (width, share, base)


@pytest.mark.parametrize("size", [4, 2])
@pytest.mark.parametrize("mean", [1e3, 1e4, -1e6])
def test_a_small_spread_beside_a_large_mean(size, mean):
    g = np.random.default_rng(3)
    for width in WIDTHS:
        x = g.standard_normal((8, width))
        x[:, ::97] *= 8
        x = (x + mean).astype(f)
        mu, rho, _, u = norm(x, 1e-5, size)
        one, none = torch.ones(8, width, dtype=torch.float64), torch.zeros(8, width, dtype=torch.float64)
        eps = float(f(1e-5))
        want, wmu, wrho = ref.norm(torch.from_numpy(x).double(), one, none, eps)
        bound, bmu, brho = ref.norm_bounds(torch.from_numpy(x).double(), one, none, eps)
        ref.close(torch.from_numpy(u), want, bound, f"u {width}")
        ref.close(torch.from_numpy(mu)[:, None], wmu, bmu, f"mu {width}")
        ref.close(torch.from_numpy(rho)[:, None], wrho, brho, f"rho {width}")
