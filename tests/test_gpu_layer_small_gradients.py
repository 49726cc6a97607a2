"""Weight gradients from 8 bits of large and small dy: every type's range, where parts of a number are subnormal."""
import pytest
import torch

import layer_reference as ref
from layer_inputs import Rows
from test_gpu_layer_checkpoint import BF16, F16, F32, Layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


@pytest.mark.parametrize("dtype,power", [(F32, 60), (F32, -60), (F32, -90), (BF16, 60), (BF16, -60), (BF16, -90), (F16, 6), (F16, -8)])
@pytest.mark.parametrize("rows,width,out", [(40, 64, 64), (1030, 300, 270)])
def test_large_and_small_numbers(B, dtype, power, rows, width, out):
    """To the same relative bound as numbers near one (the smallest here, 2^-102 or so, and their products are normal numbers)."""
    c = Layer(B, dtype, 1, rows, width, out, seed=31)
    c.dy = Rows((c.dy.values.double() * 2.0 ** power).to(dtype))
    c.check(c.run(), what=str(power))


# sizes of all three types of tiles, dense and by expert
@pytest.mark.parametrize("power", range(-126, -110, 3))
@pytest.mark.parametrize("workers,rows,width,out,experts,k", [(1, 40, 64, 64, 0, 1), (40, 64, 200, 200, 0, 1), (64, 40, 256, 256, 0, 1), (2, 60, 40, 50, 3, 2)])
def test_fp32_gradients_of_less_than_2_to_the_minus_110(B, power, workers, rows, width, out, experts, k):
    """Every number enters to within 2^-133, and the sums are fp32 sums: to dy's own 2^-149 they would be off by the bound of Layer.check(), and a step
    of fp32's smallest numbers for each addition."""
    c = Layer(B, F32, workers, rows, width, out, experts=experts, k=k, seed=32)
    g = torch.Generator().manual_seed(power + 200)
    dy = torch.randn(c.dy.values.shape, generator=g) * 2.0 ** power
    dy[torch.isnan(c.dy.values)] = float("nan")
    c.dy = Rows(dy)
    got = c.run(bias=False).cpu()
    count = c.e * out
    weight = got[:, c.weight_at:c.weight_at + count * width].reshape(workers, c.e, out, width)
    for i in sorted({0, workers - 1}):
        for e in range(c.e):
            if c.start is None:
                a, z = i * c.r, (i + 1) * c.r
                x = c.x[a:z]
            else:
                a, z = (c.start[i * (c.e + 1) + e + j].item() for j in (0, 1))
                x = c.x[c.source[a:z].long() // k]
            d = dy[a:z].double()
            size = x.abs().sum(0)
            bound = d.t().abs() @ x.abs() * 2 * ref.U * (z - a + 8) + 2.0 ** -133 * size + 3 * (z - a + 8) * 2.0 ** -149
            ref.close(weight[i, e], d.t() @ x, bound, f"2^{power} worker {i} layer {e}")
