"""Norms of rows whose spread is small beside their mean, by every kernel plan, against 64 bits.  Large columns are made before the
offset is added: what the mean's rounding leaves is far more than half a step of the spread."""
import math

import pytest
import torch

from layer_inputs import Rows
from test_gpu_layer_norm import BF16, F16, F32, Case

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
