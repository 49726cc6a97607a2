"""The norm's backward pass reads nothing into its sums from beyond a row's width, by every kernel plan."""
import math

import pytest
import torch

from layer_inputs import Rows
from test_gpu_layer_norm import BF16, EPS, F32, Case
from test_gpu_layer_norm_spread import PIECES, width_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pieces", PIECES)
@pytest.mark.parametrize("kept", [False, True])
def test_nothing_beyond_the_width_takes_part(B, dtype, pieces, kept):
    """Rows of one number with |mu| rho beyond fp32: u is zero in all columns of the row, and of no other column is there one.  2^120 is exact in 8 bits."""
    c = Case(B, dtype, 2, 5, width_of(pieces, dtype), masked=False, seed=27)
    c.x = Rows(torch.full((c.total, c.d), 2.0 ** 120, dtype=dtype))
    checkpoint = None
    if kept:
        checkpoint = torch.empty(B.dbw_checkpoint_bytes(c.shape), dtype=torch.uint8, device="cuda")
        B.dbw_checkpoint_store(c.shape, c.x.arg, checkpoint)
    c.stats.view(-1, 2)[:] = torch.tensor([2.0 ** 120, 1 / math.sqrt(EPS)])
    c.check_backward(*c.backward(checkpoint=checkpoint))
