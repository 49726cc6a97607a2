"""Layer norm and its backward pass against the same in 64 bits (layer_reference.py): types, odd sizes, strides and starts, rows that take no
part whatever they hold, none at all, in place, from 8 bits, other streams, captured calls."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref
from layer_inputs import MARK, Rows, activations, some

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
EPS = float(np.float32(1e-5))


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


class Case:
    def __init__(self, B, dtype, workers, rows, width, pad=0, shift=0, masked=True, weight=True, bias=True, seed=0, offset=0.0, pad_out=None):
        g = self.g = torch.Generator().manual_seed(seed * 7919 + width)
        self.B, self.dtype, self.n, self.t, self.d = B, dtype, workers, rows, width
        self.total = total = workers * rows
        self.mask = some(g, total) if masked else torch.ones(total, dtype=torch.uint8)
        self.on = self.mask.bool()
        x, dy = activations(g, total, width, dtype, offset), activations(g, total, width, dtype)
        x[~self.on] = math.nan
        dy[~self.on] = -math.inf
        self.pad, self.shift, self.pad_out = pad, shift, pad if pad_out is None else pad_out
        self.x, self.dy = Rows(x, pad, shift), Rows(dy, self.pad_out, shift)
        self.w, self.b = torch.ones(workers, width), torch.zeros(workers, width)
        self.at = {"weight_at": -1, "bias_at": -1}
        ld = 2 * width + 5
        p = torch.full((workers, ld), math.nan)
        if weight:
            self.w, self.at["weight_at"] = torch.randn(workers, width, generator=g), 3
            p[:, 3:3 + width] = self.w
        if bias:
            self.b, self.at["bias_at"] = torch.randn(workers, width, generator=g), 4 + width
            p[:, 4 + width:4 + 2 * width] = self.b
        self.params = p.cuda()
        self.shape = B.make_rows(workers, rows, width, dtype, ld=width + pad, ld_out=width + self.pad_out)
        self.mask_arg = self.mask.cuda() if masked else None
        self.stats = torch.full((total * 2,), MARK, device="cuda")
        self.work = torch.full((B.dbw_layer_norm_work_bytes(self.shape),), 255, dtype=torch.uint8, device="cuda")
        self.rows_w, self.rows_b = (v.double().repeat_interleave(rows, 0) for v in (self.w, self.b))

    def forward(self, y=None, checkpoint=None):
        y = y or Rows.empty(self.total, self.d, self.dtype, self.pad_out, self.shift)
        self.B.dbw_layer_norm(self.shape, self.x.arg, self.params, y.arg, mask=self.mask_arg, stats_out=self.stats, checkpoint=checkpoint, **self.at)
        return y

    def check_forward(self, y, what=""):
        x = torch.where(self.on[:, None], self.x.values.double(), 0.0)
        want, mu, rho = ref.norm(x, self.rows_w, self.rows_b, EPS)
        bound, bound_mu, bound_rho = ref.norm_bounds(x, self.rows_w, self.rows_b, EPS)
        on = self.on[:, None]
        zero = torch.zeros((), dtype=torch.float64)
        ref.close(y.result(what), torch.where(on, want, zero), torch.where(on, bound, zero), what + " y", self.dtype)
        stats = self.stats.view(-1, 2)
        ref.close(stats[:, :1], torch.where(on, mu, zero), torch.where(on, bound_mu, zero), what + " mu")
        ref.close(stats[:, 1:], torch.where(on, rho, zero), torch.where(on, bound_rho, zero), what + " rho")

    def backward(self, dx=None, checkpoint=None, dy=None, stats=None):
        dx = dx or Rows.empty(self.total, self.d, self.dtype, self.pad, self.shift)
        grads = torch.full((self.n, 2 * self.d + 5), MARK, device="cuda")
        self.B.dbw_layer_norm_grad(self.shape, (dy or self.dy).arg, None if checkpoint is not None else self.x.arg, self.stats, self.params, dx.arg, grads,
                                   self.work, mask=self.mask_arg, checkpoint=checkpoint, **self.at)
        return dx, grads

    def check_backward(self, dx, grads, x=None, what=""):
        """stats as they are on the GPU: they are inputs of the backward pass."""
        on = self.on[:, None]
        stats = self.stats.cpu().double().view(-1, 2)
        x = torch.where(on, (self.x.values.double() if x is None else x), 0.0)
        dy = torch.where(on, self.dy.values.double(), 0.0)
        mu, rho = stats[:, :1], stats[:, 1:]
        want, tw, tb = ref.norm_grad(dy, x, self.rows_w, mu, rho)
        ref.close(dx.result(what), want, ref.norm_grad_bound(dy, x, self.rows_w, mu, rho), what + " dx", self.dtype)
        got = grads.cpu()
        covered = torch.ones_like(got, dtype=torch.bool)
        for name, terms, extra in (("weight_at", tw, 3), ("bias_at", tb, 0)):
            at = self.at[name]
            if at < 0:
                continue
            terms = terms.view(self.n, self.t, self.d)
            ref.close(got[:, at:at + self.d], terms.sum(1), terms.abs().sum(1) * ref.U * (self.t + 20 + extra), what + " " + name)
            covered[:, at:at + self.d] = False
        assert (got[covered] == MARK).all(), what + ": other columns of the gradients were written"


WIDTHS = [1, 2, 7, 16, 33, 64, 100, 257, 512, 1000, 1030, 2049, 4096, 5000, 8192, 16385]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_and_its_gradient(B, dtype, width):
    c = Case(B, dtype, 3, 5, width, pad=width % 3, shift=width % 2, seed=1)
    c.check_forward(c.forward(), f"{width}")
    c.check_backward(*c.backward(), what=f"{width}")


# long rows, which registers do not hold, and many rows, which are summed in strips
@pytest.mark.parametrize("dtype,workers,rows,width,pad", [(BF16, 2, 3, 40001, 1), (F32, 1, 9, 20000, 0), (F16, 1, 2, 131072, 0), (F32, 1, 1, 300001, 3),
                                                          (F32, 3, 700, 16, 0), (BF16, 1, 2100, 100, 5), (BF16, 2, 300, 2048, 0), (F16, 5, 67, 1001, 13),
                                                          (F32, 1, 600, 5000, 0), (BF16, 600, 2, 64, 0), (F32, 40, 1, 513, 2), (BF16, 1, 1, 4096, 0),
                                                          (F16, 1, 900, 20001, 0)])
@pytest.mark.parametrize("kept", [False, True])
def test_many_rows_and_long_ones(B, dtype, workers, rows, width, pad, kept):
    c = Case(B, dtype, workers, rows, width, pad=pad, seed=2)
    checkpoint = torch.full((B.dbw_checkpoint_bytes(c.shape),), 255, dtype=torch.uint8, device="cuda") if kept else None
    c.check_forward(c.forward(checkpoint=checkpoint))
    x = None
    if kept:
        x = ref.kept(torch.where(c.on[:, None], c.x.values, 0))
        own = torch.full_like(checkpoint, 99)
        B.dbw_checkpoint_store(c.shape, c.x.arg, own, mask=c.mask_arg)
        assert torch.equal(checkpoint, own)
    c.check_backward(*c.backward(checkpoint=checkpoint), x=x)


# on either side of what 64, 128, 256 and 512 threads hold in one to four pieces of 16 bytes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pieces", [64, 128, 192, 256, 384, 512, 768, 1024, 1536, 2048])
@pytest.mark.parametrize("more", [-3, 0, 1])
def test_rows_as_long_as_registers(B, dtype, pieces, more):
    width = pieces * (4 if dtype == F32 else 8) + more
    c = Case(B, dtype, 2, 37, width, pad=1 - more % 2, seed=12)
    checkpoint = torch.full((B.dbw_checkpoint_bytes(c.shape),), 255, dtype=torch.uint8, device="cuda")
    c.check_forward(c.forward(checkpoint=checkpoint), f"{width}")
    own = torch.full_like(checkpoint, 99)
    B.dbw_checkpoint_store(c.shape, c.x.arg, own, mask=c.mask_arg)
    assert torch.equal(checkpoint, own)
    c.check_backward(*c.backward(), what=f"{width}")
    c.check_backward(*c.backward(checkpoint=checkpoint), what=f"{width} kept", x=ref.kept(torch.where(c.on[:, None], c.x.values, 0)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("width", [20, 3000, 40000])
def test_without_weight_or_bias(B, dtype, weight, bias, width):
    c = Case(B, dtype, 2, 6, width, weight=weight, bias=bias, masked=False, seed=3)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())
    if not weight and not bias:
        c.params = None
        c.check_forward(c.forward())
    # no gradients of parameters wanted
    dx = Rows.empty(c.total, c.d, dtype)
    B.dbw_layer_norm_grad(c.shape, c.dy.arg, c.x.arg, c.stats, c.params, dx.arg, None, c.work, **c.at)
    c.check_backward(dx, torch.full((c.n, 2 * width + 5), MARK, device="cuda"), what="dx alone") if not weight and not bias else None
    assert torch.equal(dx.flat, c.backward()[0].flat)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("width", [50, 2000, 30001])
def test_in_place(B, dtype, width):
    c = Case(B, dtype, 2, 7, width, pad=3, shift=1, seed=4)
    y = c.forward()
    dx, grads = c.backward()
    over_dy = Rows(c.dy.values, c.pad, c.shift)
    got, same = c.backward(dx=over_dy, dy=over_dy)
    assert torch.equal(got.result(), dx.result()) and torch.equal(same, grads)
    again = Rows(c.x.values, c.pad, c.shift)
    B.dbw_layer_norm_grad(c.shape, c.dy.arg, again.arg, c.stats, c.params, again.arg, grads, c.work, mask=c.mask_arg, **c.at)
    assert torch.equal(again.result(), dx.result())
    over = Rows(c.x.values, c.pad, c.shift)
    B.dbw_layer_norm(c.shape, over.arg, c.params, over.arg, mask=c.mask_arg, **c.at)
    assert torch.equal(over.result(), y.result())


def test_strides_of_what_goes_in_and_comes_out_differ(B):
    for width in (33, 2000, 20000):
        c = Case(B, BF16, 2, 5, width, pad=2, pad_out=7, seed=5)
        c.check_forward(c.forward())
        c.check_backward(*c.backward())


@pytest.mark.parametrize("width", [64, 1000, 20000])
def test_a_large_mean_beside_a_small_spread(B, width):
    c = Case(B, F32, 1, 4, width, masked=False, seed=6, offset=3000.0)
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


def test_rows_of_equal_numbers_and_infinities(B):
    c = Case(B, F32, 1, 4, 100, masked=False, seed=7)
    c.x.flat[:100] = 2.5
    c.x.flat[150] = math.inf
    c.x.flat[250] = math.nan
    y = c.forward().result()
    assert torch.equal(y[0], c.b[0])
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and torch.isfinite(y[3]).all()


@pytest.mark.parametrize("width", [16, 2048, 20000])
def test_no_rows_and_none_that_take_part(B, width):
    shape = B.make_rows(3, 0, width, F32)
    grads = torch.full((3, 2 * width + 4), MARK, device="cuda")
    none = torch.empty(0, device="cuda")
    params = torch.ones(3, 2 * width, device="cuda")
    work = torch.empty(B.dbw_layer_norm_work_bytes(shape), dtype=torch.uint8, device="cuda")
    B.dbw_layer_norm(shape, none, params, none, weight_at=0)
    B.dbw_layer_norm_grad(shape, none, none, none, params, none, grads, work, weight_at=0, bias_at=width + 1)
    want = torch.zeros_like(grads)
    want[:, width] = MARK
    want[:, 2 * width + 1:] = MARK
    assert torch.equal(grads, want)
    c = Case(B, BF16, 2, 9, width, seed=8)
    c.mask[:] = 0
    c.on[:] = False
    c.mask_arg = c.mask.cuda()
    c.check_forward(c.forward())
    c.check_backward(*c.backward())


def test_on_another_stream_and_twice_the_same(B):
    c = Case(B, BF16, 2, 300, 1000, seed=9)
    y, (dx, grads) = c.forward(), c.backward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        y2, (dx2, grads2) = c.forward(), c.backward()
    s.synchronize()
    assert torch.equal(y.flat, y2.flat) and torch.equal(dx.flat, dx2.flat) and torch.equal(grads, grads2)


def test_two_calls_at_once_and_masks_of_truth_values(B):
    """On two streams, with outputs and scratch memory of their own."""
    a, b = Case(B, BF16, 2, 900, 2048, seed=11), Case(B, F32, 3, 400, 500, seed=12)
    a.mask_arg = a.mask_arg.bool()
    want = [(c.forward().flat.clone(), *(v if torch.is_tensor(v) else v.flat for v in c.backward())) for c in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for turn in range(3):
        for i, c in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                y = c.forward()
                dx, grads = c.backward()
                got[i] = (y.flat, dx.flat, grads)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, w) for x, w in zip(got[i], want[i]))


@pytest.mark.parametrize("width", [100, 2048, 20000])
def test_captured_and_replayed(B, width):
    c = Case(B, BF16, 2, 200, width, seed=10)
    kept = torch.zeros(B.dbw_checkpoint_bytes(c.shape), dtype=torch.uint8, device="cuda")
    y, dx = (Rows.empty(c.total, width, BF16) for _ in range(2))
    grads = torch.zeros(2, 2 * width + 5, device="cuda")

    def step():
        B.dbw_layer_norm(c.shape, c.x.arg, c.params, y.arg, mask=c.mask_arg, stats_out=c.stats, checkpoint=kept, **c.at)
        B.dbw_layer_norm_grad(c.shape, c.dy.arg, None, c.stats, c.params, dx.arg, grads, c.work, mask=c.mask_arg, checkpoint=kept, **c.at)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step()
    for turn in range(3):
        values = activations(c.g, c.total, width, BF16)
        c.x.view(c.x.flat)[:] = values.cuda()
        c.work.fill_(turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.flat.clone(), dx.flat.clone(), grads.clone()
        c.work.fill_(200)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], y.flat) and torch.equal(got[1], dx.flat) and torch.equal(got[2], grads)
