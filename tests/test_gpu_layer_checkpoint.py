"""Rows in 8 bits against the format's definition (layer_reference.py), and the weight gradient of a linear layer from them."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref
from layer_inputs import MARK, Rows, activations, some

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def store(B, x, workers, mask=None):
    shape = B.make_rows(workers, x.total // workers, x.width, x.dtype, ld=x.ld)
    kept = torch.full((B.dbw_checkpoint_bytes(shape) + 16,), 201, dtype=torch.uint8, device="cuda")
    B.dbw_checkpoint_store(shape, x.arg, kept, mask=mask)
    assert (kept[-16:] == 201).all()
    return kept[:-16]


def load(B, kept, workers, rows, width, dtype, pad=0, shift=0):
    out = Rows.empty(workers * rows, width, dtype, pad, shift)
    B.dbw_checkpoint_load(B.make_rows(workers, rows, width, dtype, ld_out=width + pad), kept, out.arg)
    return out.result("load")


def same(got, want):
    got, want = got.double(), want.double()
    assert ((got == want) | torch.isnan(got) & torch.isnan(want)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,rows,width,pad,shift", [(1, 1, 1, 0, 0), (2, 3, 31, 1, 1), (1, 5, 32, 0, 0), (3, 4, 33, 0, 3), (2, 7, 100, 5, 2), (1, 65, 1000, 0, 0),
                                                          (2, 9, 4099, 2, 1), (1, 3, 70000, 0, 0)])
def test_stored_and_loaded(B, dtype, workers, rows, width, pad, shift):
    g = torch.Generator().manual_seed(width)
    v = activations(g, workers * rows, width, dtype)
    mask = some(g, workers * rows)
    v[mask == 0] = math.nan
    x = Rows(v, pad, shift)
    kept = store(B, x, workers, mask.cuda())
    want = ref.kept(torch.where(mask[:, None] > 0, v, 0))
    for t in (F32, BF16):
        same(load(B, kept, workers, rows, width, t, pad, shift), want)
    same(load(B, kept, workers, rows, width, F16, pad, shift), want.to(F16))
    # the layout: codes padded with zeros, then exponents
    padded = -(-width // 32) * 32
    n = workers * rows
    codes = kept[:n * padded].view(n, padded).cpu()
    assert (codes[:, width:] == 0).all()
    e = kept[n * padded:].view(n, padded // 32).cpu().double() - 127
    assert torch.equal(e, ref.exponents(torch.where(mask[:, None] > 0, v, 0)))


def test_all_sizes_of_numbers(B):
    """Every exponent of fp32, borders of rounding and of the blocks' range, infinities and NaN among finite numbers."""
    g = torch.Generator().manual_seed(1)
    e = torch.arange(-149, 128).double()
    base = torch.exp2(e)[:, None] * torch.tensor([1.0, 1.0 + 2 ** -23, 1.0625, 1.1875, 1.5, 1.75, 1.75 + 2 ** -20, 1.9375, 2 - 2 ** -23])[None]
    v = (base[:, None] * torch.exp2(-torch.randint(0, 20, (277, 7, 9), generator=g).double()) * (1 + torch.rand(277, 7, 9, generator=g))).reshape(277, -1)
    v = torch.cat([base, v], 1).float().clamp(-3.4028234663852886e38, 3.4028234663852886e38)
    v[:, ::2] *= -1
    v[100, 5], v[101, 6], v[102, 7], v[103] = math.inf, -math.inf, math.nan, math.inf
    x = Rows(v)
    same(load(B, store(B, x, 1), 1, 277, v.shape[1], F32), ref.kept(v))
    for t in (BF16, F16):
        w = v.to(t)
        same(load(B, store(B, Rows(w), 1), 1, 277, v.shape[1], F32), ref.kept(w))


def test_no_rows(B):
    shape = B.make_rows(2, 0, 7, F32)
    none = torch.empty(0, device="cuda")
    B.dbw_checkpoint_store(shape, none, torch.empty(0, dtype=torch.uint8, device="cuda"))


# --------------------------------------------------------------------------- weight gradients

class Layer:
    """dy and a checkpoint; with experts, rows sorted by expert whose input is the tokens'."""

    def __init__(self, B, dtype, workers, rows, width, out, experts=0, k=1, pad=0, shift=0, seed=0, skew=False):
        g = self.g = torch.Generator().manual_seed(seed * 104729 + width * 31 + out)
        self.B, self.n, self.t, self.width, self.out, self.e, self.k = B, workers, rows, width, out, max(experts, 1), k
        x = activations(g, workers * rows, width, BF16)
        self.kept = store(B, Rows(x), workers)
        self.x = ref.kept(x)
        self.start = self.source = None
        r = self.r = rows * k
        if experts:
            expert = torch.randint(-1, experts, (workers * r,), generator=g)
            if skew:                                        # all of one worker's to one expert, none of another's to any
                expert[:r] = experts - 1
                expert[r:2 * r] = -1
            start, _, source = ref.sort(expert.tolist(), workers, experts)
            self.start, self.source = (torch.tensor(v, dtype=torch.int32) for v in (start, source))
        dy = activations(g, workers * r, out, dtype)
        if experts:
            dy[self.source < 0] = math.nan
        self.dy = Rows(dy, pad, shift)
        self.shape = B.make_linear(workers, r, width, out, dtype, experts=self.e, tokens=rows, k=k, ld=out + pad)
        self.work = torch.full((B.dbw_checkpoint_weight_grad_work_bytes(self.shape),), 255, dtype=torch.uint8, device="cuda")
        self.weight_at, count = 3, self.e * out
        self.bias_at = 3 + count * width + 2
        self.ld = self.bias_at + count + 1

    def run(self, bias=True, status=None, source=None, start=None, grads=None):
        if grads is None:
            grads = torch.full((self.n, self.ld), MARK, device="cuda")
        source, start = self.source if source is None else source, self.start if start is None else start
        self.B.dbw_checkpoint_weight_grad(self.shape, self.dy.arg, self.kept, grads, self.work, self.weight_at, self.bias_at if bias else -1,
                                          start=None if start is None else start.cuda(), source=None if source is None else source.cuda(),
                                          status_out=status)
        return grads

    def check(self, grads, bias=True, what=""):
        """A sum of K products: every term's rounding (none, the products being exact, but for operands in parts), and K additions of fp32 at most, each off
        by at most a step, 2 U, of a partial sum."""
        got = grads.cpu()
        count = self.e * self.out
        weight = got[:, self.weight_at:self.weight_at + count * self.width].reshape(self.n, self.e, self.out, self.width)
        biases = got[:, self.bias_at:self.bias_at + count].reshape(self.n, self.e, self.out)
        dy = self.dy.values.double()
        for i in range(self.n):
            for e in range(self.e):
                if self.start is None:
                    a, z = i * self.r, (i + 1) * self.r
                    x = self.x[a:z]
                else:
                    a, z = (self.start[i * (self.e + 1) + e + j].item() for j in (0, 1))
                    x = self.x[self.source[a:z].long() // self.k]
                d = dy[a:z]
                steps = 2 * ref.U * (z - a + 8)
                ref.close(weight[i, e], d.t() @ x, d.t().abs() @ x.abs() * steps, f"{what} weight of worker {i}, layer {e}")
                if bias:
                    ref.close(biases[i, e], d.sum(0), d.abs().sum(0) * steps, f"{what} bias of worker {i}, layer {e}")
        rest = torch.ones_like(got, dtype=torch.bool)
        rest[:, self.weight_at:self.weight_at + count * self.width] = False
        if bias:
            rest[:, self.bias_at:self.bias_at + count] = False
        assert (got[rest] == MARK).all(), what + ": other columns of the gradients were written"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,rows,width,out,pad,shift", [
    (1, 1, 1, 1, 0, 0), (2, 3, 5, 7, 1, 1), (6, 64, 16, 260, 0, 0), (1, 100, 33, 65, 0, 1), (3, 17, 64, 64, 3, 0), (2, 200, 130, 129, 0, 0),
    (1, 1000, 256, 300, 2, 3), (2, 1, 500, 1000, 0, 0), (1, 33, 1000, 40, 0, 0), (1, 4100, 70, 31, 1, 0), (1, 16, 8, 2000, 0, 0)])
def test_weight_gradient(B, dtype, workers, rows, width, out, pad, shift):
    c = Layer(B, dtype, workers, rows, width, out, pad=pad, shift=shift, seed=1)
    c.check(c.run())
    c.check(c.run(bias=False), bias=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,rows,width,out,experts,k,pad", [
    (1, 1, 5, 7, 3, 1, 0), (2, 40, 100, 130, 4, 2, 1), (3, 100, 64, 64, 9, 3, 0), (2, 7, 33, 20, 64, 4, 3), (2, 600, 128, 96, 2, 2, 0), (1, 50, 300, 17, 1, 2, 0)])
@pytest.mark.parametrize("skew", [False, True])
def test_weight_gradient_by_expert(B, dtype, workers, rows, width, out, experts, k, pad, skew):
    workers = max(workers, 2) if skew else workers
    c = Layer(B, dtype, workers, rows, width, out, experts=experts, k=k, pad=pad, seed=2, skew=skew)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.check(c.run(status=status))
    assert status.item() == 0
    # rows sorted by expert and the checkpoint alike
    x = torch.zeros(workers * c.r, width, dtype=BF16)
    live = c.source >= 0
    x[live] = c.x[c.source[live].long() // k].to(BF16)
    moved = store(B, Rows(x), workers)
    shape = B.make_linear(workers, c.r, width, out, dtype, experts=experts, ld=out + pad)
    grads = torch.full((workers, c.ld), MARK, device="cuda")
    B.dbw_checkpoint_weight_grad(shape, c.dy.arg, moved, grads, c.work, c.weight_at, c.bias_at, start=c.start.cuda())
    c.check(grads, what="sorted")


def test_a_single_product(B):
    """One row.  bf16 and fp16 (two parts, 11 + 4 bits in all): exact.  fp32 is three parts h + m + l with |m + l| < 2^-7 |h|: l x goes to zero, exactly,
    m x to that, off by at most a step (2 U) of 2^-7 of the product, h x to that, off by at most a step of the product: less than 2.02 U of it."""
    for dtype in TYPES:
        c = Layer(B, dtype, 2, 1, 200, 150, seed=3)
        got = c.run().cpu()[:, 3:3 + 150 * 200].view(2, 150, 200)
        want = (c.dy.values.double()[:, :, None] * c.x[:, None, :])
        off = (got.double() - want).abs()
        assert (off <= (2.02 * ref.U * want.abs() if dtype is F32 else 0)).all()


def test_large_and_small_numbers_keep_their_size(B):
    for dtype in (F32, BF16):
        c = Layer(B, dtype, 1, 40, 64, 64, seed=4)
        for scale in (2.0 ** 60, 2.0 ** -60):
            c.dy = Rows((c.dy.values.double() * scale).to(dtype))
            c.check(c.run(), what=str(scale))


def test_no_rows_gives_zeros(B):
    shape = B.make_linear(2, 0, 5, 7, F32)
    grads = torch.full((2, 60), MARK, device="cuda")
    work = torch.empty(B.dbw_checkpoint_weight_grad_work_bytes(shape), dtype=torch.uint8, device="cuda")
    B.dbw_checkpoint_weight_grad(shape, torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda"), grads, work, 2, 40)
    want = torch.full_like(grads, MARK)
    want[:, 2:37] = 0
    want[:, 40:47] = 0
    assert torch.equal(grads, want)


def test_offsets_and_sources_out_of_order_are_reported(B):
    """Whatever they hold, nothing outside of the arrays is read."""
    c = Layer(B, BF16, 2, 30, 40, 50, experts=3, k=2, seed=5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = c.run()
    for start in (c.start.flip(0), c.start + 1000, c.start - 1000, torch.full_like(c.start, 2 ** 31 - 1), torch.full_like(c.start, -2 ** 31)):
        status.zero_()
        c.run(start=start.contiguous(), status=status)
        assert status.item() == B.ERR_INVALID
    for source in (c.source + 120, torch.full_like(c.source, 2 ** 31 - 1), torch.full_like(c.source, -5)):
        status.zero_()
        grads = c.run(source=source, status=status)
        assert status.item() == B.ERR_INVALID and torch.isfinite(grads).all()
    assert torch.equal(c.run(), good)


def test_nan_stays_in_its_columns(B):
    c = Layer(B, BF16, 1, 50, 70, 60, seed=6)
    dy = c.dy.values.clone()
    dy[7, 11] = math.nan
    c.dy = Rows(dy)
    got = c.run().cpu()
    weight, bias = got[0, 3:3 + 60 * 70].view(60, 70), got[0, c.bias_at:c.bias_at + 60]
    assert torch.isnan(weight[11]).all() and torch.isnan(weight).sum() == 70 and torch.isnan(bias).sum() == 1 and torch.isnan(bias[11])


@pytest.mark.parametrize("dtype,bits", [(F32, (0x7f800001, -0x7f0001, 0x7fffffff)), (F16, (0x7c01, -0x3ff, 0x7fff)), (BF16, (0x7f81, -0x7f, 0x7fff))])
def test_every_nan_is_one(B, dtype, bits):
    """Also those whose upper bits alone are an infinity's."""
    c = Layer(B, dtype, 1, 40, 33, 70, seed=8)
    dy = c.dy.values.clone()
    for i, b in enumerate(bits):
        dy.view(torch.int32 if dtype == F32 else torch.int16)[5 + i, 20 * i] = b
    assert torch.isnan(dy).sum() == len(bits)
    c.dy = Rows(dy)
    got = c.run().cpu()
    weight, bias = got[0, 3:3 + 70 * 33].view(70, 33), got[0, c.bias_at:c.bias_at + 70]
    for rows in (weight, bias):
        nan = torch.isnan(rows).view(70, -1)
        assert nan[0:60:20].all() and nan.sum() == len(bits) * nan.shape[1]


def test_on_another_stream_captured_and_twice_the_same(B):
    for kw in (dict(), dict(experts=4, k=2)):
        c = Layer(B, BF16, 2, 300, 100, 200, seed=7, **kw)
        grads, start, source = c.run(), c.start, c.source
        torch.cuda.synchronize()
        held = {"start": None if start is None else start.cuda(), "source": None if source is None else source.cuda()}
        again = torch.full_like(grads, MARK)

        def step():
            B.dbw_checkpoint_weight_grad(c.shape, c.dy.arg, c.kept, again, c.work, c.weight_at, c.bias_at, **held)

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            step()
            s.synchronize()
            assert torch.equal(grads, again)
            with torch.cuda.graph(graph, stream=s):
                step()
        for turn in range(3):
            again.fill_(MARK)
            c.work.fill_(turn)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(grads, again)


# --------------------------------------------------------------------------- tiles of every size

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,rows,width,out,experts,k,pad", [
    (64, 40, 256, 256, 4, 2, 0), (32, 70, 300, 270, 0, 1, 1), (3, 100, 4097, 1100, 0, 1, 0), (70, 5, 257, 300, 3, 1, 3),       # a workgroup's tile 256 wide
    (40, 30, 200, 200, 4, 2, 0), (45, 64, 129, 255, 3, 2, 1), (1, 8200, 1000, 1030, 0, 1, 0),                                   # 128 wide; and in parts
    (1, 3000, 512, 200, 0, 1, 0), (2, 2500, 33, 100, 2, 2, 0), (300, 33, 65, 64, 70, 1, 0),          # 64; in parts; more experts than are sorted
    (32, 150, 500, 1024, 0, 1, 1), (64, 300, 250, 256, 4, 2, 0), (30, 280, 500, 1000, 2, 1, 0),                                 # 256 wide, of more rows
    (16, 64, 64, 64, 16, 2, 0), (40, 100, 100, 48, 16, 1, 1), (256, 40, 130, 30, 0, 1, 0)])                                     # many layers within a tile
def test_tiles_of_every_size(B, dtype, workers, rows, width, out, experts, k, pad):
    """Against 64 bits on the GPU, inputs as in Layer: the bound is that of Layer.check()."""
    g = torch.Generator(device="cuda").manual_seed(workers * 7 + width)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    r, e = rows * k, max(experts, 1)
    x = randn(workers * rows, width).to(BF16)
    shape = B.make_rows(workers, rows, width, BF16)
    kept = torch.empty(B.dbw_checkpoint_bytes(shape), dtype=torch.uint8, device="cuda")
    B.dbw_checkpoint_store(shape, x, kept)
    B.dbw_checkpoint_load(shape, kept, x)
    x = x.double()
    flat = torch.full((workers * r, out + pad), math.nan, dtype=dtype, device="cuda")
    flat[:, :out] = randn(workers * r, out).to(dtype)
    start = source = None
    if experts:
        expert = torch.randint(-1, experts, (workers * r,), device="cuda", generator=g).int()
        expert[:k * rows // 2] = experts - 1
        routing = B.make_routing(workers, rows, k, experts)
        start = torch.empty(workers * (experts + 1), dtype=torch.int32, device="cuda")
        place, source = (torch.empty(workers * r, dtype=torch.int32, device="cuda") for _ in range(2))
        B.dbw_expert_sort(routing, expert, start, place, source, torch.empty(B.dbw_expert_work_bytes(routing), dtype=torch.uint8, device="cuda"))
        flat[source < 0] = math.nan
    linear = B.make_linear(workers, r, width, out, dtype, experts=e, tokens=rows, k=k, ld=out + pad)
    work = torch.full((B.dbw_checkpoint_weight_grad_work_bytes(linear),), 255, dtype=torch.uint8, device="cuda")
    count = e * out
    grads = torch.full((workers, count * width + count + 7), MARK, device="cuda")

    def run():
        B.dbw_checkpoint_weight_grad(linear, flat, kept, grads, work, 1, bias_at=count * width + 4, start=start, source=source)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            run()
    for _ in range(2):
        grads.fill_(MARK)
        graph.replay()
        torch.cuda.synchronize()
    replayed = grads.clone()
    grads.fill_(MARK)
    run()
    assert torch.equal(grads, replayed)
    assert (grads[:, 0] == MARK).all() and (grads[:, 1 + count * width:4 + count * width] == MARK).all() and (grads[:, -3:] == MARK).all()
    weight = grads[:, 1:1 + count * width].view(workers, e, out, width)
    bias = grads[:, 4 + count * width:4 + count * width + count].view(workers, e, out)
    starts = start.tolist() if experts else None
    for i in sorted({0, workers // 2, workers - 1}):
        for c in sorted({0, e // 2, e - 1}):
            a, z = starts[i * (e + 1) + c:i * (e + 1) + c + 2] if experts else (i * r, (i + 1) * r)
            d = flat[a:z, :out].double()
            u = x[source[a:z].long() // k] if experts else x[a:z]
            steps = 2 * ref.U * (z - a + 8)
            for got, want, size in ((weight[i, c], d.t().contiguous() @ u, d.t().abs().contiguous() @ u.abs()), (bias[i, c], d.sum(0), d.abs().sum(0))):
                assert ((got.double() - want).abs() <= 1.01 * steps * size + ref.U * want.abs() + 1e-40).all(), (i, c)


def test_a_checkpoint_of_no_tokens_is_reported(B):
    linear = B.make_linear(1, 3, 8, 5, F32, tokens=0)
    grads = torch.full((1, 45), MARK, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dbw_checkpoint_weight_grad(linear, torch.ones(15, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda"), grads,
                                 torch.empty(B.dbw_checkpoint_weight_grad_work_bytes(linear), dtype=torch.uint8, device="cuda"), 0, bias_at=40,
                                 source=torch.zeros(3, dtype=torch.int32, device="cuda"), status_out=status)
    assert (grads == 0).all() and status.item() == B.ERR_INVALID
