"""Tokens sorted by expert and back against layer_reference.py."""
import math

import pytest
import torch

import layer_reference as ref
from layer_inputs import MARK, Rows, activations

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def run_sort(B, expert, workers, tokens, k, experts):
    routing = B.make_routing(workers, tokens, k, experts)
    work = torch.full((B.dbw_expert_work_bytes(routing),), 255, dtype=torch.uint8, device="cuda")
    start = torch.full((workers * (experts + 1) + 1,), -7, dtype=torch.int32, device="cuda")
    place, source = (torch.full((workers * tokens * k + 1,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dbw_expert_sort(routing, expert.int().cuda(), start, place, source, work, status_out=status)
    assert start[-1] == -7 and place[-1] == -7 and source[-1] == -7
    return routing, start[:-1], place[:-1], source[:-1], status.item()


@pytest.mark.parametrize("workers,tokens,k,experts", [(1, 1, 1, 1), (2, 3, 2, 4), (1, 64, 1, 2), (3, 65, 1, 3), (1, 1, 8, 8), (5, 100, 3, 17), (2, 511, 2, 64), (1, 4096, 1, 5),
                                                      (2, 4097, 1, 100), (3, 5000, 2, 16), (1, 20000, 3, 600), (40, 7, 4, 1024), (1, 9000, 1, 1024), (1, 300, 1, 512),
                                                      (1, 300000, 1, 40),                                                       (2, 300, 40, 513)])
@pytest.mark.parametrize("some", ["all", "few", "one", "none"])
def test_sort(B, workers, tokens, k, experts, some):
    g = torch.Generator().manual_seed(tokens * 31 + experts)
    n = workers * tokens * k
    expert = torch.randint(0, experts, (n,), generator=g)
    if some == "few":
        expert = torch.where(torch.rand(n, generator=g) < 0.6, -1 - expert, expert)
    elif some == "one":
        expert[:] = experts - 1
    elif some == "none":
        expert[:] = -3
    _, start, place, source, status = run_sort(B, expert, workers, tokens, k, experts)
    slots = tokens * k
    e = expert.view(workers, slots)
    key = torch.where(e >= 0, e, experts)
    order = key.argsort(dim=1, stable=True)
    counts = torch.stack([torch.bincount(row, minlength=experts + 1)[:experts] for row in key])
    first = torch.arange(workers)[:, None] * slots
    want_start = torch.cat([torch.zeros(workers, 1, dtype=torch.long), counts.cumsum(1)], 1) + first
    there = torch.arange(slots)[None] < counts.sum(1)[:, None]
    want_source = torch.where(there, order + first, -1)
    want_place = torch.empty_like(order).scatter_(1, order, torch.where(there, torch.arange(slots)[None] + first, -1))
    assert torch.equal(start.cpu().long(), want_start.reshape(-1))
    assert torch.equal(source.cpu().long(), want_source.reshape(-1))
    assert torch.equal(place.cpu().long(), want_place.reshape(-1))
    assert status == 0
    if n <= 300:
        assert [start.tolist(), place.tolist(), source.tolist()] == list(ref.sort(expert.tolist(), workers, experts))


def test_experts_that_are_not_there_are_reported(B):
    expert = torch.tensor([0, 5, 2, 4, 2 ** 31 - 1, -2 ** 31])
    _, start, place, source, status = run_sort(B, expert, 1, 3, 2, 4)
    assert status == B.ERR_INVALID
    assert place.tolist() == [0, -1, 1, -1, -1, -1] and source.tolist() == [0, 2, -1, -1, -1, -1] and start.tolist() == [0, 1, 1, 2, 2]


def test_no_tokens(B):
    _, start, _, _, status = run_sort(B, torch.empty(0), 2, 0, 3, 4)
    assert start.tolist() == [0] * 10 and status == 0


class Routed:
    def __init__(self, B, dtype, workers, tokens, width, k, experts, pad=0, shift=0, seed=0, absent=0.3):
        g = self.g = torch.Generator().manual_seed(seed * 6151 + width)
        self.B, self.dtype, self.n, self.t, self.d, self.k = B, dtype, workers, tokens, width, k
        self.total, self.slots, self.pad, self.shift = workers * tokens, workers * tokens * k, pad, shift
        expert = torch.randint(0, experts, (self.slots,), generator=g)
        expert = torch.where(torch.rand(self.slots, generator=g) < absent, -1, expert)
        if self.total > 2:
            expert[k:2 * k] = -1                        # a token of nobody
        start, place, source = ref.sort(expert.tolist(), workers, experts)
        self.place, self.source = torch.tensor(place).view(self.total, k), torch.tensor(source)
        self.place_arg = self.place.reshape(-1).int().cuda()
        self.routing = B.make_routing(workers, tokens, k, experts)
        self.shape = B.make_rows(workers, tokens, width, dtype, ld=width + pad, ld_out=width + 2 * pad)
        self.x = Rows(activations(g, self.total, width, dtype), pad, shift)
        z = activations(g, self.slots, width, dtype)
        z[self.source < 0] = math.nan
        self.z = Rows(z, 2 * pad, shift)
        self.weights = torch.where(self.place >= 0, torch.randn(self.total, k, generator=g), math.nan)
        self.weights_arg = self.weights.cuda()
        self.mine = self.source >= 0

    def sorted(self):
        return Rows.empty(self.slots, self.d, self.dtype, 2 * self.pad, self.shift)

    def tokens(self):
        return Rows.empty(self.total, self.d, self.dtype, self.pad, self.shift)


SHAPES = [(1, 1, 1, 1, 1, 0, 0), (2, 3, 5, 2, 4, 1, 1), (1, 9, 64, 3, 3, 0, 0), (3, 20, 100, 2, 7, 3, 2), (4, 1, 2048, 4, 64, 0, 0), (2, 50, 1001, 1, 5, 0, 0),
          (1, 7, 5000, 8, 16, 0, 1), (2, 130, 257, 2, 9, 0, 0), (1, 3, 40000, 2, 2, 1, 0), (1, 2, 16, 70, 8, 0, 0), (1, 600, 8, 5, 3, 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,tokens,width,k,experts,pad,shift", SHAPES)
def test_gather_and_combine(B, dtype, workers, tokens, width, k, experts, pad, shift):
    c = Routed(B, dtype, workers, tokens, width, k, experts, pad, shift, seed=1)
    out = c.sorted()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dbw_expert_gather(c.routing, c.shape, c.x.arg, c.place_arg, out.arg, status_out=status)
    got = out.result("gather")
    assert torch.equal(got[c.mine], c.x.values[c.source[c.mine] // k]) and (got[~c.mine] == MARK).all()
    for weights in (c.weights, None):
        y = c.tokens()
        B.dbw_expert_combine(c.routing, c.shape, c.z.arg, c.place_arg, y.arg, weights=None if weights is None else c.weights_arg, status_out=status)
        want, size = ref.combine(c.z.values.double(), c.place, None if weights is None else weights.double())
        ref.close(y.result("combine"), want, size * ref.U * (k + 1), "combine", dtype)
    assert status.item() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("workers,tokens,width,k,experts,pad,shift", SHAPES)
def test_gradient(B, dtype, workers, tokens, width, k, experts, pad, shift):
    c = Routed(B, dtype, workers, tokens, width, k, experts, pad, shift, seed=2)
    for weights, wanted, in_place in [(True, True, False), (True, True, True), (True, False, False), (False, True, False)]:
        dz = Rows(c.z.values, 2 * pad, shift) if in_place else c.sorted()
        dw = torch.full((c.slots + 1,), MARK, device="cuda")
        B.dbw_expert_combine_grad(c.routing, c.shape, c.x.arg, dz.arg if in_place else (c.z.arg if wanted else None), c.place_arg, dz.arg,
                                  weights=c.weights_arg if weights else None, dweights=dw if wanted else None)
        got = dz.result("gradient")
        token = c.source[c.mine] // k
        w = c.weights.reshape(-1)[c.source[c.mine]].double()[:, None] if weights else 1.0
        want = c.x.values[token].double() * w
        ref.close(got[c.mine], want, want.abs() * ref.U, "rows", dtype)
        assert (torch.isnan(got[~c.mine]) if in_place else got[~c.mine] == MARK).all()
        if wanted:
            on = (c.place >= 0)[..., None]
            terms = torch.where(on, c.x.values.double()[:, None] * c.z.values.double()[c.place.clamp(min=0)], 0.0)
            ref.close(dw[:-1], terms.sum(2).reshape(-1), terms.abs().sum(2).reshape(-1) * ref.U * (ref.depth(width) + width // 64), "weights")
            assert (dw[:-1].cpu()[c.place.reshape(-1) < 0] == 0).all() and dw[-1] == MARK


def test_the_gradient_is_that_of_differences(B):
    """fp32 rows of small numbers: combine() is linear in the rows and in the weights, so that differences are exact but for rounding."""
    c = Routed(B, F32, 2, 4, 20, 2, 3, seed=3)
    dy = activations(c.g, c.total, 20, F32).cuda()
    dz, dw = c.sorted(), torch.empty(c.slots, device="cuda")
    B.dbw_expert_combine_grad(c.routing, c.shape, dy, c.z.arg, c.place_arg, dz.arg, weights=c.weights_arg, dweights=dw)

    def loss(z, weights):
        y = c.tokens()
        B.dbw_expert_combine(c.routing, c.shape, z.arg, c.place_arg, y.arg, weights=weights)
        return (y.result().double() * dy.cpu().double()).sum().item()

    size = ref.combine(c.z.values.double(), c.place, c.weights.double())[1]
    noise = 4 * ref.U * 3 * (size * dy.cpu().double().abs()).sum().item()
    at = loss(c.z, c.weights_arg)
    for slot in range(c.slots):
        p = c.place.reshape(-1)[slot].item()
        if p < 0:
            continue
        w = c.weights.clone().reshape(-1)
        w[slot] += 1
        assert abs(loss(c.z, w.view_as(c.weights).cuda()) - at - dw[slot].item()) <= noise + 30 * ref.U * abs(dw[slot].item()) + 1e-4
        z = c.z.values.clone()
        z[p, 3] += 1
        assert abs(loss(Rows(z), c.weights_arg) - at - dz.result()[p, 3].item()) <= noise + 1e-4


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_gathers_gradient_is_the_sum_of_a_tokens_rows(B, dtype):
    c = Routed(B, dtype, 2, 30, 200, 3, 5, seed=4)
    dx = c.tokens()
    B.dbw_expert_combine(c.routing, c.shape, c.z.arg, c.place_arg, dx.arg)
    want = torch.zeros(c.total, 200, dtype=torch.float64).index_add_(0, c.source[c.mine] // 3, c.z.values[c.mine].double())
    size = torch.zeros(c.total, 200, dtype=torch.float64).index_add_(0, c.source[c.mine] // 3, c.z.values[c.mine].double().abs())
    ref.close(dx.result(), want, size * ref.U * 4, "dx", dtype)


def test_places_that_are_none_are_reported(B):
    """Whatever they hold, nothing outside of the arrays is read or written."""
    c = Routed(B, BF16, 2, 10, 50, 2, 3, seed=5, absent=0.0)
    good = c.place_arg.clone()
    for bad in (20, 2 ** 31 - 1, 40, 25):                   # of the other worker, or of nobody
        place = good.clone()
        place[0] = bad
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, y, dz, dw = c.sorted(), c.tokens(), c.sorted(), torch.full((c.slots,), MARK, device="cuda")
        B.dbw_expert_gather(c.routing, c.shape, c.x.arg, place, out.arg, status_out=status)
        assert status.item() == B.ERR_INVALID
        got = out.result()
        assert (got[good[0].item()] == MARK).all() and (got[20:][c.mine[20:]] != MARK).any(1).all()
        status.zero_()
        B.dbw_expert_combine(c.routing, c.shape, c.z.arg, place, y.arg, weights=c.weights_arg, status_out=status)
        y.result()
        assert status.item() == B.ERR_INVALID
        status.zero_()
        B.dbw_expert_combine_grad(c.routing, c.shape, c.x.arg, c.z.arg, place, dz.arg, weights=c.weights_arg, dweights=dw, status_out=status)
        dz.result()
        assert status.item() == B.ERR_INVALID and dw[0] == 0


def test_sorted_gathered_and_combined_in_a_graph(B):
    """All of a step, captured once and replayed with other experts, beside an eager one."""
    workers, tokens, width, k, experts = 2, 3000, 64, 2, 10
    g = torch.Generator().manual_seed(6)
    routing, shape = B.make_routing(workers, tokens, k, experts), B.make_rows(workers, tokens, width, BF16)
    slots = workers * tokens * k
    work = torch.empty(B.dbw_expert_work_bytes(routing), dtype=torch.uint8, device="cuda")
    expert = torch.zeros(slots, dtype=torch.int32, device="cuda")
    start = torch.empty(workers * (experts + 1), dtype=torch.int32, device="cuda")
    place, source = (torch.empty(slots, dtype=torch.int32, device="cuda") for _ in range(2))
    x = activations(g, workers * tokens, width, BF16).cuda()
    weights = torch.rand(slots, generator=g).cuda()
    rows, drows = (torch.zeros(slots, width, dtype=BF16, device="cuda") for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dw = torch.empty_like(weights)

    def step():
        B.dbw_expert_sort(routing, expert, start, place, source, work)
        B.dbw_expert_gather(routing, shape, x, place, rows)
        B.dbw_expert_combine(routing, shape, rows, place, y, weights=weights)
        B.dbw_expert_combine_grad(routing, shape, y, rows, place, drows, weights=weights, dweights=dw)
        B.dbw_expert_combine(routing, shape, drows, place, dx)
        return start, place, source, rows, y, drows, dw, dx

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            step()
    for turn in range(3):
        expert.copy_(torch.randint(-1, experts, (slots,), generator=g).int())
        rows.zero_()
        drows.zero_()
        work.fill_(turn)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (start, place, source, rows, y, drows, dw, dx)]
        rows.zero_()
        drows.zero_()
        work.fill_(99)
        again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        total = torch.zeros(workers * tokens, device="cuda").index_add_(0, torch.arange(slots, device="cuda") // k, torch.where(expert >= 0, weights, 0.0))
        assert torch.allclose(y.float(), x.float() * total[:, None], rtol=2 ** -7, atol=1e-6)
