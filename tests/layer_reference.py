"""What dbw_layers.h defines, in 64 bits on the CPU, and how far fp32 arithmetic may be off from it.

Bounds count roundings: U = 2^-24 is half a step of fp32 relative to the value, a sum of n terms by any tree of depth G is off by at most G U times the
sum of the terms' magnitudes (to first order; the factor 1.01 in close() covers the rest), and the one rounding to an array's type by HALF of the
value, or half the smallest subnormal."""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
BLOCK = 32


def depth(width):
    """Additions on a term's way to a row's sum: up to 64 of a thread's own, lanes and waves; behind 16384 columns pieces one after the other as well."""
    return 96 + width // 2048


def close(got, want, bound, what="", dtype=torch.float32):
    got, want = got.detach().cpu().double(), want.double()
    bound = bound * 1.01 + HALF[dtype] * (want.abs() + bound) + TINY[dtype]
    both = torch.isnan(got) & torch.isnan(want) | (got == want)
    bad = ~(both | ((got - want).abs() <= bound))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} elements, first at {bad.nonzero()[0].tolist()}: {got[bad][0].item()} for "
                           f"{want[bad][0].item()}, bound {bound.expand_as(got)[bad][0].item():.3g}")


# --------------------------------------------------------------------------- 8 bits

def exponents(x):
    """Of the blocks of rows [n, width]: the smallest e >= -117 with all finite magnitudes at most 448 2^e."""
    n, width = x.shape
    p = torch.zeros(n, -(-width // BLOCK) * BLOCK, dtype=torch.float64)
    p[:, :width] = torch.where(torch.isfinite(x), x.double(), 0.0)
    top = p.view(n, -1, BLOCK).abs().amax(2)
    e = torch.full_like(top, -117.0)
    for step in range(-117, 121):
        e = torch.where(top > 448 * 2.0 ** (step - 1), torch.tensor(float(step), dtype=torch.float64), e)
    return e.clamp(max=120)


def kept(x):
    """What rows in 8 bits stand for."""
    n, width = x.shape
    by = torch.exp2(exponents(x)).repeat_interleave(BLOCK, 1)[:, :width]
    q = x.double() / by
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.round(q / step) * step
    q = torch.where(by == 2.0 ** 120, q.clamp(-240, 240), q)
    return torch.where(torch.isfinite(x), q * by, float("nan"))


# --------------------------------------------------------------------------- layer norm

def norm(x, w, b, eps):
    """Rows in 64 bits, [.., width]: y, mu, rho."""
    mu = x.mean(-1, keepdim=True)
    rho = 1 / torch.sqrt((x - mu).square().mean(-1, keepdim=True) + eps)
    return (x - mu) * rho * w + b, mu, rho


def norm_bounds(x, w, b, eps):
    """Of y, mu and rho.  The mean is found to G U of the magnitudes' mean; what that leaves is found again from the differences, whose
    rounding counts relative to them."""
    g = depth(x.shape[-1])
    y, mu, rho = norm(x, w, b, eps)
    d = (x - mu).abs()
    first = (g + 2) * U * x.abs().mean(-1, keepdim=True)
    off = 4 * U * (d + first) + (g + 2) * U * (d.mean(-1, keepdim=True) + first)
    variance = d.square().mean(-1, keepdim=True)
    relative = (g + 8) * U * (variance + first.square()) / (variance + eps) / 2 + 4 * U
    return w.abs() * rho * (off + d * relative) + 4 * U * ((w * d * rho).abs() + b.abs()), off.amax(-1, keepdim=True) + 2 * U * mu.abs(), rho * relative


def norm_grad(dy, x, w, mu, rho):
    """dx, and the rows' terms of dw and db.  With mu and rho of x itself this is the gradient of norm()."""
    u = (x - mu) * rho
    g = dy * w
    return rho * (g - g.mean(-1, keepdim=True) - u * (g * u).mean(-1, keepdim=True)), dy * u, dy


def norm_grad_bound(dy, x, w, mu, rho):
    k = depth(x.shape[-1])
    u = ((x - mu) * rho).abs()
    g = (dy * w).abs()
    s0, s1 = g.mean(-1, keepdim=True), (g * u).mean(-1, keepdim=True)
    return rho * U * (6 * (g + s0 + u * s1) + (k + 4) * s0 + u * (k + 8) * s1)


# --------------------------------------------------------------------------- experts

def sort(expert, workers, experts):
    """expert: list of N T k numbers.  start, place, source as lists."""
    slots = len(expert) // workers
    start, place, source = [], [-1] * len(expert), [-1] * len(expert)
    for i in range(workers):
        at = i * slots
        for e in range(experts):
            start.append(at)
            for s in range(i * slots, (i + 1) * slots):
                if expert[s] == e:
                    place[s], source[at] = at, s
                    at += 1
        start.append(at)
    return start, place, source


def combine(z, place, weights):
    """z [rows, width], place and weights [tokens, k], weights possibly None: y and the sum of the terms' magnitudes."""
    on = (place >= 0)[..., None]
    terms = torch.where(on, z[place.clamp(min=0)], 0.0)
    if weights is not None:
        terms = torch.where(on, terms * weights[..., None], 0.0)
    return terms.sum(1), terms.abs().sum(1)
