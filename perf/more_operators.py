"""Performance cases of what lies between the dense products of a language model, of all simulated workers at once: layer norm with its
gradients, activations kept in 8 bits for the backward pass, and tokens sorted by expert and back.

A state holds what a program has before the call.  One pass is one operator, or the few that such a program calls one after the other:

  norm          layer norm, every worker with its own weights (scoring, and serving a token at a time)
  norm_step     the same, keeping its input in 8 bits, then its backward pass from what was kept
  checkpoint    rows put into 8 bits and taken out again
  weight_grad   the weight and bias gradient of a linear layer whose input was kept in 8 bits; with experts the rows come sorted by expert
                and the input is the tokens' before sorting
  experts       slots of tokens sorted by expert, the tokens' rows brought into that order, the experts' results added up with weights
  experts_grad  the gradients of that: of the experts' results and the weights, and of the tokens' rows

A case is a dict of plain values; listed() holds the ones that are looked at by name, draw() makes others of the same ranges.
prepare() makes the inputs, run() is one pass (the plain form, or the library's kernels where `own` is true), exact() the same
results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

OPS = ("norm", "norm_step", "checkpoint", "weight_grad", "experts", "experts_grad")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

# rows:     token positions of each worker;  width: columns of a row (of a linear layer's input)
# left_out: rows of each worker that take no part (prompt and padding positions, tokens that go to no expert)
# pad:      elements between the end of a row and the next one's start
# out:      width of a linear layer's output;  experts, k: experts of each worker and how many of them a token goes to
_BASE = {"op": "norm", "type": "bf16", "workers": 1, "rows": 1, "width": 1024, "pad": 0, "left_out": 0, "out": 0, "experts": 0, "k": 0}


def _case(name=None, **kw):
    assert set(kw) <= set(_BASE), kw
    c = {**_BASE, **kw}
    if name is not None:
        c["name"] = name
    return c


# --------------------------------------------------------------------------- the cases

def listed():
    return [
        # Serving: the one token just sampled.  Latency is all there is.
        _case("norm-one-token", width=4096),
        # Prompts of four models.
        _case("norm-rows", workers=4, rows=2048, width=4096, left_out=200),
        # The smallest training step: single precision, rows of a few columns.
        _case("norm-step-small", op="norm_step", type="f32", workers=16, rows=64, width=16),
        # An ordinary step of eight workers.
        _case("norm-step", op="norm_step", workers=8, rows=2048, width=2048, left_out=100),
        # Half precision, rows of an odd length with a gap between them, so that hardly any starts on a boundary that a wide access likes.
        _case("norm-step-odd-rows", op="norm_step", type="f16", workers=3, rows=1501, width=1001, pad=13, left_out=33),
        # A layer's activations put aside and taken back.
        _case("checkpoint-rows", op="checkpoint", workers=4, rows=4096, width=4096),
        # The output layer of a model on bytes and four marks.
        _case("weight-grad-small", op="weight_grad", type="f32", workers=6, rows=64, width=16, out=260),
        # A square layer of four workers on a long batch.
        _case("weight-grad-dense", op="weight_grad", workers=4, rows=4096, width=2048, out=2048),
        # The first layer of eight experts, two a token; the groups are ragged.
        _case("weight-grad-experts", op="weight_grad", workers=2, rows=4096, width=1024, out=2048, experts=8, k=2, left_out=111),
        # Serving: one token of each of four workers to four of its experts.
        _case("experts-one-token", op="experts", workers=4, rows=1, width=2048, experts=64, k=4),
        # An ordinary step, forwards and backwards.
        _case("experts-rows", op="experts", workers=4, rows=4096, width=2048, experts=16, k=2, left_out=100),
        _case("experts-grad-rows", op="experts_grad", workers=4, rows=4096, width=2048, experts=16, k=2, left_out=100),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    op = rng.choice(OPS)
    kind = rng.choice(("f32", "bf16", "bf16", "f16"))
    width = _log_uniform(rng, 16, 8192)
    width = width | 1 if rng.random() < 0.5 else max(16, width // 16 * 16)     # odd ones, and rows on 16-byte boundaries
    c = _case(op=op, type=kind, workers=_log_uniform(rng, 1, 32), rows=_log_uniform(rng, 1, 8192), width=width,
              pad=rng.choice((0, 0, 0, 1, 8, 13)))
    if op == "weight_grad":
        c["out"] = _log_uniform(rng, 16, 4096)
        if rng.random() < 0.5:
            c["out"] = max(16, c["out"] // 16 * 16)
    if op in ("experts", "experts_grad") or (op == "weight_grad" and rng.random() < 0.5):
        c["experts"] = _log_uniform(rng, 2, 64)
        c["k"] = rng.randint(1, min(8, c["experts"]))
    most = max(_cost(x) for x in listed()) / 2
    while c["rows"] > 1 and _cost(c) > most:
        c["rows"] = (c["rows"] + 1) // 2
    while c["workers"] > 1 and _cost(c) > most:
        c["workers"] = (c["workers"] + 1) // 2
    while c["out"] > 16 and _cost(c) > most:
        c["out"] = (c["out"] + 1) // 2
    if op not in ("checkpoint",) and not (op == "weight_grad" and not c["experts"]):
        c["left_out"] = rng.randint(0, c["rows"] // 3)
    return c


# --------------------------------------------------------------------------- inputs

EPS = 1e-5
BLOCK = 32            # columns that share a power of two


def _padded(width):
    return -(-width // BLOCK) * BLOCK


def _power(e):
    """2^e as a 32-bit number."""
    return ((e + 127) << 23).view(torch.float32)


def _quantised(x):
    """Rows in 8 bits: codes (e4m3) [rows, padded] and exponents [rows, blocks].  A block's power of two is the smallest
    with which its largest value is within 448, the format's largest, and at least 2^-117."""
    rows, width = x.shape
    p = torch.zeros(rows, _padded(width), device=x.device, dtype=torch.float32)
    p[:, :width] = x.float()
    p = p.view(rows, -1, BLOCK)
    top = p.abs().amax(2).view(torch.int32)                       # 1.75 2^8 is 448
    e = ((top >> 23) - 127 - 8 + ((top & 0x7fffff) > 0x600000)).clamp(-117, 120).int()
    codes = (p * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(rows, -1), e


def _values(codes, e, width):
    """What they stand for, in 32 bits."""
    rows = codes.shape[0]
    return (codes.float().view(rows, -1, BLOCK) * _power(e)[..., None]).view(rows, -1)[:, :width]


def _buffer(codes, e):
    """As the library keeps them: the codes of all rows, then a byte for each block, its exponent plus 127."""
    return torch.cat([codes.view(torch.uint8).reshape(-1), (e + 127).to(torch.uint8).reshape(-1)])


def _from_buffer(buffer, rows, width):
    cut = rows * _padded(width)
    return buffer[:cut].view(torch.float8_e4m3fn).view(rows, -1), buffer[cut:].view(rows, -1).int() - 127


def _sorted_by_expert(expert, experts):
    """expert [N, T k], -1: none.  First row of every expert (and the end) [N, E + 1], the row of every slot (-1: none) and the slot of every
    row (-1: none), each worker's rows from its own first slot's number on; slots of one expert keep their order."""
    n, slots = expert.shape
    dev = expert.device
    key = torch.where(expert >= 0, expert, experts)
    order = key.argsort(dim=1, stable=True)
    first = torch.arange(n, device=dev)[:, None] * slots
    counts = (key[:, :, None] == torch.arange(experts, device=dev)).sum(1)
    start = torch.cat([torch.zeros(n, 1, dtype=counts.dtype, device=dev), counts.cumsum(1)], 1)
    position = torch.arange(slots, device=dev).expand(n, slots)
    there = position < start[:, -1:]
    source = torch.where(there, order + first, -1)
    place = torch.empty_like(order).scatter_(1, order, torch.where(there, position + first, -1))
    return (start + first).int(), place.reshape(-1).int(), source.reshape(-1).int()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    op, n, t, width, k, experts = (case[v] for v in ("op", "workers", "rows", "width", "k", "experts"))
    rows, ld, kind = n * t, width + case["pad"], TYPES[case["type"]]

    def rand(*size):
        return torch.rand(*size, device=dev, generator=g)

    def normal(*size):
        return torch.randn(*size, device=dev, generator=g)

    def activations(count, columns, stride, spread=1.0):
        """Rows of a residual stream: every row of its own size, a few columns much larger than the others."""
        flat = torch.zeros(count, stride, device=dev, dtype=kind)
        x = flat[:, :columns]
        x.copy_(normal(count, columns).mul_(normal(count, 1).exp_()).mul_(spread))
        loud = torch.randint(0, columns, (max(1, columns // 256),), device=dev, generator=g)
        x[:, loud] *= 16
        return flat

    live = torch.ones(n, t, dtype=torch.bool, device=dev)
    live.scatter_(1, rand(n, t).argsort(1)[:, :case["left_out"]], False)
    live = live.reshape(rows)
    s = {"case": dict(case), "live": live}
    if op in ("norm", "norm_step"):
        s["x"] = activations(rows, width, ld)
        s["x"][~live] = math.nan                                # nobody filled in the rest
        # weights and biases in every worker's row of parameters, behind 5 others
        s["params"] = torch.zeros(n, 2 * width + 64, device=dev)
        s["params"][:, 5:5 + width] = 1 + 0.2 * normal(n, width)
        s["params"][:, 5 + width:5 + 2 * width] = 0.1 * normal(n, width)
        s["mask"] = live.to(torch.uint8) if case["left_out"] else None
        if op == "norm_step":
            s["dy"] = activations(rows, width, ld, 0.01)
            s["dy"][~live] = math.nan
    elif op == "checkpoint":
        s["x"] = activations(rows, width, ld)
    elif op == "weight_grad":
        out = case["out"]
        s["checkpoint"] = _buffer(*_quantised(activations(rows, width, width)))
        if experts:
            expert = _choices(rand, live, n, t, k, experts)
            s["start"], _, s["source"] = _sorted_by_expert(expert, experts)
            s["dy"] = activations(rows * k, out, out + case["pad"], 0.01)
            s["dy"][s["source"] < 0] = math.nan
            s["most"] = int((s["start"][:, 1:] - s["start"][:, :-1]).max())      # what a padded product needs
        else:
            s["dy"] = activations(rows, out, out + case["pad"], 0.01)
    else:
        expert = _choices(rand, live, n, t, k, experts)
        s["weights"] = torch.softmax(normal(rows, k), 1)
        start, place, source = _sorted_by_expert(expert, experts)
        s["z"] = activations(rows * k, width, ld)
        s["z"][source < 0] = math.nan
        if op == "experts":
            s["expert"] = expert.reshape(-1).int()
            s["x"] = activations(rows, width, ld)
        else:
            s["place"], s["source"] = place, source
            s["dy"] = activations(rows, width, ld, 0.01)
            s["dsorted"] = activations(rows * k, width, ld, 0.01)
            s["dsorted"][source < 0] = math.nan
    if own:
        _prepare_own(s)
    return s


def _choices(rand, live, n, t, k, experts):
    """k different experts of each token, some of them far more popular than others; -1 where a token takes no part."""
    liking = torch.linspace(0, 1.5, experts, device=live.device)
    chosen = (rand(n * t, experts).clamp(1e-6, 1 - 1e-6).log().neg().log().neg() + liking).topk(k, 1).indices
    return torch.where(live[:, None], chosen, -1).reshape(n, t * k)


def _prepare_own(s):
    """Descriptions, outputs and scratch memory, which a program keeps."""
    from paper_2102_06280_amd import binding as B
    c = s["case"]
    op, n, t, width, k, experts = (c[v] for v in ("op", "workers", "rows", "width", "k", "experts"))
    rows, ld, kind = n * t, width + c["pad"], TYPES[c["type"]]
    dev = s["live"].device

    def empty(count):
        return torch.zeros(count, width, dtype=kind, device=dev)

    if op == "weight_grad":
        out = c["out"]
        s["shape"] = B.make_linear(n, t * max(k, 1), width, out, kind, experts=max(experts, 1), tokens=t, k=max(k, 1), ld=out + c["pad"])
        s["grads"] = torch.zeros(n, max(experts, 1) * out * (width + 1), device=dev)
        s["work"] = torch.empty(B.dbw_checkpoint_weight_grad_work_bytes(s["shape"]), dtype=torch.uint8, device=dev)
        return
    s["shape"] = B.make_rows(n, t, width, kind, ld=ld, ld_out=width)
    if op in ("norm", "norm_step"):
        s["y"], s["stats"] = empty(rows), torch.zeros(rows, 2, device=dev)
        if op == "norm_step":
            s["kept"] = torch.empty(B.dbw_checkpoint_bytes(s["shape"]), dtype=torch.uint8, device=dev)
            s["dx"], s["grads"] = torch.zeros_like(s["x"]), torch.zeros_like(s["params"])
            s["back"] = B.make_rows(n, t, width, kind, ld=ld, ld_out=ld)
            s["work"] = torch.empty(B.dbw_layer_norm_work_bytes(s["back"]), dtype=torch.uint8, device=dev)
    elif op == "checkpoint":
        s["kept"] = torch.empty(B.dbw_checkpoint_bytes(s["shape"]), dtype=torch.uint8, device=dev)
        s["y"] = empty(rows)
    else:
        s["routing"] = B.make_routing(n, t, k, experts)
        if op == "experts":
            s["work"] = torch.empty(B.dbw_expert_work_bytes(s["routing"]), dtype=torch.uint8, device=dev)
            s["start"] = torch.empty(n * (experts + 1), dtype=torch.int32, device=dev)
            s["place"], s["source"] = (torch.empty(rows * k, dtype=torch.int32, device=dev) for _ in range(2))
            s["y"] = torch.zeros_like(s["x"])
            s["sorted"] = torch.zeros_like(s["z"])
        else:
            s["dz"], s["dx"] = torch.zeros_like(s["z"]), torch.zeros_like(s["dy"])
            s["dweights"] = torch.empty(rows * k, device=dev)
        s["shape"] = B.make_rows(n, t, width, kind, ld=ld, ld_out=ld)


# --------------------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2102_06280_amd import binding as B
    c = s["case"]
    op, width = c["op"], c["width"]
    at = {"weight_at": 5, "bias_at": 5 + width}
    if op == "norm":
        B.dbw_layer_norm(s["shape"], s["x"], s["params"], s["y"], eps=EPS, mask=s["mask"], stats_out=s["stats"], **at)
        return {"y": s["y"], "stats": s["stats"]}
    if op == "norm_step":
        B.dbw_layer_norm(s["shape"], s["x"], s["params"], s["y"], eps=EPS, mask=s["mask"], stats_out=s["stats"], checkpoint=s["kept"], **at)
        B.dbw_layer_norm_grad(s["back"], s["dy"], None, s["stats"], s["params"], s["dx"], s["grads"], s["work"], mask=s["mask"],
                              checkpoint=s["kept"], **at)
        return {"y": s["y"], "stats": s["stats"], "dx": s["dx"][:, :width], "grads": s["grads"][:, 5:5 + 2 * width]}
    if op == "checkpoint":
        B.dbw_checkpoint_store(s["shape"], s["x"], s["kept"])
        B.dbw_checkpoint_load(s["shape"], s["kept"], s["y"])
        return {"y": s["y"]}
    if op == "weight_grad":
        cut = max(c["experts"], 1) * c["out"] * width
        B.dbw_checkpoint_weight_grad(s["shape"], s["dy"], s["checkpoint"], s["grads"], s["work"], weight_at=0, bias_at=cut,
                                     start=s.get("start"), source=s.get("source"))
        return {"weight": s["grads"][:, :cut], "bias": s["grads"][:, cut:]}
    if op == "experts":
        B.dbw_expert_sort(s["routing"], s["expert"], s["start"], s["place"], s["source"], s["work"])
        B.dbw_expert_gather(s["routing"], s["shape"], s["x"], s["place"], s["sorted"])
        B.dbw_expert_combine(s["routing"], s["shape"], s["z"], s["place"], s["y"], weights=s["weights"])
        return {"start": s["start"], "place": s["place"], "source": s["source"], "sorted": s["sorted"][:, :width], "y": s["y"][:, :width]}
    B.dbw_expert_combine_grad(s["routing"], s["shape"], s["dy"], s["z"], s["place"], s["dz"], weights=s["weights"], dweights=s["dweights"])
    B.dbw_expert_combine(s["routing"], s["shape"], s["dsorted"], s["place"], s["dx"])
    return {"dz": s["dz"][:, :width], "dweights": s["dweights"], "dx": s["dx"][:, :width]}


def _run_plain(s):
    c = s["case"]
    op, n, t, width, k, experts = (c[v] for v in ("op", "workers", "rows", "width", "k", "experts"))
    rows, live, kind = n * t, s["live"], TYPES[c["type"]]
    if op in ("norm", "norm_step"):
        on = live[:, None]
        w, b = (s["params"][:, a:a + width].repeat_interleave(t, 0) for a in (5, 5 + width))
        x = s["x"][:, :width].float()
        mean = x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = torch.where(on, (x - mean) * rstd * w + b, 0.0).to(kind)
        out = {"y": y, "stats": torch.where(on, torch.cat([mean, rstd], 1), 0.0)}
        if op == "norm_step":
            unit = torch.where(on, (_values(*_quantised(x), width) - mean) * rstd, 0.0)
            dy = torch.where(on, s["dy"][:, :width].float(), 0.0)
            d = dy * w
            dx = (d - d.mean(1, keepdim=True) - unit * (d * unit).mean(1, keepdim=True)) * rstd
            out["dx"] = torch.where(on, dx, 0.0).to(kind)
            out["grads"] = torch.cat([(dy * unit).view(n, t, width).sum(1), dy.view(n, t, width).sum(1)], 1)
        return out
    if op == "checkpoint":
        return {"y": _values(*_quantised(s["x"][:, :width]), width).to(kind)}
    if op == "weight_grad":
        out = c["out"]
        x = _values(*_from_buffer(s["checkpoint"], rows, width), width)
        dy = s["dy"][:, :out].float()
        if not experts:
            dy = dy.view(n, t, out)
            return {"weight": torch.bmm(dy.transpose(1, 2).contiguous(), x.reshape(n, t, width)).view(n, -1), "bias": dy.sum(1)}
        # groups padded to the longest one's length
        start, source = s["start"].long(), s["source"].long()
        first, end = start[:, :-1].reshape(-1, 1), start[:, 1:].reshape(-1, 1)
        row = first + torch.arange(s["most"], device=dy.device)
        there, row = (row < end)[..., None], row.clamp(max=rows * k - 1)
        d = torch.where(there, dy[row], 0.0)
        u = torch.where(there, x[(source[row] // k).clamp(min=0)], 0.0)
        weight = torch.bmm(d.transpose(1, 2).contiguous(), u)
        return {"weight": weight.view(n, -1), "bias": d.sum(1).view(n, -1)}
    out = {}
    if op == "experts":
        start, place, source = _sorted_by_expert(s["expert"].view(n, t * k), experts)
        there = (source >= 0)[:, None]
        out = {"start": start.view(-1), "place": place, "source": source,
               "sorted": torch.where(there, s["x"][:, :width][(source.long() // k).clamp(min=0)], 0.0)}
    else:
        place, source = s["place"], s["source"]
    at = place.long().view(rows, k).clamp(min=0)
    on = (place >= 0).view(rows, k, 1)
    z = torch.where(on, s["z"][:, :width][at].float(), 0.0)
    if op == "experts":
        out["y"] = (z * s["weights"][:, :, None]).sum(1).to(kind)
        return out
    dy = s["dy"][:, :width].float()
    out["dweights"] = (z * dy[:, None]).sum(2).view(-1)
    slot = source.long().clamp(min=0)
    out["dz"] = torch.where((source >= 0)[:, None], dy[slot // k] * s["weights"].view(-1)[slot][:, None], 0.0).to(kind)
    out["dx"] = torch.where(on, s["dsorted"][:, :width][at].float(), 0.0).sum(1).to(kind)
    return out


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size, op = SIZE[case["type"]], case["op"]
    n, t, width, k, experts = (case[v] for v in ("workers", "rows", "width", "k", "experts"))
    rows, live = n * t, n * (t - case["left_out"])
    kept = _padded(width) + _padded(width) // BLOCK              # bytes of a row in 8 bits
    if op in ("norm", "norm_step"):
        bytes_ = live * width * size + rows * (width * size + 8) + n * width * 8
        flops = live * width * 8
        if op == "norm_step":
            bytes_ += 2 * live * kept + live * width * size + rows * width * size + live * 8 + n * width * 12
            flops += live * width * 20
        return {"bytes": bytes_ + (rows if case["left_out"] else 0), "flops": flops}
    if op == "checkpoint":
        return {"bytes": 2 * rows * (width * size + kept), "flops": rows * width * 4}
    if op == "weight_grad":
        out, groups, used = case["out"], n * max(experts, 1), live * max(k, 1)
        return {"bytes": used * out * size + live * kept + groups * out * (width + 1) * 4 + (used * 4 + groups * 4 if experts else 0),
                "flops": 2 * used * out * (width + 1)}
    used = live * k
    if op == "experts":
        return {"bytes": rows * k * 16 + n * (experts + 1) * 4 + (live + used) * width * size + (used + rows) * width * size,
                "flops": 2 * used * width}
    return {"bytes": rows * k * 12 + (live + used) * width * size + (used + used + rows) * width * size, "flops": 4 * used * width}


# --------------------------------------------------------------------------- the same in 64 bits

def _stands_for(x):
    """What rows in 8 bits stand for: x rounded to multiples of the format's step, four significant bits within a block's range."""
    rows, width = x.shape
    p = torch.zeros(rows, _padded(width), device=x.device, dtype=torch.float64)
    p[:, :width] = x.double()
    p = p.view(rows, -1, BLOCK)
    top = p.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0) / 256))
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e).clamp(min=-117)
    e = torch.where(top > 0, e, -117.0)
    q = p * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(q / step) * step * torch.exp2(e)).view(rows, -1)[:, :width]


def exact(case, seed):
    """From the definitions, in 64 bits; the whole numbers by counting."""
    s = prepare(case, seed)
    op, n, t, width, k, experts = (case[v] for v in ("op", "workers", "rows", "width", "k", "experts"))
    rows, live = n * t, s["live"]
    dev = live.device

    def zeros(*size):
        return torch.zeros(*size, dtype=torch.float64, device=dev)

    if op in ("norm", "norm_step"):
        y, stats, dx, grads = zeros(rows, width), zeros(rows, 2), zeros(rows, width), zeros(n, 2 * width)
        for i in range(n):
            r = torch.nonzero(live[i * t:(i + 1) * t])[:, 0] + i * t
            w, b = s["params"][i, 5:5 + width].double(), s["params"][i, 5 + width:5 + 2 * width].double()
            x = s["x"][r, :width].double()
            m = x.sum(1, keepdim=True) / width
            variance = (x * x).sum(1, keepdim=True) / width - m * m
            root = torch.rsqrt(variance + EPS)
            y[r] = w * (x - m) * root + b
            stats[r] = torch.cat([m, root], 1)
            if op == "norm_step":
                dy, unit = s["dy"][r, :width].double(), (_stands_for(s["x"][r, :width]) - m) * root
                grads[i, :width], grads[i, width:] = (dy * unit).sum(0), dy.sum(0)
                d = w * dy
                dx[r] = root * d - root / width * (d.sum(1, keepdim=True) + unit * (d * unit).sum(1, keepdim=True))
        return {"y": y, "stats": stats} if op == "norm" else {"y": y, "stats": stats, "dx": dx, "grads": grads}
    if op == "checkpoint":
        return {"y": _stands_for(s["x"][:, :width])}
    if op == "weight_grad":
        out, size = case["out"], max(experts, 1)
        weight, bias = zeros(n, size, out, width), zeros(n, size, out)
        cut = rows * _padded(width)
        sign, field = s["checkpoint"][:cut].view(rows, -1).int() >> 7, s["checkpoint"][:cut].view(rows, -1).int() & 127
        plain = torch.where(field >= 8, (8 + field % 8) * torch.exp2((field // 8 - 10).double()), field * 2.0 ** -9)
        x = plain * (1 - 2 * sign) * torch.exp2(s["checkpoint"][cut:].view(rows, -1).double() - 127).repeat_interleave(BLOCK, 1)
        for i in range(n):
            for e in range(size):
                if experts:
                    a, z = s["start"][i, e].item(), s["start"][i, e + 1].item()
                    d, u = s["dy"][a:z, :out].double(), x[s["source"][a:z].long() // k, :width]
                else:
                    d, u = s["dy"][i * t:(i + 1) * t, :out].double(), x[i * t:(i + 1) * t, :width]
                weight[i, e], bias[i, e] = d.t().contiguous() @ u, d.sum(0)
        return {"weight": weight.view(n, -1), "bias": bias.view(n, -1)}
    if op == "experts":
        order, out = s["expert"].tolist(), {}
        start, place, source = [], [-1] * (rows * k), [-1] * (rows * k)
        for i in range(n):
            by = [[] for _ in range(experts)]
            for slot in range(i * t * k, (i + 1) * t * k):
                if order[slot] >= 0:
                    by[order[slot]].append(slot)
            at = i * t * k
            for those in by:
                start.append(at)
                for slot in those:
                    place[slot], source[at] = at, slot
                    at += 1
            start.append(at)
        out = {name: torch.tensor(v, dtype=torch.int32, device=dev) for name, v in (("start", start), ("place", place), ("source", source))}
        moved, to = zeros(rows * k, width), out["place"].long()
        slots = torch.nonzero(to >= 0)[:, 0]
        moved[to[slots]] = s["x"][slots // k, :width].double()
        out["sorted"] = moved
        place, z = to, s["z"]
    else:
        out, place, z = {}, s["place"].long(), s["dsorted"]
    y, weights = zeros(rows, width), s["weights"].double()
    if op == "experts_grad":
        dz, dweights = zeros(rows * k, width), zeros(rows, k)
    for j in range(k):
        at = place.view(rows, k)[:, j]
        r = torch.nonzero(at >= 0)[:, 0]
        by = weights[r, j, None] if op == "experts" else 1.0
        y[r] += by * z[at[r], :width].double()
        if op == "experts_grad":
            dz[at[r]] = weights[r, j, None] * s["dy"][r, :width].double()
            dweights[r, j] = (s["dy"][r, :width].double() * s["z"][at[r], :width].double()).sum(1)
    if op == "experts":
        return {**out, "y": y}
    return {"dz": dz, "dweights": dweights.view(-1), "dx": y}
