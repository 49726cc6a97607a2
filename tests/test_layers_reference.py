"""The 64-bit reference of what lies between a language model's products, against differences and closed forms, and what the entry points
refuse before any work reaches the GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import layer_reference as ref


def _differences(f, x, h=1e-6):
    out = torch.zeros_like(x)
    for i in range(x.numel()):
        hi, lo = x.clone().reshape(-1), x.clone().reshape(-1)
        hi[i] += h
        lo[i] -= h
        out.view(-1)[i] = (f(hi.view_as(x)) - f(lo.view_as(x))) / (2 * h)
    return out


def test_norm_gradient_is_differences():
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(3, 7, dtype=torch.float64, generator=g) for _ in range(2))
    w, b = (torch.randn(7, dtype=torch.float64, generator=g) for _ in range(2))
    _, mu, rho = ref.norm(x, w, b, 1e-3)
    dx, dw, db = ref.norm_grad(dy, x, w, mu, rho)
    loss = lambda a, c, d: (ref.norm(a, c, d, 1e-3)[0] * dy).sum()
    assert torch.allclose(dx, _differences(lambda a: loss(a, w, b), x), rtol=0, atol=1e-8)
    assert torch.allclose(dw.sum(0), _differences(lambda a: loss(x, a, b), w), rtol=0, atol=1e-8)
    assert torch.allclose(db.sum(0), _differences(lambda a: loss(x, w, a), b), rtol=0, atol=1e-8)
    assert torch.allclose(dx.sum(1), torch.zeros(3, dtype=torch.float64), atol=1e-12)


def test_eight_bits_are_the_nearest_codes():
    """Against all 253 numbers of the format."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    codes = codes[torch.isfinite(codes)].unique()
    assert codes.max() == 448 and codes[codes > 0].min() == 2.0 ** -9 and codes.numel() == 253
    g = torch.Generator().manual_seed(2)
    x = torch.randn(40, 70, generator=g) * torch.exp(3 * torch.randn(40, 70, generator=g))
    x[3, :40] = 0
    x[5, 2] = 448.0
    x[6, 2] = 448.1
    got, e = ref.kept(x), ref.exponents(x)
    for r in range(40):
        for k in range(3):
            block = x[r, 32 * k:32 * k + 32].double()
            by = 2.0 ** e[r, k].item()
            assert block.abs().max() <= 448 * by and (by == 2.0 ** -117 or block.abs().max() > 224 * by)
            for c, v in enumerate(block):
                d = (codes * by - v).abs()
                assert d.min() == (got[r, 32 * k + c] - v).abs()
    # the largest numbers, the smallest, and what is not one
    row = torch.tensor([[3.4e38, -3.0e38, 1.0, math.nan], [math.inf, 5.0, -math.inf, 0.0], [2.0 ** -126, 2.0 ** -127, 2.0 ** -130, 0.0]])
    got = ref.kept(row)
    assert got[0, 0] == 1.875 * 2.0 ** 127 and got[0, 2] == 0 and math.isnan(got[0, 3])
    assert math.isnan(got[1, 0]) and got[1, 1] == 5 and got[2, 0] == 2.0 ** -126 and got[2, 2] == 0


def test_combining_what_was_sorted_gives_every_token_its_rows():
    g = np.random.default_rng(3)
    expert = g.integers(-1, 4, 2 * 5 * 3).tolist()
    start, place, source = ref.sort(expert, 2, 4)
    assert len(start) == 10 and start[0] == 0 and start[5] == 15
    for i in range(2):
        rows = source[15 * i:15 * i + start[5 * i + 4] - 15 * i]
        assert rows == sorted(rows, key=lambda s: (expert[s], s)) and all(expert[s] >= 0 for s in rows)
    assert all(source[p] == s for s, p in enumerate(place) if p >= 0)
    x = torch.randn(10, 6, dtype=torch.float64, generator=torch.Generator().manual_seed(4))
    rows = torch.zeros(30, 6, dtype=torch.float64)
    for s, p in enumerate(place):
        if p >= 0:
            rows[p] = x[s // 3]
    y, _ = ref.combine(rows, torch.tensor(place).view(10, 3), None)
    named = torch.tensor([sum(e >= 0 for e in expert[3 * t:3 * t + 3]) for t in range(10)], dtype=torch.float64)
    assert torch.allclose(y, named[:, None] * x)


# --------------------------------------------------------------------------- refusals, on the host

@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


def at(i):
    """Addresses far from one another, never dereferenced: every call below is refused first."""
    return C.c_void_p((i + 1) << 32)


NAMES = ("x", "y", "mask", "params", "stats", "kept", "dy", "dx", "grads", "work", "expert", "start", "place", "source", "sorted", "weights",
         "dsorted", "dweights")
DEFAULTS = dict(ld_params=64, weight_at=0, bias_at=32, eps=1e-5, ld_grads=64)


def _calls(B, rows=None, routing=None, linear=None, only=None, **kw):
    """Codes of all entry points with these arguments, or of some."""
    a = {**{n: at(i) for i, n in enumerate(NAMES)}, **DEFAULTS, **kw}
    p = C.byref(rows) if rows is not None else None
    q = C.byref(routing) if routing is not None else None
    l = C.byref(linear) if linear is not None else None
    L = B._lib
    calls = {
        "bytes": lambda: L.dbw_checkpoint_bytes(p), "norm_work": lambda: L.dbw_layer_norm_work_bytes(p),
        "store": lambda: L.dbw_checkpoint_store(p, a["x"], None, a["kept"], None),
        "load": lambda: L.dbw_checkpoint_load(p, a["kept"], a["y"], None),
        "norm": lambda: L.dbw_layer_norm(p, a["x"], None, a["params"], a["ld_params"], a["weight_at"], a["bias_at"], a["eps"], a["y"], a["stats"],
                                         a["kept"], None),
        "norm_grad": lambda: L.dbw_layer_norm_grad(p, a["dy"], a["x"], a.get("checkpoint"), None, a["stats"], a["params"], a["ld_params"],
                                                   a["weight_at"], a["bias_at"], a["dx"], a["grads"], a["ld_grads"], a["work"], None),
        "sort_work": lambda: L.dbw_expert_work_bytes(q),
        "sort": lambda: L.dbw_expert_sort(q, a["expert"], a["start"], a["place"], a["source"], None, a["work"], None),
        "gather": lambda: L.dbw_expert_gather(q, p, a["x"], a["place"], a["sorted"], None, None),
        "combine": lambda: L.dbw_expert_combine(q, p, a["sorted"], a["place"], a["weights"], a["y"], None, None),
        "combine_grad": lambda: L.dbw_expert_combine_grad(q, p, a["dy"], a["sorted"], a["place"], a["weights"], a["dsorted"], a["dweights"], None,
                                                          None),
        "linear_work": lambda: L.dbw_checkpoint_weight_grad_work_bytes(l),
        "linear": lambda: L.dbw_checkpoint_weight_grad(l, a["dy"], a["kept"], a["start"], a["source"], a["grads"], a["ld_grads"], a["weight_at"],
                                                       a["bias_at"], None, a["work"], None),
    }
    return {name: calls[name]() for name in (only.split() if only else calls)}


ROWS = "bytes norm_work store load norm norm_grad gather combine combine_grad"
ROUTED = "sort_work sort gather combine combine_grad"


def _rows(B, **kw):
    return B.make_rows(**{**dict(workers=2, rows=3, width=5, type=B.TYPE_F32), **kw})


def _routing(B, **kw):
    return B.make_routing(**{**dict(workers=2, tokens=3, k=2, experts=4), **kw})


def _linear(B, **kw):
    return B.make_linear(**{**dict(workers=2, rows=6, inputs=5, outputs=2, type=B.TYPE_F32, experts=2, tokens=3, k=2), **kw})


@pytest.mark.parametrize("kw,code", [
    (dict(workers=0), "ERR_INVALID"), (dict(rows=-1), "ERR_INVALID"), (dict(width=0), "ERR_INVALID"), (dict(type=3), "ERR_INVALID"),
    (dict(type=-1), "ERR_INVALID"), (dict(ld=4), "ERR_INVALID"), (dict(ld_out=4), "ERR_INVALID"), (dict(ld=-7), "ERR_INVALID"),
    (dict(workers=1 << 20, rows=1 << 20), "ERR_UNSUPPORTED"), (dict(workers=(1 << 22) + 1), "ERR_UNSUPPORTED"), (dict(ld=1 << 62), "ERR_UNSUPPORTED"),
    (dict(ld_out=1 << 62), "ERR_UNSUPPORTED"), (dict(width=(1 << 20) + 1), "ERR_UNSUPPORTED")])
def test_rows_that_are_refused(B, kw, code):
    assert set(_calls(B, _rows(B, **kw), _routing(B), only=ROWS).values()) == {getattr(B, code)}
    with pytest.raises(B.DbwError) as e:
        B.dbw_checkpoint_bytes(_rows(B, **kw))
    assert e.value.code == getattr(B, code)


@pytest.mark.parametrize("kw,code", [
    (dict(workers=0), "ERR_INVALID"), (dict(tokens=-1), "ERR_INVALID"), (dict(k=0), "ERR_INVALID"), (dict(experts=0), "ERR_INVALID"),
    (dict(experts=1025), "ERR_UNSUPPORTED"), (dict(workers=(1 << 22) + 1), "ERR_UNSUPPORTED"), (dict(tokens=1 << 30), "ERR_UNSUPPORTED"),
    (dict(tokens=1 << 30, k=1 << 30), "ERR_UNSUPPORTED"), (dict(workers=1 << 22, experts=600), "ERR_UNSUPPORTED")])
def test_routings_that_are_refused(B, kw, code):
    assert set(_calls(B, _rows(B), _routing(B, **kw), only=ROUTED).values()) == {getattr(B, code)}


@pytest.mark.parametrize("kw,code", [
    (dict(workers=0), "ERR_INVALID"), (dict(rows=-1), "ERR_INVALID"), (dict(inputs=0), "ERR_INVALID"), (dict(outputs=0), "ERR_INVALID"),
    (dict(type=3), "ERR_INVALID"), (dict(experts=0), "ERR_INVALID"), (dict(tokens=-1), "ERR_INVALID"), (dict(k=0), "ERR_INVALID"),
    (dict(ld=1), "ERR_INVALID"), (dict(ld=1 << 62), "ERR_UNSUPPORTED"), (dict(experts=1025), "ERR_UNSUPPORTED"),
    (dict(workers=(1 << 22) + 1), "ERR_UNSUPPORTED"), (dict(rows=1 << 30), "ERR_UNSUPPORTED"), (dict(tokens=1 << 30), "ERR_UNSUPPORTED"),
    (dict(inputs=(1 << 20) + 1), "ERR_UNSUPPORTED"), (dict(outputs=(1 << 20) + 1), "ERR_UNSUPPORTED")])
def test_linear_layers_that_are_refused(B, kw, code):
    assert set(_calls(B, linear=_linear(B, **kw), only="linear_work linear").values()) == {getattr(B, code)}


def test_missing_pointers_are_refused(B):
    rows, routing, linear = _rows(B), _routing(B), _linear(B)
    assert set(_calls(B, None, routing, None, only=ROWS + " linear_work linear").values()) == {B.ERR_NULL}
    assert set(_calls(B, rows, None, only=ROUTED).values()) == {B.ERR_NULL}
    needs = {"store": "x kept", "load": "kept y", "norm": "x y params", "norm_grad": "dy x dx stats params work", "sort": "expert start place source work",
             "gather": "x place sorted", "combine": "sorted place y", "combine_grad": "dy sorted place dsorted", "linear": "dy kept start grads work"}
    for call, names in needs.items():
        for name in names.split():
            assert _calls(B, rows, routing, linear, only=call, **{name: None}) == {call: B.ERR_NULL}, (call, name)


def test_misaligned_pointers_are_refused(B):
    odd = lambda name, by=1: {name: C.c_void_p(at(NAMES.index(name)).value + by)}
    for t in (B.TYPE_F32, B.TYPE_BF16, B.TYPE_F16):
        rows, routing, linear = _rows(B, type=t), _routing(B), _linear(B, type=t)
        for call, names in {"store": "x", "load": "y", "norm": "x y", "norm_grad": "dy x dx", "gather": "x sorted", "combine": "sorted y",
                            "combine_grad": "dy sorted dsorted", "linear": "dy"}.items():
            for name in names.split():
                assert _calls(B, rows, routing, linear, only=call, **odd(name)) == {call: B.ERR_INVALID}, (call, name)
    rows = _rows(B)
    for call, name, by in [("store", "kept", 8), ("load", "kept", 8), ("norm", "kept", 8), ("norm", "params", 2), ("norm_grad", "work", 8),
                           ("norm_grad", "grads", 2), ("sort", "work", 8), ("linear", "work", 8), ("linear", "kept", 4), ("linear", "grads", 2)]:
        assert _calls(B, rows, _routing(B), _linear(B), only=call, **odd(name, by)) == {call: B.ERR_INVALID}, (call, name)


def test_numbers_out_of_range_are_refused(B):
    rows, linear = _rows(B), _linear(B)
    for eps in (0.0, -1e-5, math.inf, math.nan):
        assert _calls(B, rows, only="norm", eps=eps) == {"norm": B.ERR_INVALID}
    for kw in (dict(weight_at=60), dict(bias_at=60), dict(ld_params=4), dict(weight_at=1 << 62)):
        assert _calls(B, rows, only="norm", **kw) == {"norm": B.ERR_INVALID}
    for kw in (dict(weight_at=60), dict(bias_at=60), dict(ld_grads=30), dict(ld_params=4), dict(checkpoint=at(5))):
        assert _calls(B, rows, only="norm_grad", **kw) == {"norm_grad": B.ERR_INVALID}
    for kw in (dict(weight_at=-1), dict(weight_at=45), dict(bias_at=61), dict(ld_grads=19), dict(source=None)):
        assert _calls(B, linear=linear, only="linear", **kw) == {"linear": B.ERR_INVALID}
    for kw in (dict(workers=3), dict(rows=4)):
        assert set(_calls(B, _rows(B, **kw), _routing(B), only="gather combine combine_grad").values()) == {B.ERR_INVALID}
    assert _calls(B, rows, only="norm_grad", ld_grads=1 << 62) == {"norm_grad": B.ERR_UNSUPPORTED}
    assert _calls(B, linear=linear, only="linear", ld_grads=1 << 62) == {"linear": B.ERR_UNSUPPORTED}


def test_overlaps_are_refused(B):
    rows, routing, linear = _rows(B), _routing(B), _linear(B)
    near = lambda name, by: C.c_void_p(at(NAMES.index(name)).value + by)
    alias = lambda call, r=rows, **kw: _calls(B, r, routing, linear, only=call, **kw) == {call: B.ERR_ALIAS}
    for by in (4, -4, 2 * 3 * 5 * 4 - 4):
        assert alias("norm", y=near("x", by)) and alias("norm_grad", dx=near("x", by)) and alias("norm_grad", dx=near("dy", by))
    assert alias("norm", _rows(B, ld_out=6), y=near("x", 0)) and alias("norm_grad", _rows(B, ld_out=6), dx=near("dy", 0))
    assert alias("gather", sorted=near("x", 0)) and alias("gather", x=near("sorted", 2 * 6 * 5 * 4 - 4))
    assert alias("combine", y=near("sorted", 100)) and alias("combine_grad", dsorted=near("dy", 0)) and alias("combine_grad", dsorted=near("sorted", 4))
    assert alias("norm_grad", bias_at=4) and alias("norm_grad", weight_at=30)
    assert alias("linear", bias_at=19) and alias("linear", weight_at=30)


def test_the_binding_refuses_wrong_tensors(B):
    shape = _rows(B)
    x, y, params = torch.zeros(30), torch.zeros(30), torch.zeros(2, 16)
    for bad in (dict(x=x.double()), dict(x=x[:29]), dict(params=params[0]), dict(params=torch.zeros(3, 16)), dict()):      # the last: host memory
        a = {**dict(x=x, params=params), **bad}
        with pytest.raises(ValueError):
            B.dbw_layer_norm(shape, a["x"], a["params"], y, weight_at=0)


def test_sizes_of_checkpoints_and_scratch_memory(B):
    assert B.dbw_checkpoint_bytes(_rows(B, width=1)) == 6 * 33
    assert B.dbw_checkpoint_bytes(_rows(B, width=64, type=B.TYPE_BF16, ld=70)) == 6 * 66
    assert B.dbw_checkpoint_bytes(_rows(B, rows=0)) == 0
    for width in (1, 100, 5000, 50000):
        for rows in (0, 1, 10000):
            assert B.dbw_layer_norm_work_bytes(_rows(B, rows=rows, width=width)) >= 0
    assert B.dbw_expert_work_bytes(_routing(B, tokens=0)) >= 0 and B.dbw_checkpoint_weight_grad_work_bytes(_linear(B)) >= 0


def test_structs_match_the_header(B, tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {s: [f[0] for f in getattr(B, s)._fields_] for s in ("dbw_rows", "dbw_routing", "dbw_linear")}
    src = tmp_path / "layout.c"
    parts = [f'printf("%zu ", sizeof({s}));' + "".join(f'printf("%zu ", offsetof({s}, {f}));' for f in names) for s, names in fields.items()]
    src.write_text('#include <stdio.h>\n#include "dbw_layers.h"\nint main(void) { ' + " ".join(parts) +
                   'printf("%d %d\\n", DBW_LAYER_MAX_WIDTH, DBW_EXPERTS_MAX); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for s, names in fields.items():
        want += [C.sizeof(getattr(B, s))] + [getattr(getattr(B, s), f).offset for f in names]
    assert got == want + [B.LAYER_MAX_WIDTH, B.EXPERTS_MAX]
