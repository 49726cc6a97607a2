"""The 64-bit reference of the losses on logits against differences and closed forms, and what the entry points refuse before any work
reaches the GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import loss_reference as ref


def _differences(f, x, entries, h=1e-5):
    out = []
    for r, v in entries:
        hi, lo = x.clone(), x.clone()
        hi[r, v] += h
        lo[r, v] -= h
        out.append((f(hi) - f(lo)).item() / (2 * h))
    return np.array(out)


@pytest.mark.parametrize("tail", [False, True])
def test_distillation_gradient_is_the_formula(tail):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(3, 11, dtype=torch.float64, generator=g) * 2
    index = torch.tensor([[4, 0, 7], [10, -1, 2], [-1, 5, -1]])
    value = torch.randn(3, 3, dtype=torch.float64, generator=g)
    lse = torch.logsumexp(torch.where(index >= 0, value * 0.5, -math.inf), 1) + 0.3 if tail else None
    f = lambda a: ref.distill_rows(a, index, value, 0.5, lse).sum()
    xg = x.clone().requires_grad_()
    f(xg).backward()
    entries = [(r, v) for r in range(3) for v in range(11)]
    assert np.allclose(xg.grad.reshape(-1).numpy(), _differences(f, x, entries), rtol=0, atol=1e-8)
    # s (p - q) in K; s p (1 - R / S) outside, or s p
    p = torch.softmax(0.5 * x, 1)
    want = p.clone()
    for r in range(3):
        k = [int(v) for v in index[r] if v >= 0]
        t = torch.stack([0.5 * value[r, j] for j in range(3) if index[r, j] >= 0])
        q = torch.exp(t - (lse[r] if tail else torch.logsumexp(t, 0)))
        if tail:
            outside = torch.ones(11, dtype=torch.bool)
            outside[k] = False
            want[r] = p[r] * (1 - (1 - q.sum()) / p[r][outside].sum())
        want[r, k] = p[r, k] - q
    assert torch.allclose(xg.grad, 0.5 * want, rtol=0, atol=1e-12)


def test_distillation_from_oneself_costs_nothing():
    x = torch.randn(2, 9, dtype=torch.float64, generator=torch.Generator().manual_seed(5))
    index = torch.tensor([[1, 3, 5], [8, 0, 2]])
    xg = x.clone().requires_grad_()
    loss = ref.distill_rows(xg, index, x.gather(1, index), 1.0, torch.logsumexp(x, 1))
    assert torch.allclose(loss, torch.zeros(2, dtype=torch.float64), atol=1e-14)
    loss.sum().backward()
    assert xg.grad.abs().max() < 1e-14


def test_policy_and_preference_gradients_are_differences():
    g = torch.Generator().manual_seed(7)
    x = torch.randn(6, 9, dtype=torch.float64, generator=g) * 2
    y = torch.randint(0, 9, (6,), generator=g)
    base = ref.token_logp(x, y, 0.8)
    old, rf = base - torch.tensor([0.1, -0.3, 0.5, -0.1, 0.4, -0.5]), base + torch.randn(6, dtype=torch.float64, generator=g) * 0.3
    adv = torch.tensor([1.0, 1.0, 1.0, -1.0, -0.5, -2.0], dtype=torch.float64)
    w = torch.tensor([0.5, 1.0, 0.25, 2.0, 1.0, 1.0], dtype=torch.float64)
    for f in (lambda a: (w * ref.policy_rows(ref.token_logp(a, y, 0.8), old, rf, adv, 0.2, 0.28, 0.05)[0]).sum(),
              lambda a: ref.preference(ref.token_logp(a, y, 0.8), rf, w, [0, 2, 2, 3, 6], 0.7, 0.1, 2, 1)[0].sum()):
        xg = x.clone().requires_grad_()
        f(xg).backward()
        entries = [(r, v) for r in range(6) for v in range(9)]
        assert np.allclose(xg.grad.reshape(-1).numpy(), _differences(f, x, entries), rtol=0, atol=1e-8)
    # a ratio beyond the bound that its advantage's sign looks at has no surrogate gradient
    logp = base.clone().requires_grad_()
    ref.policy_rows(logp, old, None, adv, 0.2, 0.28, 0.0)[0].sum().backward()
    rho = torch.exp(base - old)
    want = torch.where(((adv > 0) & (rho > 1.28)) | ((adv < 0) & (rho < 0.8)), 0.0, -rho * adv)
    assert torch.allclose(logp.grad, want, atol=1e-7)


# --------------------------------------------------------------------------- refusals, on the host

@pytest.fixture(scope="module")
def B():
    from paper_2102_06280_amd import binding
    return binding


FAKE = C.c_void_p(1 << 20)          # never dereferenced: every call below is refused first


def _calls(B, shape, logits=FAKE, dlogits=None, work=FAKE, k=2, teacher_type=0, pairs=1, beta=0.1, smoothing=0.0, low=0.2, high=0.2,
           kl=0.1, out=FAKE, data=FAKE, leave=()):
    """Codes of all entry points but those in `leave`, which would go on to the GPU with these arguments."""
    p = C.byref(shape) if shape is not None else None
    L = B._lib
    grad = dlogits if dlogits is not None else C.c_void_p(1 << 40)
    calls = {
        "logp": lambda: L.dbw_token_logp(p, logits, data, out, None, None, work, None),
        "grad": lambda: L.dbw_token_logp_grad(p, logits, data, data, data, grad, None, None),
        "distill": lambda: L.dbw_distill_loss(p, k, logits, data, teacher_type, data, None, None, out, None, grad, None, work, None),
        "preference": lambda: L.dbw_preference_loss(p, pairs, logits, data, data, data, None, beta, smoothing, out, out, None, grad, None, work,
                                            None),
        "policy": lambda: L.dbw_policy_loss(p, logits, data, data, None, data, None, low, high, kl, out, None, None, grad, None, work,
                                            None),
    }
    return {name: call() for name, call in calls.items() if name not in leave}


def _shape(B, **kw):
    return B.make_logits(**{**dict(workers=2, rows=3, vocab=5, type=B.TYPE_F32), **kw})


@pytest.mark.parametrize("kw,code", [
    (dict(workers=0), "ERR_INVALID"), (dict(rows=-1), "ERR_INVALID"), (dict(vocab=0), "ERR_INVALID"), (dict(type=3), "ERR_INVALID"),
    (dict(type=-1), "ERR_INVALID"), (dict(ld=4), "ERR_INVALID"), (dict(ld_grad=4), "ERR_INVALID"), (dict(ld=-7), "ERR_INVALID"),
    (dict(scale=0.0), "ERR_INVALID"), (dict(scale=-1.0), "ERR_INVALID"), (dict(scale=math.inf), "ERR_INVALID"),
    (dict(scale=math.nan), "ERR_INVALID"), (dict(workers=1 << 20, rows=1 << 20), "ERR_UNSUPPORTED"),
    (dict(workers=(1 << 22) + 1), "ERR_UNSUPPORTED"), (dict(ld=1 << 62), "ERR_UNSUPPORTED"), (dict(vocab=(1 << 28) + 1), "ERR_UNSUPPORTED")])
def test_shapes_that_are_refused(B, kw, code):
    shape = _shape(B, **kw)
    want = getattr(B, code)
    assert B._lib.dbw_loss_work_bytes(C.byref(shape)) == want
    assert set(_calls(B, shape).values()) == {want}
    with pytest.raises(B.DbwError) as e:
        B.dbw_loss_work_bytes(shape)
    assert e.value.code == want


def test_missing_pointers_are_refused(B):
    assert B._lib.dbw_loss_work_bytes(None) == B.ERR_NULL
    assert set(_calls(B, None).values()) == {B.ERR_NULL}
    assert set(_calls(B, _shape(B), logits=None).values()) == {B.ERR_NULL}
    assert set(_calls(B, _shape(B), data=None).values()) == {B.ERR_NULL}
    for what in (dict(work=None), dict(out=None)):
        assert set(_calls(B, _shape(B), **what, leave=("grad",)).values()) == {B.ERR_NULL}
    assert B._lib.dbw_token_logp_grad(C.byref(_shape(B)), FAKE, FAKE, FAKE, FAKE, None, None, None) == B.ERR_NULL


def test_misaligned_pointers_are_refused(B):
    odd = C.c_void_p((1 << 20) + 1)
    for t in (B.TYPE_F32, B.TYPE_BF16, B.TYPE_F16):
        assert set(_calls(B, _shape(B, type=t), logits=odd).values()) == {B.ERR_INVALID}
    assert set(_calls(B, _shape(B), dlogits=odd, leave=("logp",)).values()) == {B.ERR_INVALID}
    assert set(_calls(B, _shape(B), work=C.c_void_p((1 << 20) + 4), leave=("grad",)).values()) == {B.ERR_INVALID}


def test_numbers_out_of_range_are_refused(B):
    s = _shape(B)
    for kw in (dict(k=0), dict(k=-3), dict(teacher_type=3), dict(teacher_type=-1)):
        assert _calls_one(B, s, "distill", **kw) == B.ERR_INVALID, kw
    assert _calls_one(B, s, "distill", k=B.TEACHER_MAX + 1) == B.ERR_UNSUPPORTED
    assert _calls_one(B, _shape(B, vocab=B.DISTILL_MAX_VOCAB + 1), "distill") == B.ERR_UNSUPPORTED
    for kw in (dict(pairs=-1), dict(beta=math.inf), dict(beta=math.nan), dict(smoothing=-0.1), dict(smoothing=1.5), dict(smoothing=math.nan)):
        assert _calls_one(B, s, "preference", **kw) == B.ERR_INVALID, kw
    assert _calls_one(B, s, "preference", pairs=1 << 22) == B.ERR_UNSUPPORTED
    for kw in (dict(low=-0.1), dict(low=1.1), dict(low=math.nan), dict(high=-0.1), dict(high=math.nan), dict(kl=math.inf), dict(kl=math.nan)):
        assert _calls_one(B, s, "policy", **kw) == B.ERR_INVALID, kw


def _calls_one(B, shape, name, **kw):
    """One entry point alone, with numbers of its own."""
    p, L, d = C.byref(shape), B._lib, dict(k=2, teacher_type=0, pairs=1, beta=0.1, smoothing=0.0, low=0.2, high=0.2, kl=0.1)
    d.update(kw)
    if name == "distill":
        return L.dbw_distill_loss(p, d["k"], FAKE, FAKE, d["teacher_type"], FAKE, None, None, FAKE, None, None, None, FAKE, None)
    if name == "preference":
        return L.dbw_preference_loss(p, d["pairs"], FAKE, FAKE, FAKE, FAKE, None, d["beta"], d["smoothing"], FAKE, FAKE, None, None, None,
                                     FAKE, None)
    return L.dbw_policy_loss(p, FAKE, FAKE, FAKE, None, FAKE, None, d["low"], d["high"], d["kl"], FAKE, None, None, None, None, FAKE, None)


@pytest.mark.parametrize("offset,ld_grad", [(4, 0), (-4, 0), (2 * 3 * 5 * 4 - 4, 0), (0, 6), (-(5 * 6 + 5) * 4 + 4, 6)])
def test_gradients_that_overlap_the_logits_in_part_are_refused(B, offset, ld_grad):
    calls = _calls(B, _shape(B, ld=5, ld_grad=ld_grad), dlogits=C.c_void_p((1 << 20) + offset), leave=("logp",))
    assert set(calls.values()) == {B.ERR_ALIAS}


def test_the_binding_refuses_wrong_tensors(B):
    shape = _shape(B)
    work = torch.empty(B.dbw_loss_work_bytes(shape), dtype=torch.uint8)
    x, tokens, out = torch.zeros(30), torch.zeros(6, dtype=torch.int32), torch.zeros(6)
    for bad in (dict(x=x.double()), dict(x=torch.zeros(29)), dict(tokens=tokens.long()), dict(tokens=tokens[:5]), dict(out=out[:5]),
                dict(work=work[:-1]), dict()):          # the last: host memory
        a = {**dict(x=x, tokens=tokens, out=out, work=work), **bad}
        with pytest.raises(ValueError):
            B.dbw_token_logp(shape, a["x"], a["tokens"], a["out"], a["work"])


def test_scratch_memory_as_the_binding_counts_it(B):
    for n, t in ((1, 0), (1, 1), (3, 7), (16, 4096)):
        shape = _shape(B, workers=n, rows=t)
        assert B._rows(shape)[-1] == B.dbw_loss_work_bytes(shape)


def test_logits_struct_matches_the_header(B, tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "dbw_losses.h"\nint main(void) { printf("%zu %zu %zu %zu %d %d\\n", sizeof(dbw_logits), '
                   'offsetof(dbw_logits, ld), offsetof(dbw_logits, ld_grad), offsetof(dbw_logits, scale), DBW_TEACHER_MAX, '
                   'DBW_DISTILL_MAX_VOCAB); return 0; }\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(B.dbw_logits), B.dbw_logits.ld.offset, B.dbw_logits.ld_grad.offset, B.dbw_logits.scale.offset, B.TEACHER_MAX,
                   B.DISTILL_MAX_VOCAB]
