"""Activation checkpoints: GELU's tail, values at the ends of their types, rows written in place."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def phi(x):
    """(Phi, its density) in float64, the tail to full relative accuracy."""
    return 0.5 * torch.special.erfc(-x / math.sqrt(2)), torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_gelu_keeps_its_relative_accuracy_on_the_tail(dtype):
    """x Phi(x) from -13 on: Phi's relative error (2e-6, in 16-bit types 2e-5), and one rounding."""
    import paper_2211_15023_b200 as P
    dt = TYPES[dtype]
    x = torch.linspace(-13, 3, 1 << 16, device="cuda").to(dt).view(64, 1024)
    info = torch.finfo(dt)
    rel, tiny = (2e-6 if dtype == "fp32" else 2e-5) + 1.01 * info.eps / 2, info.smallest_normal * info.eps
    y, _ = P.ckpt_save(x, "gelu")
    xd = x.double().cpu()
    want = xd * phi(xd)[0]
    assert ((y.double().cpu() - want).abs() <= rel * want.abs() + tiny).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_the_slope_of_gelu_keeps_it_too(dtype):
    """Phi(x) + x phi(x): the terms' relative errors, and one rounding."""
    import paper_2211_15023_b200 as P
    dt = TYPES[dtype]
    info = torch.finfo(dt)
    q = torch.arange(-127, 1, device="cuda", dtype=torch.int32).view(4, 32).to(torch.int8)
    for e in (127 - 3, 127 - 4, 127 - 5, 127 - 9):  # steps of 1/8 (to -15.9) and less
        ex = torch.full((4, 1), e, device="cuda", dtype=torch.uint8)
        x = (q.double() * 2.0 ** (e - 127)).cpu()
        got = P.ckpt_act_backward(torch.ones((4, 32), device="cuda", dtype=dt), (q, ex), "gelu").double().cpu()
        cdf, density = phi(x)
        want = cdf + x * density
        rel = 3e-6 if dtype == "fp32" else 3e-5
        tol = rel * (cdf + (x * density).abs()) + 1.01 * info.eps / 2 * want.abs() + info.smallest_normal * info.eps
        assert ((got - want).abs() <= tol)[x >= -13].all()
        assert (got.abs() <= 1e-30)[x < -13].all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_slopes_at_the_type_s_largest_values(act, dtype):
    """A mask of the type's lowest value rounds to -2^128 in the checkpoint: the slope there is 0 (or 1), not NaN."""
    import paper_2211_15023_b200 as P
    dt = TYPES[dtype]
    x = torch.ones((4, 128), device="cuda", dtype=dt)
    x[0, 3], x[1, 40], x[2, 70], x[3, 100] = torch.finfo(dt).min, torch.finfo(dt).max, -1e30, 1e30
    y, ckpt = P.ckpt_save(x, act)
    assert torch.isfinite(y).all()
    dx = P.ckpt_act_backward(torch.full_like(x, 0.5), ckpt, act)
    kept = P.ckpt_load(ckpt, 128, torch.float32).double()
    one = {"none": 1.0, "relu": 1.0, "gelu": 1.0833154705876864, "silu": 0.9276705118714869}[act]  # the slope at 1
    low = 1.0 if act == "none" else 0.0
    zero = {"none": 1.0, "relu": 0.0, "gelu": 0.5, "silu": 0.5}[act]  # where a block's scale leaves nothing of the ones
    want = torch.where(kept == 1, one, torch.where(kept == 0, zero, torch.where(kept < 0, low, 1.0))) * 0.5
    assert torch.isfinite(dx).all() and ((dx.double() - want).abs() <= torch.finfo(dt).eps * want).all()
    assert float(dx[0, 3]) == low * 0.5 and float(dx[1, 40]) == 0.5 and float(dx[2, 70]) == low * 0.5 and float(dx[3, 100]) == 0.5
