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
