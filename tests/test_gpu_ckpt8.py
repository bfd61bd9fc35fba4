"""Activation checkpoints in 8 bits (blocks of 32 values that share a power of two): kept, read back and used in the
backward pass, against their definition in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = [(1, 1), (1, 31), (3, 32), (5, 33), (160, 512), (7, 1000), (2, 4096), (33, 8191), (3, 16400), (1, 40001), (700, 64)]


def codes(x):
    """(q, e) of the definition, float64 on the host."""
    x = x.double().cpu()
    t, k = x.shape
    b = torch.nn.functional.pad(x, (0, -k % 32)).view(t, -1, 32)
    top = b.abs().amax(2)
    broken = ~torch.isfinite(b).all(2)
    safe = torch.where(broken, torch.ones_like(top), top)
    power = torch.frexp(safe).exponent.double() - 7
    power = torch.where(torch.round(safe * torch.exp2(-power)) > 127, power + 1, power).clamp(min=-126)
    power = torch.where(safe == 0, torch.full_like(power, -126.0), power)
    q = torch.round(torch.where(broken[:, :, None], torch.zeros_like(b), b) * torch.exp2(-power)[:, :, None])
    e = torch.where(broken, torch.full_like(power, 255.0), power + 127)
    return q.to(torch.int8).view(t, -1), e.to(torch.uint8)


def values(q, e, k):
    scale = torch.where(e == 255, torch.full_like(e, 1, dtype=torch.float64) * math.nan, torch.exp2(e.double() - 127))
    return (q.double().view(q.shape[0], -1, 32) * scale[:, :, None]).view(q.shape[0], -1)[:, :k]


def act64(x, act):
    if act == "relu":
        return torch.relu(x), (x > 0).double()
    if act == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * torch.sigmoid(-x)
    if act == "gelu":
        c = torch.special.ndtr(x)
        return x * c, c + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return x, torch.ones_like(x)


def matrix(t, k, dtype, seed, pad=0, offset=0):
    g = torch.Generator("cuda").manual_seed(seed)
    flat = torch.full((offset + t * (k + pad),), float("nan"), device="cuda", dtype=dtype)
    x = flat[offset:].view(t, k + pad)[:, :k]
    x.copy_(torch.randn((t, k), device="cuda", generator=g) * torch.exp(2 * torch.randn((t, 1), device="cuda", generator=g)))
    return x


def close(got, want, dtype, factor=1.0):
    """Computed in fp32 and rounded once: half a step of the type, and on top the absolute error of Phi or of the
    logistic function (3e-7, and 2^-21 for what their factors round) times `factor`, the largest that multiplies it."""
    half = torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    got, want = got.double().cpu(), want.double().cpu()
    tol = 1.01 * half * want.abs() + 8e-7 * factor + tiny
    bad = (got - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


@pytest.mark.parametrize("t,k", SIZES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_kept_read_back_and_used_in_the_backward_pass(t, k, dtype, act):
    import paper_2211_15023_b200 as P
    x = matrix(t, k, TYPES[dtype], 100 * t + k)
    x[0, 0] = 0.0
    y, (q, e) = P.ckpt_save(x, act)
    want_q, want_e = codes(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(e.cpu(), want_e)
    if act == "none":
        assert y is x
    else:
        close(y, act64(x.double(), act)[0], TYPES[dtype], x.abs().double().cpu())
    kept = values(want_q, want_e, k)
    for out in TYPES.values():
        back = P.ckpt_load((q, e), k, out)
        assert torch.equal(back.cpu(), kept.to(out))
    # off by at most half a step of the block's scale; bf16 holds every kept value
    assert torch.equal(P.ckpt_load((q, e), k, torch.bfloat16).double().cpu(), kept)
    blocks = torch.nn.functional.pad((x.double().cpu() - kept).abs(), (0, -k % 32)).view(t, -1, 32).amax(2)
    assert (blocks <= 0.5 * torch.exp2(want_e.double() - 127) * (1 + 1e-12) + 0.5 * (blocks > 0) * 2.0 ** -126).all()
    dy = matrix(t, k, TYPES[dtype], 3 * t + k)
    dx = P.ckpt_act_backward(dy, (q, e), act)
    slope = act64(kept, act)[1]
    close(dx, dy.double().cpu() * slope, TYPES[dtype], dy.abs().double().cpu() * (1 + kept.abs()).clamp(max=32))


@pytest.mark.parametrize("pad,offset", [(3, 0), (8, 1), (0, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_at_any_distance_and_alignment_and_in_place(dtype, pad, offset):
    import paper_2211_15023_b200 as P
    t, k, dt = 9, 333, TYPES[dtype]
    x = matrix(t, k, dt, 1, pad, offset)
    y0, (q0, e0) = P.ckpt_save(x.contiguous(), "gelu")
    wide = torch.full((offset + t * (k + pad),), 7.0, device="cuda", dtype=dt)
    out = wide[offset:].view(t, k + pad)[:, :k]
    y, (q, e) = P.ckpt_save(x, "gelu", out=out)
    assert y is out and torch.equal(y, y0) and torch.equal(q, q0) and torch.equal(e, e0)
    assert (wide[:offset] == 7).all() and (wide[offset:].view(t, k + pad)[:, k:] == 7).all()
    dy = matrix(t, k, dt, 2, pad, offset)
    dx0 = P.ckpt_act_backward(dy.contiguous(), (q, e), "silu")
    assert torch.equal(P.ckpt_act_backward(dy, (q, e), "silu", out=dy), dx0) and torch.equal(dy, dx0)
    assert torch.equal(P.ckpt_save(x, "gelu", out=x)[0], y0) and torch.equal(x, y0)
    # a checkpoint that is part of a wider one
    qw, ew = torch.zeros((t, 512), device="cuda", dtype=torch.int8), torch.zeros((t, 16), device="cuda", dtype=torch.uint8)
    qw[:, 64:64 + q.shape[1]], ew[:, 2:2 + e.shape[1]] = q, e
    part = (qw[:, 64:64 + q.shape[1]], ew[:, 2:2 + e.shape[1]])
    assert torch.equal(P.ckpt_load(part, k, dt), P.ckpt_load((q, e), k, dt))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_blocks_at_the_ends_of_the_range(dtype):
    """Zeros, the type's smallest and largest values, a mantissa that rounds to 128, infinities and NaN: only the block
    that holds one is lost."""
    import paper_2211_15023_b200 as P
    dt = TYPES[dtype]
    info = torch.finfo(dt)
    x = torch.ones((8, 96), device="cuda", dtype=dt)
    x[1] = 0
    x[2, :40] = info.smallest_normal * info.eps
    x[3, 3], x[3, 50] = info.max, info.min
    x[4, 32:64] = torch.linspace(-255 / 128, 255 / 128, 32, device="cuda").to(dt)
    x[5, 1], x[5, 40] = math.inf, -math.inf
    x[6, 95] = math.nan
    x[7, :32] = 127.5 / 64
    y, (q, e) = P.ckpt_save(x, "relu")
    want_q, want_e = codes(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(e.cpu(), want_e)
    assert torch.equal(torch.isnan(y), torch.isnan(x))
    back = P.ckpt_load((q, e), 96, dt)
    lost = torch.zeros((8, 3), dtype=torch.bool)
    lost[5, 0] = lost[5, 1] = lost[6, 2] = True
    assert torch.equal(torch.isnan(back).cpu().view(8, 3, 32).all(2), lost)
    assert torch.equal(torch.isnan(back).cpu().view(8, 3, 32).any(2), lost)
    dx = P.ckpt_act_backward(torch.ones_like(x), (q, e), "silu")
    assert torch.equal(torch.isnan(dx).cpu().view(8, 3, 32).all(2), lost)


def test_slopes_against_differences():
    """(act(x + h) - act(x - h)) / 2h of the kernel's own fp32 activation: its error 3e-7 |x| / h, the third derivative
    (below 2) times h^2 / 6."""
    import paper_2211_15023_b200 as P
    q = torch.arange(-127, 128, device="cuda", dtype=torch.int32)
    q = torch.cat([q, q[:1]]).view(8, 32).to(torch.int8)
    e = torch.full((8, 1), 127 - 5, device="cuda", dtype=torch.uint8)  # steps of 1/32, +-3.97
    x = P.ckpt_load((q, e), 32, torch.float32)
    h = 2.0 ** -6
    for act in ("gelu", "silu"):
        d = P.ckpt_act_backward(torch.ones_like(x), (q, e), act)
        up, down = P.ckpt_save(x + h, act)[0], P.ckpt_save(x - h, act)[0]
        assert ((up.double() - down.double()) / (2 * h) - d.double()).abs().max() < 3e-7 * 4 / h + 2 * h * h / 6


def test_many_rows_pass_32_bits_of_offset():
    """2.3e9 values of 16 bits: the first and the last rows of the matrix, against the same rows alone."""
    import paper_2211_15023_b200 as P
    t, k = 70001, 32768
    x = torch.zeros((t, k), device="cuda", dtype=torch.bfloat16)
    ends = [slice(0, 9), slice(t - 9, t)]
    for i, part in enumerate(ends):
        x[part] = torch.randn((9, k), device="cuda", generator=torch.Generator("cuda").manual_seed(i)).bfloat16()
    alone = [P.ckpt_save(x[part].clone(), "gelu") for part in ends]
    y, (q, e) = P.ckpt_save(x, "gelu", out=x)
    assert y is x
    back = P.ckpt_load((q, e), k, torch.bfloat16)
    for part, (y1, (q1, e1)) in zip(ends, alone):
        assert torch.equal(x[part], y1) and torch.equal(q[part], q1) and torch.equal(e[part], e1)
        assert torch.equal(back[part], P.ckpt_load((q1, e1), k, torch.bfloat16))
    assert not q[9:t - 9].any()
    dx = P.ckpt_act_backward(x, (q, e), "silu", out=x)
    for part, (y1, c1) in zip(ends, alone):
        assert torch.equal(dx[part], P.ckpt_act_backward(y1, c1, "silu"))
