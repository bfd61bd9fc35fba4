"""Weight and bias gradients from 8-bit activation checkpoints, against the sums in 64 bits, and one training step of an
int8 token policy from all of the Learner's operators together."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def inputs(t, n, k, dtype, seed, pad=0, offset=0):
    import paper_2211_15023_b200 as P
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((t, k), device="cuda", generator=g) * torch.exp(torch.randn((t, 1), device="cuda", generator=g))
    _, ckpt = P.ckpt_save(x.to(dtype))
    flat = torch.full((offset + t * (n + pad),), float("nan"), device="cuda", dtype=dtype)
    dy = flat[offset:].view(t, n + pad)[:, :n]
    dy.copy_(torch.randn((t, n), device="cuda", generator=g))
    return dy, ckpt


def sums(dy, ckpt, k):
    """float64 (dw, db), and for each a bound of what an fp32 sum of its exact products may be off.

    The tensor cores add sixteen products and the running sum at a time, and cut off: an addition loses less than a step
    of its result and of the sixteen products as they are aligned, 2^-23 of each at most, 2^-22 with the final one's.  A
    part of the tokens (the sum may be taken in parts) runs from one prefix sum to another, so no running sum is larger
    than twice the largest prefix sum."""
    import paper_2211_15023_b200 as P
    x, d = P.ckpt_load(ckpt, k, torch.float32).double(), dy.double()
    x = torch.cat([x, torch.ones_like(x[:, :1])], 1)  # (db: the product with ones)
    run = torch.zeros((d.shape[1], k + 1), dtype=torch.float64, device="cuda")
    top, steps = torch.zeros_like(run), 0
    for i in range(0, d.shape[0], 16):
        run += d[i:i + 16].t() @ x[i:i + 16]
        top, steps = torch.maximum(top, run.abs()), steps + 1
    slack = 2.0 ** -22 * (d.abs().t() @ x.abs() + 2 * (steps + 1) * top)
    return (run[:, :k], run[:, k]), (slack[:, :k], slack[:, k])


def check(got, want, slack, out):
    """The sum's error, and one rounding to the type."""
    half = torch.finfo(out).eps / 2
    tiny = torch.finfo(out).smallest_normal * torch.finfo(out).eps
    for g, w, m in zip(got, want, slack):
        if g is None:
            continue
        assert g.dtype == out
        bad = (g.double() - w).abs() > half * 1.01 * w.abs() + 1.01 * m + tiny
        assert not bad.any(), (int(bad.sum()), float((g.double() - w).abs().max()), tuple(g.shape))


# tokens: parts of a stage, split over a cluster or not; n: every tile width and parts of it; k: parts of a tile and a block
SIZES = [(1, 1, 1), (3, 16, 32), (64, 64, 128), (65, 70, 129), (63, 130, 40), (200, 256, 100), (512, 257, 300), (1000, 18, 512),
         (2047, 256, 2592), (300, 1000, 1000), (129, 515, 2100), (5000, 40, 200), (1030, 4100, 1300),
         (70, 3000, 2900), (3333, 2050, 2570), (1, 5000, 2500), (200, 600, 9000), (2500, 300, 14001)]


@pytest.mark.parametrize("t,n,k", SIZES)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
def test_gradients_match_the_sums(t, n, k, dtype, out):
    import paper_2211_15023_b200 as P
    dy, ckpt = inputs(t, n, k, TYPES[dtype], t + n + k)
    want, mag = sums(dy, ckpt, k)
    got = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out])
    P.device_check()
    check(got, want, mag, TYPES[out])
    again = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out])
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    dw, none = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out], bias=False)
    assert none is None and torch.equal(dw, got[0])


@pytest.mark.parametrize("t,n,k", [(5, 33, 70), (130, 300, 260), (2000, 64, 500)])
def test_rows_at_any_distance_and_sums_over_micro_batches(t, n, k):
    import paper_2211_15023_b200 as P
    for pad, offset in ((0, 0), (3, 1), (8, 3), (0, 8)):
        dy, ckpt = inputs(t, n, k, torch.bfloat16, t, pad, offset)
        want, mag = sums(dy, ckpt, k)
        wide = torch.full((n, k + 5), 7.0, device="cuda")
        out = (wide[:, 2:2 + k], torch.full((n,), 7.0, device="cuda"))
        got = P.ckpt_weight_grad(dy, ckpt, k, out=out)
        check(got, want, mag, torch.float32)
        assert (wide[:, :2] == 7).all() and (wide[:, 2 + k:] == 7).all()
        once = [g.clone() for g in got]
        P.ckpt_weight_grad(dy, ckpt, k, out=out, accumulate=True)
        # (x + y is rounded once: twice a value is exact)
        assert torch.equal(out[0], 2 * once[0]) and torch.equal(out[1], 2 * once[1])


def test_blocks_that_are_lost_or_empty_and_the_range_of_fp16():
    """A block kept as NaN spoils its 32 columns of dw and no other; zero blocks and scales beyond fp16's range do not."""
    import paper_2211_15023_b200 as P
    t, n, k = 100, 70, 200
    for dtype in (torch.bfloat16, torch.float16):
        x = torch.randn((t, k), device="cuda", generator=torch.Generator("cuda").manual_seed(5))
        x[:, 160:192] = 0
        x[:, 32:64] *= 2.0 ** -17
        x[:, 64:96] *= 2.0 ** 13
        x[3, 100] = math.inf
        _, ckpt = P.ckpt_save(x.to(dtype))
        dy = torch.randn((t, n), device="cuda", generator=torch.Generator("cuda").manual_seed(6)).to(dtype)
        dw, db = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
        lost = torch.zeros(k, dtype=torch.bool, device="cuda")
        lost[96:128] = True
        assert torch.isnan(dw[:, lost]).all() and torch.isfinite(dw[:, ~lost]).all() and torch.isfinite(db).all()
        ckpt[1][3, 3], ckpt[0][3, 96:128] = 127, 0
        want, mag = sums(dy, ckpt, k)
        check((dw[:, ~lost], db), (want[0][:, ~lost], want[1]), (mag[0][:, ~lost], mag[1]), torch.float32)


def test_against_differences_of_a_scalar():
    """sum(dy * (x w^T)) is linear in w: its difference in one weight is the gradient, up to fp64 arithmetic."""
    import paper_2211_15023_b200 as P
    dy, ckpt = inputs(40, 6, 50, torch.bfloat16, 9)
    dw, db = P.ckpt_weight_grad(dy, ckpt, 50, out_dtype=torch.float32)
    x, d = P.ckpt_load(ckpt, 50, torch.float32).double(), dy.double()
    w = torch.zeros((6, 50), dtype=torch.float64, device="cuda")
    f = lambda w, b: float((d * (x @ w.t() + b)).sum())  # noqa: E731
    zero = torch.zeros(6, dtype=torch.float64, device="cuda")
    for i, j in ((0, 0), (5, 49), (3, 17)):
        up = w.clone()
        up[i, j] = 1.0
        assert abs(f(up, zero) - f(w, zero) - float(dw[i, j])) < 1e-4
        b = zero.clone()
        b[i] = 1.0
        assert abs(f(w, b) - f(w, zero) - float(db[i])) < 1e-4


def test_a_training_step_of_an_int8_token_policy():
    """Two int8 layers with a GELU between them and a policy loss on top; the activations are kept in 8 bits.  Every
    gradient against the same step in float64 on the values that were kept (the backward pass is linear in them), with
    the roundings of bf16 in between; run directly, and captured into a graph and replayed with new inputs."""
    import paper_2211_15023_b200 as P
    t, k, h, v = 300, 256, 640, 1000
    g = torch.Generator("cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    w1, w2 = (r(h, k) / 16).bfloat16(), (r(v, h) / 16).bfloat16()
    b1 = 0.1 * r(h)
    x = r(t, k).bfloat16()
    a = torch.randint(0, v, (t,), device="cuda", generator=g)
    adv, w = r(t), torch.full((t,), 1.0 / t, device="cuda")
    logp_old = torch.full((t,), -math.log(v), device="cuda") + 0.1 * r(t)

    def step():
        q1, q2 = P.quant_rows(w1), P.quant_rows(w2)
        _, kept_x = P.ckpt_save(x)
        z1 = P.linear_i8(x, q1, bias=b1)
        y1, kept_z = P.ckpt_save(z1, "gelu")
        _, kept_y = P.ckpt_save(y1)
        z2 = P.linear_i8(y1, q2)
        loss = P.policy_loss(z2, a, logp_old, adv, weights=w, kl_coef=0.1, logp_ref=logp_old, entropy_coef=0.01)
        dz2 = loss["grad"]
        dw2, _ = P.ckpt_weight_grad(dz2, kept_y, h, out_dtype=torch.float32, bias=False)
        dy1 = dz2 @ w2
        dz1 = P.ckpt_act_backward(dy1, kept_z, "gelu")
        dw1, db1 = P.ckpt_weight_grad(dz1, kept_x, k, out_dtype=torch.float32)
        return dict(loss=loss["stats"], dw1=dw1, db1=db1, dw2=dw2, dz2=dz2, z2=z2, kept=(kept_x, kept_z, kept_y))

    def verify(o):
        kx, kz, ky = (P.ckpt_load(c, n, torch.float32).double() for c, n in zip(o["kept"], (k, h, h)))
        z = o["z2"].double().requires_grad_(True)
        lp = torch.log_softmax(z, 1)
        taken = lp.gather(1, a[:, None])[:, 0]
        ratio = (taken - logp_old.double()).exp()
        ad = adv.double()
        pg = -torch.minimum(ratio * ad, ratio.clamp(0.8, 1.2) * ad)
        d = logp_old.double() - taken
        total = (w.double() * (pg + 0.1 * (d.exp() - 1 - d) + 0.01 * (lp.exp() * lp).sum(1))).sum()
        dz2, = torch.autograd.grad(total, z)
        assert abs(float(total) - float(o["loss"][0])) < 1e-5 * max(1.0, abs(float(total)))
        cdf = torch.special.ndtr(kz)
        dz1 = (dz2 @ w2.double()) * (cdf + kz * torch.exp(-kz * kz / 2) / math.sqrt(2 * math.pi))
        # relative in norm: each bf16 rounding on the way (dz2; then the product with w2, then dz1) adds 2^-8 at most
        for got, want, steps in ((o["dz2"], dz2, 1), (o["dw2"], dz2.t() @ ky, 1), (o["dw1"], dz1.t() @ kx, 3),
                                 (o["db1"], dz1.sum(0), 3)):
            off = (got.double() - want).norm() / want.norm()
            assert off < steps * 2.0 ** -8 * 1.01, float(off)

    verify(step())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = step()
    for seed in (1, 2):
        x.copy_(torch.randn((t, k), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).bfloat16())
        graph.replay()
        verify(o)
    P.device_check()


@pytest.mark.parametrize("t,n,k", [(200, 70, 300), (300, 2001, 4000), (1000, 520, 15000)])
def test_named_streams_captures_and_two_calls_at_once_on_another_stream(t, n, k):
    """Every kernel's form (small tiles over a cluster, read back first, decoded by pairs): on a stream named by its
    address while torch reuses what the call gave back, beside a layer's product on another stream, captured and replayed
    with other inputs."""
    import paper_2211_15023_b200 as P
    dy, ckpt = inputs(t, n, k, torch.bfloat16, t, pad=1)  # (rows off 16 bytes: a workspace too)
    want = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
    w = P.quant_rows(torch.randn((3000, 640), device="cuda"))
    x = torch.randn((40, 640), device="cuda").bfloat16()
    y = P.linear_i8(x, w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got, ys = [], []
    for _ in range(10):
        got.append(P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32, stream=side.cuda_stream))
        ys.append(P.linear_i8(x, w))
        torch.empty(1 << 22, device="cuda", dtype=torch.uint8).fill_(255)  # (what the first call's workspace was, were it free)
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
    assert all(torch.equal(v, y) for v in ys)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
    other, _ = inputs(t, n, k, torch.bfloat16, t + 1, pad=1)
    for new in (dy.clone(), other):
        dy.copy_(new)
        graph.replay()
        direct = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
        assert torch.equal(out[0], direct[0]) and torch.equal(out[1], direct[1])
    P.device_check()
