"""The clipped policy loss with its KL and entropy terms, forward and backward, against its definition in 64 bits
(Section 2.3, Eq. IS; Section 2.2, Eq. KD)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def definition(z, a, logp_old, adv, w, zr=None, logp_ref=None, clip=(0.2, 0.2), kl_coef=0.0, entropy_coef=0.0):
    """Loss, sums and per-row values in float64, the gradient by automatic differentiation of exactly that loss."""
    z = z.detach().double().cpu().requires_grad_(True)
    w, adv, logp_old, a = w.double().cpu(), adv.double().cpu(), logp_old.double().cpu(), a.long().cpu()
    used = w != 0
    zs = torch.where(used[:, None], z, torch.zeros_like(z))
    alive = torch.isfinite(zs).any(1)  # a row of -inf only has no distribution
    zs = torch.where(alive[:, None], zs, torch.zeros_like(zs))
    lp = torch.log_softmax(zs, 1)
    p = lp.exp()
    lp0 = torch.where(p > 0, lp, torch.zeros_like(lp))
    logp = lp.gather(1, a[:, None])[:, 0]
    r = (logp - logp_old).exp()
    rc = r.clamp(1 - clip[0], 1 + clip[1])
    inside = r * adv <= rc * adv
    pg = -torch.where(inside, r * adv, (rc * adv).detach())
    H = -(p * lp0).sum(1)
    kl = torch.zeros_like(logp)
    if zr is not None:
        zq = torch.where((used & alive)[:, None], zr.double().cpu(), torch.zeros_like(zs))
        lq = torch.log_softmax(zq, 1)
        kl = (p * torch.where(p > 0, lp0 - lq, torch.zeros_like(lp))).sum(1)
    elif logp_ref is not None:
        d = logp_ref.double().cpu() - logp
        kl = d.exp() - 1 - d
    live = used & alive
    zero = torch.zeros_like(logp)
    row = torch.where(live, pg + kl_coef * kl - entropy_coef * H, zero)
    loss = (torch.where(live, w, zero) * row).sum()
    g, = torch.autograd.grad(loss, z)
    g = torch.where(live[:, None], g, torch.zeros_like(g))
    pick = lambda x: torch.where(live, x.detach(), zero)  # noqa: E731
    sums = [(w * pick(x)).sum() for x in (row, pg, kl, H, (~inside).double())]
    return dict(grad=g, kl=pick(kl), entropy=pick(H), logp=torch.where(live, logp.detach(), torch.where(used, -math.inf, 0.0)),
                stats=torch.stack(sums + [w.sum(), pick(kl)[used].max() if used.any() else zero.sum(), (w * pick(r)).sum()]),
                hits=int((live & ~inside).sum()))


def inputs(t, v, dtype, seed, pad=0, offset=0):
    g = torch.Generator("cuda").manual_seed(seed)
    def rows():  # rows of v elements inside a wider matrix, its base `offset` elements off
        flat = torch.full((offset + t * (v + pad),), float("nan"), device="cuda", dtype=dtype)
        return flat[offset:].view(t, v + pad)[:, :v]
    z, zr = rows(), rows()
    base = torch.randn((t, v), device="cuda", generator=g) * 2
    z.copy_(base)
    zr.copy_(base + 0.3 * torch.randn((t, v), device="cuda", generator=g))
    a = torch.randint(0, v, (t,), device="cuda", generator=g)
    lp = torch.log_softmax(z.double(), 1).gather(1, a[:, None])[:, 0]
    logp_old = (lp + 0.2 * torch.randn(t, device="cuda", generator=g)).float()
    logp_ref = (lp + 0.3 * torch.randn(t, device="cuda", generator=g)).float()
    adv = torch.randn(t, device="cuda", generator=g)
    w = (torch.rand(t, device="cuda", generator=g) > 0.2).float() * torch.rand(t, device="cuda", generator=g)
    w[t // 2] = 1.0
    return dict(z=z, zr=zr, a=a, logp_old=logp_old, logp_ref=logp_ref, adv=adv, w=w)


def check(out, want, dtype, grad_scale):
    """Tolerances.  A logit difference in base 2 carries 2^-23 relative, an exponential 2^-22, sums of them less; log-
    probabilities and entropies here stay below 40, KL below 10: 40 * 2^-22 < 1e-5 absolute.  A gradient element is
    rounded once, half a step of its type, on top of the same relative error of its factors, whose cancelling terms
    are as large as the row's largest coefficient (`grad_scale`) times p_v <= 1."""
    for k in ("logp", "kl", "entropy"):
        np.testing.assert_allclose(out[k].double().cpu().numpy(), want[k].numpy(), rtol=4e-6, atol=1e-5, err_msg=k)
    np.testing.assert_allclose(out["stats"].double().cpu().numpy(), want["stats"].numpy(), rtol=1e-5,
                               atol=2e-5 * max(1.0, float(want["stats"][5].abs())))
    if out["grad"] is not None:
        got, g = out["grad"].double().cpu(), want["grad"]
        half = torch.finfo(dtype).eps / 2
        tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        tol = half * 1.01 * g.abs() + 2e-5 * grad_scale * torch.softmax(want["z"], 1) + 1e-5 * grad_scale * want["onehot"] + tiny
        bad = (got - g).abs() > tol
        assert not bad.any(), (int(bad.sum()), float((got - g).abs().max()), grad_scale)


def run(s, dtype, ref, clip=(0.2, 0.2), kl_coef=0.05, entropy_coef=0.02, grad=True, actions=None):
    import paper_2211_15023_b200 as P
    kw = dict(logits_ref=s["zr"]) if ref == "logits" else dict(logp_ref=s["logp_ref"]) if ref == "logp" else {}
    want = definition(s["z"], s["a"], s["logp_old"], s["adv"], s["w"], s["zr"] if ref == "logits" else None,
                      s["logp_ref"] if ref == "logp" else None, clip, kl_coef, entropy_coef)
    zz = s["z"].double().cpu()
    want["z"] = torch.nan_to_num(zz, nan=0.0, neginf=-1e30)
    want["onehot"] = torch.nn.functional.one_hot(s["a"].long().cpu(), zz.shape[1]).double()
    out = P.policy_loss(s["z"], s["a"] if actions is None else s["a"].to(actions), s["logp_old"], s["adv"], weights=s["w"],
                        clip=clip, kl_coef=kl_coef, entropy_coef=entropy_coef, grad=grad, **kw)
    return out, want


def scale_of(s):
    ratio = 5.0  # the largest ratio that inputs() draws: exp(0.2 * 5 + rounding) with room
    return float((s["w"].abs() * (s["adv"].abs() * ratio + 20)).max())


# both sides of every choice of kernel: lanes a row (8, 16, 32, 64 actions), a warp (65 .. 2041 and 4-byte 1021), CTAs, clusters
SIZES = [(1, 1), (3, 2), (160, 18), (5, 8), (77, 9), (33, 64), (31, 65), (129, 255), (9, 1021), (7, 1024), (6, 2041),
         (5, 2049), (4, 4097), (3, 16385), (2, 33000), (2, 70001), (1, 131057)]


@pytest.mark.parametrize("t,v", SIZES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("ref", ["none", "logp", "logits"])
def test_loss_and_gradient_match_the_definition(t, v, dtype, ref):
    s = inputs(t, v, TYPES[dtype], 1000 * t + v)
    out, want = run(s, TYPES[dtype], ref)
    check(out, want, TYPES[dtype], scale_of(s))


@pytest.mark.parametrize("t,v", [(1, 262128), (2, 140000)])
def test_the_largest_vocabularies(t, v):
    for dtype in ("fp32", "bf16"):
        s = inputs(t, v, TYPES[dtype], v)
        out, want = run(s, TYPES[dtype], "logits")
        check(out, want, TYPES[dtype], scale_of(s))


@pytest.mark.parametrize("pad,offset", [(3, 0), (8, 1), (0, 5), (1, 7)])
@pytest.mark.parametrize("t,v", [(13, 18), (11, 301), (5, 5003), (3, 40001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_at_any_distance_and_alignment(t, v, dtype, pad, offset):
    """Rows of a wider matrix, bases off 16 bytes; the gradient aligned alike, otherwise, and in place."""
    import paper_2211_15023_b200 as P
    s = inputs(t, v, TYPES[dtype], t + v, pad, offset)
    out, want = run(s, TYPES[dtype], "logits")
    check(out, want, TYPES[dtype], scale_of(s))
    for lie in (offset, (offset + 3) % 8):
        g = torch.full((lie + t * (v + pad),), 7.0, device="cuda", dtype=TYPES[dtype])
        view = g[lie:].view(t, v + pad)[:, :v]
        out2, _ = run(s, TYPES[dtype], "logits", grad=view)
        assert torch.equal(out2["grad"], out["grad"])
        assert (g[:lie] == 7).all() and (g[lie:].view(t, v + pad)[:, v:] == 7).all()
    z = s["z"]
    r = P.policy_loss(z, s["a"], s["logp_old"], s["adv"], weights=s["w"], logits_ref=s["zr"], kl_coef=0.05,
                      entropy_coef=0.02, grad=z)
    assert r["grad"] is z and torch.equal(z, out["grad"]) and torch.equal(r["stats"], out["stats"])


@pytest.mark.parametrize("v", [18, 700, 9000, 60000])
@pytest.mark.parametrize("ref", ["none", "logits"])
def test_masked_logits_rows_and_weights(v, ref):
    """-inf and the type's lowest value as masks; a row that its mask empties; rows of weight 0 that hold NaN."""
    for dtype in (torch.float32, torch.bfloat16):
        s = inputs(8, v, dtype, v)
        s["w"][:] = 0.5
        low = torch.finfo(dtype).min
        keep = s["a"].clone()
        s["z"][0, 1:v // 2] = -math.inf
        s["z"][1, v // 2:] = low
        s["z"][2, :] = -math.inf          # nothing left
        s["z"][3, :] = low                # every logit the lowest: uniform
        s["z"][4, :] = float("nan")       # padding
        s["zr"][4, :] = float("nan")
        s["w"][4] = 0.0
        s["z"][5, 1:] = -math.inf         # one action only
        s["a"][0], s["a"][1], s["a"][5] = 0, 0, 0
        s["zr"][0, 1:v // 2] = -math.inf  # masked in the reference too
        lp = torch.log_softmax(s["z"].double(), 1).gather(1, s["a"][:, None])[:, 0]
        s["logp_old"] = torch.nan_to_num(lp + 0.1, nan=0.0, neginf=0.0).float()
        del keep
        out, want = run(s, dtype, ref)
        check(out, want, dtype, scale_of(s))
        assert not out["grad"][2].any() and not out["grad"][4].any() and out["logp"][2] == -math.inf and out["logp"][4] == 0
        assert not out["grad"][0, 1:v // 2].any()


def test_clip_boundaries_infinite_clips_and_64_bit_actions():
    s = inputs(512, 33, torch.float32, 3)
    for clip in ((0.0, 0.0), (0.1, 0.3), (math.inf, math.inf), (0.2, math.inf)):
        out, want = run(s, torch.float32, "none", clip=clip)
        check(out, want, torch.float32, scale_of(s))
        out32, _ = run(s, torch.float32, "none", clip=clip, actions=torch.int32)
        assert torch.equal(out32["grad"], out["grad"]) and torch.equal(out32["stats"], out["stats"])


@pytest.mark.parametrize("v", [18, 300, 20000])
def test_an_action_outside_the_row_is_nan_there_and_nowhere_else(v):
    import paper_2211_15023_b200 as P
    s = inputs(6, v, torch.float32, v)
    s["w"][:] = 1.0
    a = s["a"].clone()
    a[2], a[3] = v, -1
    r = P.policy_loss(s["z"], a, s["logp_old"], s["adv"], weights=s["w"], kl_coef=0.0)
    bad = torch.tensor([False, False, True, True, False, False], device="cuda")
    assert torch.equal(torch.isnan(r["grad"]).all(1), bad) and torch.equal(torch.isnan(r["logp"]), bad)
    assert torch.isnan(r["stats"][0])


def test_without_weights_every_row_counts_alike_and_no_gradient_is_optional():
    import paper_2211_15023_b200 as P
    s = inputs(100, 77, torch.float32, 5)
    a = P.policy_loss(s["z"], s["a"], s["logp_old"], s["adv"], entropy_coef=0.1)
    w = torch.full((100,), 0.01, device="cuda")
    b = P.policy_loss(s["z"], s["a"], s["logp_old"], s["adv"], weights=w, entropy_coef=0.1, grad=False)
    assert b["grad"] is None
    torch.testing.assert_close(a["stats"], b["stats"], rtol=1e-6, atol=1e-7)


def test_gradient_against_differences_of_the_loss():
    """Central differences of the returned loss: fp32 rows, one logit moved at a time.  The loss is about 1 and right to
    1e-6 at worst, the step 2e-2: an error of 1e-6 / 4e-2 = 2.5e-5 of the difference, and h^2 / 6 = 7e-5 times the third
    derivative (below 3 here) of the formula."""
    import paper_2211_15023_b200 as P
    s = inputs(4, 6, torch.float32, 11)
    s["w"][:] = 0.25
    f = lambda z: float(P.policy_loss(z, s["a"], s["logp_old"], s["adv"], weights=s["w"], logits_ref=s["zr"],  # noqa: E731
                                      clip=math.inf, kl_coef=0.5, entropy_coef=0.3, grad=False)["stats"][0])
    g = P.policy_loss(s["z"], s["a"], s["logp_old"], s["adv"], weights=s["w"], logits_ref=s["zr"], clip=math.inf,
                      kl_coef=0.5, entropy_coef=0.3)["grad"]
    h = 2e-2
    for t in range(4):
        for v in range(6):
            up, down = s["z"].clone(), s["z"].clone()
            up[t, v] += h
            down[t, v] -= h
            assert abs((f(up) - f(down)) / (2 * h) - float(g[t, v])) < 3e-4


def test_many_rows_sum_in_a_fixed_order():
    import paper_2211_15023_b200 as P
    for t in (1024, 1025, 8192, 8193, 40000):
        s = inputs(t, 6, torch.float32, t)
        out, want = run(s, torch.float32, "logp")
        check(out, want, torch.float32, scale_of(s))
        again, _ = run(s, torch.float32, "logp")
        assert torch.equal(out["stats"], again["stats"]) and torch.equal(out["grad"], again["grad"])


def test_captured_and_replayed_beside_another_stream():
    import paper_2211_15023_b200 as P
    s, other = inputs(64, 5000, torch.bfloat16, 1), inputs(64, 5000, torch.bfloat16, 2)
    call = lambda x: P.policy_loss(x["z"], x["a"], x["logp_old"], x["adv"], weights=x["w"], logits_ref=x["zr"], kl_coef=0.1)  # noqa: E731
    want, want_other = call(s), call(other)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(s)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for x in (s, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(x))
        graphs.append(g)
    for _ in range(5):
        for o in outs:
            o["grad"].zero_()
            o["stats"].zero_()
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, (want, want_other)):
            assert torch.equal(o["grad"], w["grad"]) and torch.equal(o["stats"], w["stats"])


@pytest.mark.parametrize("dtype,v,ref", [("bf16", 70001, "logits"), ("fp32", 70003, "none"), ("fp16", 66000, "logits"),
                                         ("bf16", 140007, "logp")])
def test_many_very_long_rows_that_are_streamed(dtype, v, ref):
    """A row for every SM and more: rows of weight 0 and NaN, masks, rows with nothing left, a reference without a
    probability that the policy has; the gradient apart, in place and not wanted; against the definition row by row."""
    import paper_2211_15023_b200 as P
    dt, t = TYPES[dtype], 301
    s = inputs(t, v, dt, v)
    s["w"][:] = 0.5
    low = torch.finfo(dt).min
    s["z"][3, 1:v // 2] = -math.inf
    s["zr"][3, 1:v // 2] = -math.inf
    s["z"][4, v // 2:] = low
    s["z"][5, :] = -math.inf
    s["z"][6, :] = low
    s["z"][150, :] = float("nan")
    s["zr"][150, :] = float("nan")
    s["w"][150] = 0.0
    s["z"][299, 1:] = -math.inf
    s["z"][300, :] = -math.inf
    for i in (3, 4, 299):
        s["a"][i] = 0
    lp = torch.log_softmax(s["z"].double(), 1).gather(1, s["a"][:, None])[:, 0]
    s["logp_old"] = torch.nan_to_num(lp + 0.1, nan=0.0, neginf=0.0).float()
    s["logp_ref"] = torch.nan_to_num(lp - 0.2, nan=0.0, neginf=0.0).float()
    kw = dict(logits_ref=s["zr"]) if ref == "logits" else dict(logp_ref=s["logp_ref"]) if ref == "logp" else {}
    call = lambda grad, **k: P.policy_loss(s["z"], s["a"], s["logp_old"], s["adv"], weights=s["w"], kl_coef=0.05,  # noqa: E731
                                           entropy_coef=0.02, grad=grad, **k)
    out = call(True, **kw)
    P.device_check()
    some = torch.tensor([0, 1, 2, 3, 4, 5, 6, 147, 148, 149, 150, 151, 296, 299, 300], device="cuda")
    part = {k: x[some] for k, x in s.items()}
    _, want = run(part, dt, ref)
    got = {k: out[k][some] for k in ("logp", "kl", "entropy", "grad")}
    got["stats"] = torch.zeros(8)
    want["stats"] = torch.zeros(8, dtype=torch.float64)
    check(got, want, dt, scale_of(s))
    # the same rows through the kernels for few rows: the sums of all
    few = [P.policy_loss(s["z"][i:i + 43], s["a"][i:i + 43], s["logp_old"][i:i + 43], s["adv"][i:i + 43],
                         weights=s["w"][i:i + 43], kl_coef=0.05, entropy_coef=0.02,
                         **{k: x[i:i + 43] for k, x in kw.items()}) for i in range(0, t, 43)]
    total = sum(f["stats"][[0, 1, 2, 3, 4, 5, 7]].double() for f in few)
    torch.testing.assert_close(out["stats"][[0, 1, 2, 3, 4, 5, 7]].double(), total, rtol=1e-5, atol=1e-3)
    none = call(False, **kw)
    assert torch.equal(none["stats"], out["stats"]) and torch.equal(none["logp"], out["logp"])
    again = call(True, **kw)
    assert torch.equal(again["grad"], out["grad"]) and torch.equal(again["stats"], out["stats"])
    if ref == "logits":
        hole = s["zr"].clone()
        hole[7, 11] = -math.inf
        with_hole = call(True, logits_ref=hole)
        assert with_hole["kl"][7] == math.inf and torch.equal(with_hole["kl"][8:], out["kl"][8:])
        assert not torch.isfinite(with_hole["grad"][7]).all() and torch.equal(with_hole["grad"][8:], out["grad"][8:])
    inplace = call(s["z"], **kw)
    assert torch.equal(s["z"], out["grad"]) and torch.equal(inplace["stats"], out["stats"])
    P.device_check()
