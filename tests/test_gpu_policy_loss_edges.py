"""The clipped policy loss where masks, references and offsets are extreme, over widths that reach each of its kernels."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_policy_loss import TYPES, check, definition, inputs, scale_of  # noqa: E402

# (rows, actions): a group of lanes a row, a warp, a CTA, a cluster, streamed (148 rows and more, 256 KB of both arrays)
WIDTHS = [(8, 18), (8, 300), (8, 9000), (8, 60000), (301, 70001)]


def some_of(s, rows=16):
    """The first rows, where a case puts what it is about, for the definition in 64 bits."""
    return {k: x[:rows] for k, x in s.items()}


def loss(s, ref="logits", grad=True, **kw):
    import paper_2211_15023_b200 as P
    kw.update(dict(logits_ref=s["zr"]) if ref == "logits" else dict(logp_ref=s["logp_ref"]) if ref == "logp" else {})
    out = P.policy_loss(s["z"], s["a"], s["logp_old"], s["adv"], weights=s["w"], grad=grad, **kw)
    P.device_check()
    return out


def against_definition(s, out, dtype, ref="logits", rows=16, **kw):
    """The first rows' outputs and gradients (and the sums, where these are all rows)."""
    part = some_of(s, rows)
    want = definition(part["z"], part["a"], part["logp_old"], part["adv"], part["w"], part["zr"] if ref == "logits" else None,
                      part["logp_ref"] if ref == "logp" else None, **kw)
    z = part["z"].double().cpu()
    want["z"] = torch.nan_to_num(z, nan=0.0, neginf=-1e30)
    want["onehot"] = torch.nn.functional.one_hot(part["a"].long().cpu(), z.shape[1]).double()
    got = {k: out[k][:rows] for k in ("logp", "kl", "entropy", "grad")}
    got["stats"] = out["stats"]
    if s["z"].shape[0] > rows:
        got["stats"], want["stats"] = torch.zeros(8), torch.zeros(8, dtype=torch.float64)
    check(got, want, dtype, scale_of(part))
    assert not torch.isnan(got["grad"].cpu()[~torch.isnan(want["grad"])]).any()
    return want


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_vocabulary_padded_with_the_lowest_value_in_both_arrays(t, v, dtype):
    """Weights of a scaled loss: the reference's coefficient times the lowest value goes beyond fp32, the probability is 0."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v)
    pad = max(1, v // 20)
    s["z"][:, -pad:] = torch.finfo(dt).min
    s["zr"][:, -pad:] = torch.finfo(dt).min
    s["a"].zero_()
    s["z"][1::2, 0] += 20.0  # (a sum of probabilities near the largest)
    s["zr"][1::2, 0] += 20.0
    lp = torch.log_softmax(s["z"].double(), 1)[:, 0]
    s["logp_old"], s["w"] = (lp + 0.1).float(), torch.full_like(s["w"], 64.0)
    out = loss(s, kl_coef=0.05, entropy_coef=0.02)
    assert torch.isfinite(out["grad"]).all() and not out["grad"][:, -pad:].any()
    against_definition(s, out, dt, kl_coef=0.05, entropy_coef=0.02)


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_divergence_that_is_only_watched_does_not_touch_the_gradient(t, v, dtype):
    """kl_coef 0 and a reference without a probability that the policy has: an infinite KL, the loss without it."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v + 1)
    s["w"][:] = 0.5
    s["zr"][2, 3], s["zr"][5, v - 1], s["zr"][6, :] = -math.inf, -math.inf, -math.inf
    out = loss(s, kl_coef=0.0, entropy_coef=0.02)
    assert out["kl"][2] == math.inf and out["kl"][5] == math.inf and not torch.isfinite(out["kl"][6])
    assert torch.isfinite(out["grad"]).all() and torch.isfinite(out["stats"][[0, 1, 3, 4, 5, 7]]).all()
    out["kl"] = torch.zeros_like(out["kl"])
    out["stats"][[2, 6]] = 0.0
    against_definition(s, out, dt, ref="none", kl_coef=0.0, entropy_coef=0.02)


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_watched_divergence_of_the_actions_taken_does_not_touch_the_gradient(t, v, dtype):
    """kl_coef 0 and an action that the reference's log-probs hold for likely and the policy for (next to) impossible:
    exp(logp_ref - logp) goes beyond the range, the loss does without it."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v + 2)
    s["w"][:] = 0.5
    s["a"][:8] = 1
    s["z"][2, 1], s["z"][5, 1], s["z"][6, 1] = -100.0, -1000.0, -math.inf
    s["logp_old"][:8] = -3.0
    s["logp_ref"][:8] = -1.0
    out = loss(s, ref="logp", kl_coef=0.0, entropy_coef=0.02)
    assert out["kl"][2] > 1e38 and out["kl"][5] == math.inf and out["kl"][6] == math.inf
    assert torch.isfinite(out["grad"]).all() and torch.isfinite(out["stats"][[0, 1, 3, 4, 5, 7]]).all()
    s["z"][6, 1] = -200.0  # (the definition has no derivative at -inf; a probability of e^-200 moves nothing)
    part = some_of(s, 8)
    want = definition(part["z"], part["a"], part["logp_old"], part["adv"], part["w"], kl_coef=0.0, entropy_coef=0.02)["grad"]
    # (rounded once, with the tolerance of check() for the factors)
    p = torch.softmax(part["z"].double().cpu(), 1) + 0.5 * torch.nn.functional.one_hot(part["a"].cpu(), v)
    slack = 2e-5 * scale_of(part) * p + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    assert ((out["grad"][:8].double().cpu() - want).abs() <= torch.finfo(dt).eps / 2 * 1.01 * want.abs() + slack).all()


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("ref", ["none", "logp", "logits"])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_that_hold_nan_are_not_rows_that_a_mask_empties(t, v, ref, dtype):
    s = inputs(t, v, TYPES[dtype], v + 3)
    s["w"][:] = 0.5
    s["z"][1, :] = math.nan
    s["z"][2, :] = -math.inf
    s["z"][2, v // 2] = math.nan
    s["z"][3, v - 1] = math.nan
    s["z"][4, :] = -math.inf
    s["a"][1:5] = 0
    s["logp_old"][4] = -1.0
    out = loss(s, ref=ref, kl_coef=0.05 if ref != "none" else 0.0, entropy_coef=0.02)
    assert torch.isnan(out["logp"][1:4]).all() and torch.isnan(out["entropy"][1:4]).all() and torch.isnan(out["stats"][[0, 1, 3]]).all()
    assert torch.isnan(out["stats"][2]) == (ref != "none") and torch.isnan(out["kl"][1:4]).all() == (ref != "none")  # (0 with neither)
    assert torch.isnan(out["grad"][1]).all() and torch.isnan(out["grad"][2, v // 2]) and torch.isnan(out["grad"][3, v - 1])
    assert out["logp"][4] == -math.inf and not out["grad"][4].any() and not out["entropy"][4] and not out["kl"][4]
    assert torch.isfinite(out["grad"][5:]).all() and torch.isfinite(out["logp"][5:]).all()


@pytest.mark.parametrize("t,v", [(8, 18), (2000, 18), (9000, 18), (8, 300)])
def test_the_largest_divergence_is_nan_where_a_row_has_none(t, v):
    """(sums in the same launch, by one CTA, by a cluster)"""
    s = inputs(t, v, torch.float32, v + 4)
    s["w"][:] = 0.5
    s["zr"][1, 1] = math.nan
    assert torch.isnan(loss(s, kl_coef=0.05)["stats"][6])
    s["w"][1] = 0.0
    out = loss(s, kl_coef=0.05)
    assert out["stats"][6] == out["kl"].max()


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_ratios_beyond_fp32_times_small_advantages(t, v, dtype):
    """A behaviour log-prob of some -95: the ratio is infinite in fp32, its product with an advantage of 0 is 0, with one of
    -1e-3 it fits, with a positive one the clamp decides."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v + 5)
    s["w"][:] = 0.5
    lp = torch.log_softmax(s["z"][:8].double(), 1).gather(1, s["a"][:8, None])[:, 0]
    s["logp_old"][1:5] = (lp[1:5] - 92.0).float()
    s["adv"][1:5] = torch.tensor([0.0, -1e-3, 0.5, -0.0])
    out = loss(s, ref="none")
    part = some_of(s, 8)
    want = definition(part["z"], part["a"], part["logp_old"], part["adv"], part["w"])["grad"]
    # (a ratio carries the absolute error of the two log-probs, some 1e-5; the rest as in check())
    tol = torch.finfo(dt).eps / 2 * 1.01 * want.abs() + 5e-5 * want.abs().amax(1, keepdim=True) + torch.finfo(dt).smallest_normal
    assert ((out["grad"][:8].double().cpu() - want).abs() <= tol).all()
    assert not out["grad"][1].any() and not out["grad"][3].any() and not out["grad"][4].any() and out["grad"][2].any()
    assert float(out["stats"][0]) > 1e36 and torch.isfinite(out["stats"][[0, 1, 4, 5]]).all()


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("offset", [100.0, -1000.0, 3000.0])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_log_probabilities_do_not_depend_on_the_logits_offset(t, v, offset, dtype):
    """Logits around `offset` (one more offset a row: a part's maximum is not the row's), with every reference."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v + 6)
    for x in ("z", "zr"):
        s[x].copy_(s[x].float() + offset + torch.arange(t, device="cuda")[:, None] % 7)
    lp = torch.log_softmax(s["z"][:16].double(), 1).gather(1, s["a"][:16, None])[:, 0]
    s["logp_old"][:16] = (lp + 0.1).float()
    s["logp_ref"][:16] = (lp - 0.2).float()
    s["w"][1] = 1.0
    for ref in ("none", "logp", "logits"):
        out = loss(s, ref=ref, kl_coef=0.05, entropy_coef=0.02)
        against_definition(s, out, dt, ref=ref, kl_coef=0.05, entropy_coef=0.02)


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("value", ["lowest", -1e33, -2e30])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_reference_far_below_where_the_policy_is_not(t, v, value, dtype):
    """Finite reference logits below -1e30 in entries that the policy does not mask count as they are: the KL is p times
    them.  Beside entries that both mask, rows of which one or both hold nothing else, and a row of the reference with one
    further below than the rest."""
    dt = TYPES[dtype]
    value = torch.finfo(dt).min if value == "lowest" else value
    s = inputs(t, v, dt, v + 7)
    s["w"][:] = 0.5
    s["a"][:] = 0
    pad = max(1, v // 20)
    s["z"][:, -pad:] = torch.finfo(dt).min
    s["zr"][:, -pad:] = torch.finfo(dt).min
    s["zr"][1, 3] = value
    s["zr"][2, 2:v // 2] = value
    s["zr"][3, :-pad] = value                     # (what is masked in the policy lies below, or alike)
    s["z"][4, :], s["zr"][4, 1:] = value, value   # uniform, against one action
    s["z"][5, 2:], s["zr"][5, 1] = -math.inf, value
    s["zr"][6, 5] = -math.inf                     # an infinite divergence
    s["z"][7, :], s["zr"][7, :] = value, value    # uniform both
    s["zr"][7, 4] = torch.finfo(dt).min
    lp = torch.log_softmax(s["z"].double(), 1)[:, 0]
    s["logp_old"] = (lp + 0.1).float()
    out = loss(s, kl_coef=0.03125, entropy_coef=0.02)
    assert out["kl"][6] == math.inf and not torch.isfinite(out["grad"][6]).all()
    rows = [0, 1, 2, 3, 4, 5, 7]
    part = {k: x[rows] for k, x in s.items()}
    want = definition(part["z"], part["a"], part["logp_old"], part["adv"], part["w"], part["zr"], kl_coef=0.03125, entropy_coef=0.02)
    got = out["kl"][rows].double().cpu()
    torch.testing.assert_close(got, want["kl"], rtol=8e-6, atol=1e-5)
    torch.testing.assert_close(out["logp"][rows].double().cpu(), want["logp"], rtol=4e-6, atol=1e-5)
    # a gradient is w p (base + kl_coef (delta - KL) + ...): once rounded, with the relative error of p (some 2^-20, of an fp32
    # exponential and a sum of them) and of delta and KL, which cancel
    z, zr = part["z"].double().cpu(), part["zr"].double().cpu()
    p = torch.softmax(z, 1)
    delta = torch.where(p > 0, torch.log_softmax(z, 1) - torch.log_softmax(zr, 1), torch.zeros_like(p)).abs()
    slack = 2e-5 * p * (scale_of(part) + 0.5 * 0.03125 * (delta + want["kl"][:, None]))
    slack[:, 0] += 1e-5 * scale_of(part)
    g = out["grad"][rows].double().cpu()
    tol = torch.finfo(dt).eps / 2 * 1.01 * want["grad"].abs() + slack + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    assert torch.isfinite(g).all() and ((g - want["grad"]).abs() <= tol).all()
    assert not g[[0, 1, 2], -pad:].any()
    again = loss(s, grad=s["z"], kl_coef=0.03125, entropy_coef=0.02)
    assert torch.equal(torch.nan_to_num(again["grad"]), torch.nan_to_num(out["grad"])) and torch.equal(again["kl"], out["kl"])


@pytest.mark.parametrize("native", [True, False])
def test_the_gradient_of_each_sequence_s_last_token_takes_its_own_memory(native, monkeypatch):
    """Rows of a [batch, length, vocabulary] tensor that lie a whole sequence apart; on both ways in."""
    import types

    import paper_2211_15023_b200 as P
    from paper_2211_15023_b200 import binding
    s = inputs(64, 5003, torch.bfloat16, 1)
    whole = torch.zeros((64, 40, 5003), device="cuda", dtype=torch.bfloat16)
    whole[:, -1] = s["z"]
    call = lambda z: P.policy_loss(z, s["a"], s["logp_old"], s["adv"], weights=s["w"], entropy_coef=0.1)  # noqa: E731
    want = call(s["z"])
    if not native:
        monkeypatch.setattr(binding, "_CALLS", types.SimpleNamespace(policy_loss=lambda *a: None))
    before = torch.cuda.memory_allocated()
    got = call(whole[:, -1])
    assert torch.cuda.memory_allocated() - before < 2 * 64 * 5003 * 2
    # (rows that lie otherwise to 16 bytes are summed in another order: a gradient may round to its neighbour)
    torch.testing.assert_close(got["grad"].float(), want["grad"].float(), rtol=2.0 ** -7, atol=1e-8)
    torch.testing.assert_close(got["stats"], want["stats"], rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("dtype,t,v", [("bf16", 301, 151937), ("fp16", 299, 262128), ("fp32", 150, 131072)])
def test_streamed_rows_of_which_l2_does_not_hold_all(dtype, t, v):
    import paper_2211_15023_b200 as P
    s = inputs(t, v, TYPES[dtype], v)
    out = loss(s, kl_coef=0.05, entropy_coef=0.02)
    against_definition(s, out, TYPES[dtype], rows=6, kl_coef=0.05, entropy_coef=0.02)
    few = {k: x[-40:] for k, x in s.items()}  # (fewer rows than SMs: a cluster a row)
    other = loss(few, kl_coef=0.05, entropy_coef=0.02)
    for k in ("logp", "kl", "entropy"):
        torch.testing.assert_close(out[k][-40:], other[k], rtol=8e-6, atol=2e-5)
    assert torch.equal(loss(s, grad=s["z"], kl_coef=0.05, entropy_coef=0.02)["grad"], out["grad"])
    P.device_check()


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -1e20])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masks_that_are_added(t, v, mask, dtype):
    """A third of every row lies around `mask` in both arrays (parts of a row hold nothing else), some rows lie there whole, or
    as far up; rounded shifts of such parts are off by up to 2^39."""
    dt = TYPES[dtype]
    s = inputs(t, v, dt, v + 8)
    s["w"][:] = 0.5
    s["a"][:] = 0
    third = max(1, v // 3)
    for x in ("z", "zr"):
        s[x][:, -third:] = (s[x][:, -third:].float() + mask).to(dt)
        s[x][1] = (s[x][1].float() + mask).to(dt)
        s[x][2] = (s[x][2].float().clamp(min=-8) - 2 * mask).to(dt)
        s[x][3, 1:] = (s[x][3, 1:].float() + mask).to(dt)
    lp = torch.log_softmax(s["z"].double(), 1)[:, 0]
    s["logp_old"] = (lp.clamp(min=-30) + 0.1).float()
    s["logp_ref"] = (lp.clamp(min=-30) - 0.1).float()
    rows = [i for i in range(8) if float(lp[i]) > -1e5]  # (an action that a row's mask takes away has a log-prob near `mask`)
    for ref in ("none", "logits"):
        out = loss(s, ref=ref, kl_coef=0.05, entropy_coef=0.02)
        assert torch.isfinite(out["grad"]).all() and torch.isfinite(out["stats"]).all()
        part = {k: x[rows] for k, x in s.items()}
        sub = {k: (x[rows] if x is not None and x.shape[0] == t else x) for k, x in out.items()}
        sub["stats"] = None
        want = definition(part["z"], part["a"], part["logp_old"], part["adv"], part["w"], part["zr"] if ref == "logits" else None,
                          kl_coef=0.05, entropy_coef=0.02)
        want["z"] = part["z"].double().cpu()
        want["onehot"] = torch.nn.functional.one_hot(part["a"].long().cpu(), v).double()
        sub["stats"], want["stats"] = torch.zeros(8), torch.zeros(8, dtype=torch.float64)
        check(sub, want, dt, scale_of(part))
        assert not torch.isnan(sub["grad"]).any()


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("offset", [1e4, -1e5, 1e6, -2e7, 4e7, -1e9])
def test_gradients_do_not_depend_on_the_logits_offset(t, v, offset):
    """fp32 rows far from 0, on both sides of where they are kept relative to their maximum (a step of fp32 there is up to 64)."""
    s = inputs(t, v, torch.float32, v + 9)
    for x in ("z", "zr"):
        s[x].copy_(s[x] + offset)
    lp = torch.log_softmax(s["z"][:16].double(), 1).gather(1, s["a"][:16, None])[:, 0]
    s["logp_old"][:16] = (lp.clamp(min=-30) + 0.1).float()
    s["w"][1] = 1.0
    rows = [i for i in range(min(t, 16)) if float(lp[i]) > -40]
    s = {k: torch.cat([x[rows], x[len(rows):]]) for k, x in s.items()}
    for ref in ("none", "logits"):
        out = loss(s, ref=ref, kl_coef=0.5, entropy_coef=0.5)
        against_definition(s, out, torch.float32, ref=ref, rows=len(rows), kl_coef=0.5, entropy_coef=0.5)


@pytest.mark.parametrize("t,v", WIDTHS)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_broken_reference_that_is_only_watched(t, v, dtype):
    """NaN and infinities in the reference, kl_coef 0: its KL is not finite, the gradient is the loss's without it."""
    s = inputs(t, v, TYPES[dtype], v + 10)
    s["w"][:] = 0.5
    s["zr"][1, 2], s["zr"][2, v - 1], s["zr"][3, :], s["zr"][4, v // 2] = math.nan, math.nan, math.nan, math.inf
    out = loss(s, kl_coef=0.0, entropy_coef=0.02)
    assert torch.isnan(out["kl"][1:4]).all() and not torch.isfinite(out["kl"][4]) and torch.isfinite(out["kl"][5:]).all()
    alone = loss(s, ref="none", kl_coef=0.0, entropy_coef=0.02)
    half = torch.finfo(TYPES[dtype]).eps
    torch.testing.assert_close(out["grad"].float(), alone["grad"].float(), rtol=2 * half, atol=1e-6)
    broken = loss(s, kl_coef=0.05, entropy_coef=0.02)
    assert torch.isnan(broken["grad"][1]).any() and torch.isnan(broken["grad"][3]).any() and torch.isfinite(broken["grad"][5:]).all()


@pytest.mark.parametrize("dtype,t,v", [("fp32", 4, 80001), ("fp32", 40, 129830), ("fp32", 147, 77465), ("fp32", 2, 262128), ("bf16", 3, 150001),
                                       ("fp16", 2, 262128)])
@pytest.mark.parametrize("ref", ["none", "logp", "logits"])
def test_every_part_of_a_row_has_a_gradient(dtype, t, v, ref):
    """Rows that are split over up to sixteen CTAs, by the definition; no part without one."""
    s = inputs(t, v, TYPES[dtype], v)
    s["w"][:] = 0.5
    out = loss(s, ref=ref, kl_coef=0.05, entropy_coef=0.02)
    assert torch.isfinite(out["grad"]).all()
    against_definition(s, out, TYPES[dtype], ref=ref, rows=4, kl_coef=0.05, entropy_coef=0.02)
    sixteenths = out["grad"][0].float().abs().tensor_split(16)
    assert all(float(x.max()) > 0 for x in sixteenths)
