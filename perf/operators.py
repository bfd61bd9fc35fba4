"""The operators of training and serving an int8 policy over tokens, as cases that can be measured and compared.

``linear_i8``: a layer of int8 weights with a scale per channel on activations that are quantised on the way with a scale
per token.  ``ckpt_save`` / ``ckpt_load`` / ``ckpt_act_backward`` / ``ckpt_weight_grad``: activations kept in 8 bits for the
backward pass (blocks of 32 values share a power of two), and the two products that read them there.  ``policy_loss``: the
clipped policy loss with its KL and entropy terms over rows of logits, and its gradient.

``own`` chooses between elementary torch operations (the plain form) and the library's entry points.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of one sequence through a square projection: weights are read, little is computed
        dict(name="linear_one_token", op="linear", t=1, k=4096, n=4096, dtype="bf16", bias=False, relu=False),
        # a decode step of some tens of sequences through an up projection
        dict(name="linear_decode_batch", op="linear", t=24, k=4096, n=14336, dtype="bf16", bias=False, relu=False),
        # the hidden layer of the Atari network (3136 -> 512) with activations quantised per state, as in training
        dict(name="linear_hidden_8192", op="linear", t=8192, k=3136, n=512, dtype="fp32", bias=True, relu=True),
        # a long batch of prompts
        dict(name="linear_prompt_batch", op="linear", t=8192, k=4096, n=14336, dtype="bf16", bias=False, relu=False),
        # the Actor batch of the paper, hidden layer of 512 features: latency
        dict(name="keep_hidden_160", op="keep", t=160, k=512, act="relu", dtype="fp32"),
        # the widest activations of a token network, kept and read back
        dict(name="keep_wide_gelu", op="keep", t=8192, k=14336, act="gelu", dtype="bf16"),
        # their backward pass, ragged sizes
        dict(name="act_backward_silu", op="act_backward", t=4099, k=10922, act="silu", dtype="fp16"),
        # weight gradient of the residual network's hidden layer (2592 -> 256), an odd number of states
        dict(name="weight_grad_hidden", op="weight_grad", t=2047, k=2592, n=256, dtype="fp16", out="fp16"),
        # weight gradient of a square projection into 32-bit main gradients
        dict(name="weight_grad_tokens", op="weight_grad", t=8192, k=4096, n=4096, dtype="bf16", out="fp32"),
        # one Actor step's states of an Atari policy with 18 actions
        dict(name="loss_atari_160", op="loss", t=160, v=18, dtype="fp32", ref="none"),
        # a padded batch of sequences over an odd vocabulary, the reference known by its log-probs
        dict(name="loss_tokens_ref_logp", op="loss", t=4096, v=49999, dtype="bf16", ref="logp"),
        # the full KL against the reference's logits over a large vocabulary
        dict(name="loss_tokens_ref_logits", op="loss", t=2048, v=128001, dtype="bf16", ref="logits"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "keep", "act_backward", "weight_grad", "loss"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "linear":
        t, k, n = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192), _log_int(rng, 16, 16384)
        return dict(op=op, t=min(t, 8192 * 4096 * 14336 // (k * n)), k=k, n=n, dtype=dtype,
                    bias=rng.random() < 0.5, relu=rng.random() < 0.3)
    if op == "weight_grad":
        t, k, n = _log_int(rng, 1, 16384), _log_int(rng, 32, 8192), _log_int(rng, 16, 8192)
        dtype = rng.choice(("bf16", "fp16"))
        return dict(op=op, t=min(t, 8192 * 4096 * 4096 // (k * n)), k=k, n=n, dtype=dtype,
                    out=rng.choice((dtype, "fp32")))
    if op == "loss":
        v = _log_int(rng, 2, 128001)
        t = min(_log_int(rng, 1, 131072), 2048 * 128001 // (v * (2 if dtype == "fp32" else 1)))
        return dict(op=op, t=t, v=v, dtype=dtype, ref=rng.choice(("none", "logp", "logits")))
    t, k = _log_int(rng, 1, 8192), _log_int(rng, 16, 14336)
    return dict(op=op, t=t if dtype != "fp32" else max(1, t // 2), k=k, act=rng.choice(("none", "relu", "gelu", "silu")), dtype=dtype)


def work(case):
    t, es = case["t"], 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "linear":
        k, n = case["k"], case["n"]
        return dict(bytes=t * k * es + n * k + 4 * n * (2 if case["bias"] else 1) + t * n * es, flops=2 * t * n * k)
    if case["op"] == "weight_grad":
        k, n = case["k"], case["n"]
        return dict(bytes=t * n * es + t * k * 33 / 32 + (n * k + n) * (4 if case["out"] == "fp32" else 2), flops=2 * t * n * k)
    if case["op"] == "loss":
        v = case["v"]
        return dict(bytes=t * v * es * (3 if case["ref"] == "logits" else 2) + t * 4 * 8, flops=t * v * 8)
    k = case["k"]
    if case["op"] == "keep":  # x in; y and the checkpoint out; the checkpoint in and its values out
        return dict(bytes=t * k * (3 * es + 2 * 33 / 32), flops=t * k * 10)
    return dict(bytes=t * k * (2 * es + 33 / 32), flops=t * k * 10)


# --------------------------------------------------------------------------------- inputs
def _aligned_rows(rows, cols, dtype, device="cuda"):
    """[rows, cols] whose rows start at multiples of 32 bytes."""
    pad = -(-cols // 32) * 32
    return torch.empty((rows, pad), dtype=dtype, device=device)[:, :cols]


def _activations(g, t, k, dtype):
    """Tokens of different norms, and a few channels that stand out, as hidden states have them."""
    x = torch.randn((t, k), device="cuda", generator=g)
    x *= torch.exp(0.5 * torch.randn((t, 1), device="cuda", generator=g))
    channel = torch.ones(k, device="cuda")
    channel[torch.randint(0, k, (max(1, k // 256),), device="cuda", generator=g)] = 8.0
    return (x * channel).to(dtype)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    dtype, t = TYPES[case["dtype"]], case["t"]
    s = dict(case)
    if case["op"] == "linear":
        k, n = case["k"], case["n"]
        s["x"] = _activations(g, t, k, dtype)
        w = torch.randn((n, k), device="cuda", generator=g) * (1.0 / math.sqrt(k))
        q, s["ws"] = _quantised_rows(w)
        s["wq"] = _aligned_rows(n, k, torch.int8)
        s["wq"].copy_(q)
        s["bias"] = torch.randn(n, device="cuda", generator=g) * 0.1 if case["bias"] else None
    elif case["op"] == "loss":
        v = case["v"]
        z = torch.randn((t, v), device="cuda", generator=g) * 2.0
        s["logits"] = z.to(dtype)
        z = s["logits"].float()
        noise = torch.rand((t, v), device="cuda", generator=g).clamp_(1e-12, 1.0).log_().neg_().log_()
        s["actions"] = (z - noise).argmax(1).int()
        del noise
        logp = z.gather(1, s["actions"].long()[:, None])[:, 0] - torch.logsumexp(z, 1)
        s["logp_old"] = logp + 0.15 * torch.randn(t, device="cuda", generator=g)
        s["advantages"] = torch.randn(t, device="cuda", generator=g)
        s["logp_ref"] = logp + 0.3 * torch.randn(t, device="cuda", generator=g) if case["ref"] == "logp" else None
        s["logits_ref"] = None
        if case["ref"] == "logits":
            s["logits_ref"] = (z + 0.3 * torch.randn((t, v), device="cuda", generator=g)).to(dtype)
        # one token in eight is padding; the mean is over the others
        keep = (torch.rand(t, device="cuda", generator=g) >= 0.125).float()
        keep[0] = 1.0
        # (fp16 gradients of a mean underflow: training in fp16 scales its loss)
        s["weights"] = keep / keep.sum() * (1024.0 if case["dtype"] == "fp16" else 1.0)
    else:
        x = _activations(g, t, case["k"], dtype)
        if case["op"] == "keep":
            s["x"] = x
            return s
        q, e = _blocks_of_32(x.float())
        s["q"], s["e"] = q, e
        cols = case["n"] if case["op"] == "weight_grad" else case["k"]
        s["dy"] = (torch.randn((t, cols), device="cuda", generator=g) * 0.05).to(dtype)
    return s


# ----------------------------------------------------------------------------- plain forms
def _quantised_rows(x):
    """int8 rows and their scales: s = max |x| / 127 and q = rint(x / s), both divisions rounded to 32 bits."""
    s = x.abs().amax(1) / torch.full((1,), 127.0, device=x.device)
    q = torch.round(x / torch.where(s > 0, s, torch.ones_like(s))[:, None]).clamp_(-127, 127)
    return q.to(torch.int8), s


def _blocks_of_32(x):
    """The checkpoint of fp32 x [t, k]: q int8 [t, kp] and e uint8 [t, kp / 32], kp = k rounded up to 32; values are
    q 2^(e - 127), 2^(e - 127) the smallest power of two that leaves |q| <= 127."""
    t, k = x.shape
    kp = -(-k // 32) * 32
    b = torch.zeros((t, kp), device=x.device)
    b[:, :k] = x
    b = b.view(t, kp // 32, 32)
    bits = b.abs().amax(2).view(torch.int32)
    e = (((bits + 0x10000) >> 23) - 6).clamp_(min=1)
    q = torch.round(b / (e << 23).view(torch.float32)[:, :, None])
    return q.to(torch.int8).view(t, kp), e.to(torch.uint8)


def _values(q, e, k):
    scale = (e.int() << 23).view(torch.float32)
    return (q.float().view(q.shape[0], -1, 32) * scale[:, :, None]).view(q.shape[0], -1)[:, :k]


def _act(x, act):
    if act == "relu":
        return x.clamp_min(0)
    if act == "gelu":
        return 0.5 * x * torch.special.erfc(x * -math.sqrt(0.5))
    return x / (1 + torch.exp(-x)) if act == "silu" else x


def _act_slope(x, act):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "gelu":
        return 0.5 * torch.special.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        sig = 1 / (1 + torch.exp(-x))
        return sig * (1 + x * (1 - sig))
    return torch.ones_like(x)


CLIP, KL_COEF, ENTROPY_COEF = 0.2, 0.05, 0.02


def _plain_loss(s):
    z, a = s["logits"].float(), s["actions"].long()[:, None]
    w = s["weights"]
    # a log-probability, and more so the difference of two, is a small difference of large numbers: 64 bits
    lse = torch.logsumexp(z.double(), 1, keepdim=True)
    logq = z.double() - lse
    logp = logq.gather(1, a)[:, 0]
    p = torch.exp(logq.float())
    entropy = -(p.double() * logq).sum(1)
    ratio = torch.exp(logp - s["logp_old"].double())
    adv = s["advantages"].double()
    clipped = ratio.clamp(1 - CLIP, 1 + CLIP)
    pg = -torch.minimum(ratio * adv, clipped * adv)
    slope = torch.where(ratio * adv <= clipped * adv, -ratio * adv, torch.zeros_like(adv))
    kl = torch.zeros_like(logp)
    d = ENTROPY_COEF * p * (logq.float() + entropy.float()[:, None])
    if s["logits_ref"] is not None:
        zr = s["logits_ref"].double()
        delta = logq - (zr - torch.logsumexp(zr, 1, keepdim=True))
        kl = (torch.exp(logq) * delta).sum(1)
        d += KL_COEF * p * (delta - kl[:, None]).float()
    elif s["logp_ref"] is not None:
        diff = s["logp_ref"].double() - logp
        kl = torch.expm1(diff) - diff
        slope = slope - KL_COEF * torch.expm1(diff)
    d -= slope.float()[:, None] * p
    d.scatter_add_(1, a, slope.float()[:, None])
    d *= w[:, None]
    wd = w.double()
    used = w > 0
    per_row = [torch.where(used, v, torch.zeros_like(v)) for v in (logp, kl, entropy)]
    hit = ((ratio * adv) > (clipped * adv)).double()
    sums = [(wd * v).sum() for v in (pg + KL_COEF * kl - ENTROPY_COEF * entropy, pg, kl, entropy, hit)]
    return dict(loss=sums[0].float(), stats=torch.stack(sums[1:]).float(), grad=d.to(s["logits"].dtype),
                logp=per_row[0].float(), kl=per_row[1].float(), entropy=per_row[2].float())


def run(state):
    s, op = state, state["op"]
    if own:
        return _own(s)
    if op == "linear":
        q, scale = _quantised_rows(s["x"].float())
        y = (q.float() @ s["wq"].float().t()) * (scale[:, None] * s["ws"][None, :])
        if s["bias"] is not None:
            y += s["bias"]
        return (y.clamp_min_(0) if s["relu"] else y).to(s["x"].dtype)
    if op == "keep":
        x = s["x"].float()
        q, e = _blocks_of_32(x)
        return _act(x, s["act"]).to(s["x"].dtype), _values(q, e, s["k"]).to(s["x"].dtype)
    if op == "act_backward":
        return (s["dy"].float() * _act_slope(_values(s["q"], s["e"], s["k"]), s["act"])).to(s["dy"].dtype)
    if op == "weight_grad":
        dy = s["dy"].float()
        return ((dy.t() @ _values(s["q"], s["e"], s["k"])).to(TYPES[s["out"]]), dy.sum(0).to(TYPES[s["out"]]))
    return _plain_loss(s)


def _own(s):
    import paper_2211_15023_b200 as P
    op = s["op"]
    if op == "linear":
        return P.linear_i8(s["x"], (s["wq"], s["ws"]), bias=s["bias"], relu=s["relu"])
    if op == "keep":
        y, ckpt = P.ckpt_save(s["x"], act=s["act"])
        return y, P.ckpt_load(ckpt, s["k"], s["x"].dtype)
    if op == "act_backward":
        return P.ckpt_act_backward(s["dy"], (s["q"], s["e"]), act=s["act"])
    if op == "weight_grad":
        return P.ckpt_weight_grad(s["dy"], (s["q"], s["e"]), s["k"], out_dtype=TYPES[s["out"]])
    r = P.policy_loss(s["logits"], s["actions"], s["logp_old"], s["advantages"], weights=s["weights"],
                      logits_ref=s["logits_ref"], logp_ref=s["logp_ref"], clip=CLIP, kl_coef=KL_COEF,
                      entropy_coef=ENTROPY_COEF)
    return dict(loss=r["stats"][0], stats=r["stats"][1:5], grad=r["grad"], logp=r["logp"], kl=r["kl"], entropy=r["entropy"])


# ---------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "linear":
        x = s["x"].double()
        scale = (x.abs().max(1).values / 127.0).float().double()
        ok = scale > 0
        q = torch.where(ok[:, None], x / torch.where(ok, scale, 1.0)[:, None], 0.0).float().round().clamp(-127, 127)
        y = q.double() @ s["wq"].double().t()
        # (the product of the two scales is rounded to 32 bits by definition)
        y *= (scale.float()[:, None] * s["ws"][None, :]).double()
        y = y if s["bias"] is None else y + s["bias"].double()
        return torch.relu(y) if s["relu"] else y
    if op == "loss":
        return _exact_loss(s)
    if op == "keep":
        x, k = s["x"].double(), s["k"]
        kp = -(-k // 32) * 32
        b = torch.nn.functional.pad(x, (0, kp - k)).view(x.shape[0], -1, 32)
        top = b.abs().amax(2)
        power = torch.frexp(top).exponent.double() - 7  # top / 2^power lies in [64, 128)
        power = torch.where(torch.round(top / torch.exp2(power)) > 127, power + 1, power).clamp(min=-126)
        step = torch.exp2(power)[:, :, None]
        return _exact_act(x, s["act"])[0], (torch.round(b / step) * step).view(x.shape[0], -1)[:, :k]
    kept = s["q"].double().view(case["t"], -1, 32) * torch.exp2(s["e"].double() - 127)[:, :, None]
    kept = kept.view(case["t"], -1)[:, :s["k"]]
    if op == "act_backward":
        return s["dy"].double() * _exact_act(kept, s["act"])[1]
    return torch.matmul(s["dy"].double().t(), kept), s["dy"].double().sum(0)


def _exact_act(x, act):
    """Value and slope of an activation, by its definition."""
    if act == "none":
        return x, torch.ones_like(x)
    if act == "relu":
        return torch.where(x > 0, x, 0.0), torch.where(x > 0, 1.0, 0.0).double()
    if act == "silu":
        up = torch.sigmoid(x)
        return x * up, up + x * up * torch.sigmoid(-x)
    cdf = torch.special.ndtr(x)
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def _exact_loss(s):
    """Row by row block, the gradient from the softmax's Jacobian applied to each term's own gradient."""
    t = s["t"]
    out = dict(loss=torch.zeros((), dtype=torch.float64, device="cuda"), stats=torch.zeros(4, dtype=torch.float64, device="cuda"),
               grad=torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda"),
               **{n: torch.zeros(t, dtype=torch.float64, device="cuda") for n in ("logp", "kl", "entropy")})
    step = max(1, (1 << 26) // s["v"])
    for i in range(0, t, step):
        rows = slice(i, min(t, i + step))
        z, w, adv = s["logits"][rows].double(), s["weights"][rows].double(), s["advantages"][rows].double()
        lp = torch.log_softmax(z, 1)
        p, pick = lp.exp(), torch.nn.functional.one_hot(s["actions"][rows].long(), s["v"])
        taken = (lp * pick).sum(1)
        r = (taken - s["logp_old"][rows].double()).exp()
        inside = r * adv <= r.clamp(1 - CLIP, 1 + CLIP) * adv
        pg = torch.where(inside, -r * adv, -r.clamp(1 - CLIP, 1 + CLIP) * adv)
        entropy = -(p * lp).sum(1)
        # d loss / d log p of every action, then through the log-softmax: g - p sum(g)
        g = torch.where(inside, -r * adv, 0.0)[:, None] * pick + ENTROPY_COEF * p * (lp + 1)
        kl = torch.zeros_like(taken)
        if s["logits_ref"] is not None:
            d = lp - torch.log_softmax(s["logits_ref"][rows].double(), 1)
            kl = (p * d).sum(1)
            g = g + KL_COEF * p * (d + 1)
        if s["logp_ref"] is not None:
            d = s["logp_ref"][rows].double() - taken
            kl = d.exp() - 1 - d
            g = g + (KL_COEF * (1 - d.exp()))[:, None] * pick
        out["grad"][rows] = w[:, None] * (g - p * g.sum(1, keepdim=True))
        out["loss"] += (w * (pg + KL_COEF * kl - ENTROPY_COEF * entropy)).sum()
        out["stats"] += torch.stack([(w * v).sum() for v in (pg, kl, entropy, (~inside).double())])
        for n, v in (("logp", taken), ("kl", kl), ("entropy", entropy)):
            out[n][rows] = torch.where(w > 0, v, 0.0)
    return out
