"""Calls on a stream that is named while torch's current stream is another one and busy: the memory that a call allocates is
not what work on the current stream still writes, and a result that is given back is not written again while the current
stream still reads it."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SLEEP = 40_000_000  # cycles: some 20 to 30 ms


def rand(*shape, seed=0):
    return torch.randn(shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


def flat(r):
    """The tensors of a result, in order."""
    if isinstance(r, torch.Tensor):
        return [r]
    return [t for x in (r.values() if isinstance(r, dict) else r) if x is not None for t in flat(x)]


def calls():
    """name -> a call with a stream; every entry that allocates, on both ways in (native, and the one that takes the rest)."""
    import paper_2211_15023_b200 as P
    x, w, z = rand(300, 1000).bfloat16(), P.quant_rows(rand(700, 1000, seed=1)), rand(200, 3000, seed=2)
    xq, bias = P.quant_rows(x), rand(700, seed=3)
    _, ckpt = P.ckpt_save(x)
    dy, big = rand(300, 701, seed=4).bfloat16()[:, :700], rand(300, 2001, seed=5).bfloat16()[:, :2000]
    _, wide = P.ckpt_save(rand(300, 4000, seed=6).bfloat16())
    a, f = torch.arange(200, device="cuda") * 3, rand(200, seed=7)
    lo = torch.full((200,), -8.0, device="cuda")
    logits, other, m = rand(5000, 18, seed=8), rand(5000, 18, seed=10), rand(20, 160, seed=9)
    out = torch.empty((300, 1000), device="cuda", dtype=torch.bfloat16)
    return {
        "quant_rows": lambda s: P.quant_rows(x, stream=s),
        "linear_i8": lambda s: P.linear_i8(x, w, bias, relu=True, stream=s),
        "linear_i8 of a pair": lambda s: P.linear_i8(xq, w, bias, stream=s),
        "ckpt_save": lambda s: P.ckpt_save(x, "gelu", stream=s),
        "ckpt_save into": lambda s: P.ckpt_save(x, "silu", out=out, stream=s)[1],
        "ckpt_load": lambda s: P.ckpt_load(ckpt, 1000, torch.float32, stream=s),
        "ckpt_act_backward": lambda s: P.ckpt_act_backward(x, ckpt, "gelu", stream=s),
        "ckpt_weight_grad, rows off 16 bytes": lambda s: P.ckpt_weight_grad(dy, ckpt, 1000, out_dtype=torch.float32, stream=s),
        "ckpt_weight_grad, read back": lambda s: P.ckpt_weight_grad(big, wide, 4000, stream=s),
        "policy_loss": lambda s: P.policy_loss(z, a, lo, f, kl_coef=0.1, logits_ref=z, stream=s),
        "kl": lambda s: P.kl(logits, other, stream=s),
        "vtrace": lambda s: P.vtrace(m, m, m, m, m[0].contiguous(), 0.99, stream=s),
    }


NAMES = ["quant_rows", "linear_i8", "linear_i8 of a pair", "ckpt_save", "ckpt_save into", "ckpt_load", "ckpt_act_backward",
         "ckpt_weight_grad, rows off 16 bytes", "ckpt_weight_grad, read back", "policy_loss", "kl", "vtrace"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_has_given_back_but_still_writes(name):
    call = calls()[name]
    want = [t.clone() for t in flat(call(None))]
    side = torch.cuda.Stream()
    call(side.cuda_stream)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for _ in range(3):
        blocks = [torch.empty(1 << i, dtype=torch.uint8, device="cuda") for i in range(9, 26) for _ in range(3)]
        torch.cuda._sleep(SLEEP)
        for _ in range(20):
            for b in blocks:
                b.fill_(0x55)
        del blocks
        b = None
        got = flat(call(side.cuda_stream))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(torch.nan_to_num(g), torch.nan_to_num(w))
        del got, g


@pytest.mark.parametrize("name", NAMES)
def test_a_result_that_the_current_stream_still_reads(name):
    call = calls()[name]
    side = torch.cuda.Stream()
    want = [t.clone() for t in flat(call(None))]
    torch.cuda.synchronize()
    got = flat(call(side.cuda_stream))
    side.synchronize()
    torch.cuda._sleep(SLEEP)
    copies = [g.clone() for g in got]  # (waits behind the sleep)
    sizes = [g.untyped_storage().nbytes() for g in got]
    del got
    with torch.cuda.stream(side):
        for n in sizes:
            for _ in range(4):
                torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0x55)
    torch.cuda.synchronize()
    for c, w in zip(copies, want):
        assert torch.equal(torch.nan_to_num(c), torch.nan_to_num(w))


def test_policies_too():
    import workloads as W
    import paper_2211_15023_b200 as P
    from parity_util import calibrated
    b = 64
    policy = P.Policy(calibrated("nature_cnn_b160"), b)
    obs, u = torch.from_numpy(W.observations("nature_cnn_b160", b)).cuda(), torch.from_numpy(W.uniforms("nature_cnn_b160", b)).cuda()
    side = torch.cuda.Stream()
    for call in (lambda s: policy.act(obs, u, stream=s), lambda s: policy.act_ex(obs, u, stream=s)):
        want = [t.clone() for t in flat(call(None))]
        call(side.cuda_stream)
        torch.cuda.synchronize()
        blocks = [torch.empty(1 << i, dtype=torch.uint8, device="cuda") for i in range(8, 16) for _ in range(4)]
        torch.cuda._sleep(SLEEP)
        for x in blocks:
            x.fill_(0x55)
        del blocks, x
        got = flat(call(side.cuda_stream))
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
