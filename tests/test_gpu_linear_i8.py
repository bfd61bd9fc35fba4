"""int8 layers on activations quantised per token: the quantiser and the product, against their definitions in 64 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def quantised(x):
    """(q int8, scale fp32) of the definition, from float64; a fp32 quotient is the double quotient rounded (53 >= 2 24 + 2)."""
    x = x.double().cpu()
    broken = ~torch.isfinite(x).all(1)
    top = torch.where(broken[:, None], torch.zeros_like(x), x).abs().amax(1)
    s = (top / 127.0).float()
    ratio = torch.where((s > 0)[:, None], x / s.double()[:, None], torch.zeros_like(x)).float()
    q = torch.where(broken[:, None], torch.zeros_like(ratio), ratio).round().clamp(-127, 127).to(torch.int8)
    return q, torch.where(broken, torch.full_like(s, math.nan), s)


def matrix(t, k, dtype, seed, pad=0, offset=0):
    g = torch.Generator("cuda").manual_seed(seed)
    flat = torch.full((offset + t * (k + pad),), float("nan"), device="cuda", dtype=dtype)
    x = flat[offset:].view(t, k + pad)[:, :k]
    x.copy_(torch.randn((t, k), device="cuda", generator=g) * torch.exp(torch.randn((t, 1), device="cuda", generator=g)))
    return x


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=1e30), torch.nan_to_num(b, nan=1e30))


# a warp per row (up to 512 / 1024 elements), CTAs of every size, rows that do not fit the registers
@pytest.mark.parametrize("t,k", [(1, 1), (5, 7), (9, 64), (3, 511), (130, 1000), (4, 1025), (3, 4096), (2, 5003), (2, 16384),
                                 (2, 32769), (1, 70001)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_are_quantised_as_defined(t, k, dtype):
    import paper_2211_15023_b200 as P
    for pad, offset in ((0, 0), (3, 1), (8, 4)):
        x = matrix(t, k, TYPES[dtype], 10 * t + k, pad, offset)
        q, s = P.quant_rows(x)
        want_q, want_s = quantised(x)
        assert torch.equal(s.cpu(), want_s) and torch.equal(q.cpu(), want_q)
        assert q.stride(0) % 16 == 0


@pytest.mark.parametrize("k", [40, 3000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_unusual_values(k, dtype):
    """Zeros, the ends of the type's range, values at and next to the rounding ties, infinities and NaN."""
    import paper_2211_15023_b200 as P
    dt = TYPES[dtype]
    info = torch.finfo(dt)
    x = torch.ones((9, k), device="cuda", dtype=dt)
    x[1] = 0
    x[2] = info.smallest_normal * info.eps
    x[3, 0], x[3, 1] = info.max, info.min
    x[4, 7] = math.inf
    x[5, k - 1] = math.nan
    x[6] = (torch.arange(k, device="cuda") % 255 - 127.0 + 0.5).to(dt)
    x[6, 0] = 127.0  # scale 1: every other value lies on a tie
    x[7] = (torch.arange(k, device="cuda") % 127 * 2.0 ** -14).to(dt)
    x[8, ::2] = -x[8, ::2]
    q, s = P.quant_rows(x)
    want_q, want_s = quantised(x)
    assert same(s.cpu(), want_s) and torch.equal(q.cpu(), want_q)


def layer(t, k, n, dtype, seed, bias=True):
    import paper_2211_15023_b200 as P
    g = torch.Generator("cuda").manual_seed(seed)
    x = matrix(t, k, dtype, seed)
    w = torch.randn((n, k), device="cuda", generator=g) / math.sqrt(k)
    b = torch.randn(n, device="cuda", generator=g) if bias else None
    return x, P.quant_rows(w), b


def product(xq, xs, wq, ws, bias, relu):
    """float64, the two scales' product rounded to fp32 first, as defined."""
    acc = xq.double().cpu() @ wq.double().cpu().t()
    y = acc.float().double() * (xs.cpu()[:, None] * ws.cpu()[None, :]).double()
    y = y + bias.double().cpu() if bias is not None else y
    return torch.relu(y) if relu else y


def close(got, want, dtype):
    """One fma in fp32 (half a step, 2^-24) and one rounding to the type; a fp32 value next to a type's rounding border may
    fall to the other side: 2^-24 of the value again."""
    half = torch.finfo(dtype).eps / 2
    got, want = got.double().cpu(), want.to(torch.float64)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    bad = (got - want).abs() > (half + 2.0 ** -22) * want.abs() + tiny
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


# tokens: every width of the instruction and its edges; k: parts of a 128-byte chunk, one chunk, many; n: parts of a tile
@pytest.mark.parametrize("t,k,n", [(1, 1, 1), (4, 4097, 1000), (3, 9000, 5001), (2, 33000, 40), (4, 30000, 33), (5, 700, 90), (1, 64, 16), (1, 4096, 512), (2, 127, 130), (16, 129, 128), (17, 512, 129),
                                   (32, 1000, 257), (33, 640, 100), (64, 2592, 256), (65, 3136, 512), (128, 4100, 640),
                                   (129, 256, 300), (300, 1537, 1000), (1000, 384, 2000), (257, 16, 4097), (2047, 2592, 256),
                                   (4000, 300, 700), (9700, 130, 250), (513, 1000, 5000), (300, 64, 20001)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_layers_match_the_definition(t, k, n, dtype):
    import paper_2211_15023_b200 as P
    x, (wq, ws), bias = layer(t, k, n, TYPES[dtype], 7 * t + k + n)
    xq, xs = quantised(x)
    y = P.linear_i8(x, (wq, ws), bias=bias)
    assert y.dtype == TYPES[dtype] and tuple(y.shape) == (t, n)
    close(y, product(xq, xs, wq, ws, bias, False), TYPES[dtype])
    for out in TYPES.values():
        close(P.linear_i8(x, (wq, ws), relu=True, out_dtype=out), product(xq, xs, wq, ws, None, True), out)
    # tokens quantised beforehand: the same bits
    again = P.linear_i8(P.quant_rows(x), (wq, ws), bias=bias, out_dtype=TYPES[dtype])
    assert torch.equal(again, y)
    P.device_check()


@pytest.mark.parametrize("t", [1, 5, 40, 100, 300, 1500])
def test_strided_tokens_weights_and_outputs(t):
    import paper_2211_15023_b200 as P
    k, n = 700, 333
    x, (wq, ws), bias = layer(t, k, n, torch.bfloat16, t)
    want = P.linear_i8(x, (wq, ws), bias=bias)
    wide = matrix(t, k, torch.bfloat16, 3, pad=5, offset=3)
    wide.copy_(x)
    w_wide = torch.full((n, 1024), 99, device="cuda", dtype=torch.int8)
    w_wide[:, 32:32 + k] = wq
    out = torch.full((t, n + 7), 7.0, device="cuda", dtype=torch.bfloat16)
    got = P.linear_i8(wide, (w_wide[:, 32:32 + k], ws), bias=bias, out=out[:, 3:3 + n])
    assert torch.equal(got, want) and (out[:, :3] == 7).all() and (out[:, 3 + n:] == 7).all()


@pytest.mark.parametrize("t", [1, 20, 200, 700])
def test_a_broken_token_is_nan_and_no_other(t):
    import paper_2211_15023_b200 as P
    x, w, bias = layer(t, 300, 200, torch.bfloat16, t)
    want = P.linear_i8(x, w, bias=bias)
    x[t // 2, 17] = math.inf
    got = P.linear_i8(x, w, bias=bias)
    bad = torch.zeros(t, dtype=torch.bool, device="cuda")
    bad[t // 2] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


def test_the_largest_sums():
    """127 x 127 over the longest row stays inside int32, and is exact until it is rounded to float."""
    import paper_2211_15023_b200 as P
    k, n = 131072, 130
    w = torch.full((n, k), 127, device="cuda", dtype=torch.int8)
    w[1::2] = -127
    ws = torch.ones(n, device="cuda")
    for t in (1, 33, 260):
        xq, xs = torch.full((t, k), 127, device="cuda", dtype=torch.int8), torch.ones(t, device="cuda")
        y = P.linear_i8((xq, xs), (w, ws))
        want = torch.full((t, n), float(np.float32(127 * 127 * k)))
        want[:, 1::2] *= -1
        assert torch.equal(y.cpu(), want)


def test_captured_on_two_streams_and_after_the_weights_were_made():
    """Weights quantised right before the call on the same stream; two graphs that replay at the same time."""
    import paper_2211_15023_b200 as P
    g = torch.Generator("cuda").manual_seed(1)
    w = torch.randn((1000, 900), device="cuda", generator=g)
    cases = [matrix(t, 900, torch.bfloat16, t) for t in (3, 600, 1, 12000)]
    call = lambda x: P.linear_i8(x, P.quant_rows(w), relu=True)  # noqa: E731
    want = [call(x) for x in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in cases:
            call(x)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for x in cases:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(call(x))
        graphs.append(gr)
    for _ in range(10):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for gr in graphs[::2]:
            gr.replay()
        with torch.cuda.stream(side):
            for gr in graphs[1::2]:
                gr.replay()
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            assert torch.equal(o, v)
    for _ in range(50):  # new weights each time: nothing of the last call is read
        w.normal_(generator=g)
        y = call(cases[0])
        xq, xs = quantised(cases[0])
        q, s = quantised(w)
        close(y, product(xq, xs, q, s, None, True), torch.bfloat16)
    P.device_check()
