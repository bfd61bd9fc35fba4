"""Weight and bias gradients from 8-bit checkpoints: the same bits with and without db, long sums, infinities, limits."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_weight_grad import TYPES, check, inputs, sums  # noqa: E402


# sizes at which db's tiles are more than the chip holds beside dw's split as far as it goes, and others
@pytest.mark.parametrize("t,n,k", [(2048, 768, 768), (8192, 1024, 2304), (2048, 64, 4736), (2048, 512, 2304), (1000, 3100, 130),
                                   (4096, 12544, 128), (700, 130, 900)])
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_dw_is_the_same_whether_db_is_wanted(t, n, k, out):
    import paper_2211_15023_b200 as P
    dy, ckpt = inputs(t, n, k, torch.bfloat16, t + n + k)
    dw, db = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out])
    alone, none = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out], bias=False)
    P.device_check()
    assert none is None and torch.equal(dw, alone)
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()
    want, mag = sums(dy, ckpt, k)
    check((dw, db), want, mag, TYPES[out])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, 0.9, 0.24])
def test_gradients_beyond_the_ordinary_in_rows_off_16_bytes(dtype, value):
    """Infinities and values near the type's end in the last columns of rows that are copied for the TMA: they keep their bits.
    (0.24: bf16 values whose bits are an infinity's or a NaN's of fp16.)"""
    import paper_2211_15023_b200 as P
    t, n, k = 70, 37, 64
    info = torch.finfo(TYPES[dtype])
    dy, ckpt = inputs(t, n, k, TYPES[dtype], 5, pad=2)
    dy[11, 36] = dy[12, 33] = dy[13, 35] = value if math.isinf(value) else value * info.max if value > 0.5 else 2.0 ** 122 if dtype == "bf16" else 1.0
    dw, db = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=torch.float32)
    x = P.ckpt_load(ckpt, k, torch.float32).double()
    want, want_b = dy.double().t() @ x, dy.double().sum(0)
    if math.isinf(value):
        for got, w in ((dw, want), (db, want_b)):
            assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(torch.isinf(got), torch.isinf(w))
            assert torch.equal(got[torch.isinf(got)], w[torch.isinf(w)].float())
        return
    # (sums in fp32 of at most 70 products: each addition cuts off at most 2^-22 of what it holds)
    for got, w, mag in ((dw, want, dy.double().abs().t() @ x.abs()), (db, want_b, dy.double().abs().sum(0))):
        fits = mag < torch.finfo(torch.float32).max  # (0.9 of bf16's largest times a value above 1 is infinite)
        assert torch.isfinite(got[fits]).all() and ((got.double() - w).abs()[fits] <= 70 * 2.0 ** -22 * mag[fits]).all()
        assert torch.isinf(got[w.abs() > 1.001 * torch.finfo(torch.float32).max]).all()


@pytest.mark.parametrize("t,n,k", [(1 << 22, 64, 64), (40000, 2050, 2570), (40000, 520, 15000)])
@pytest.mark.parametrize("dtype,out", [("fp16", "fp16"), ("bf16", "bf16"), ("fp16", "fp32")])
def test_long_sums_of_one_sign(t, n, k, dtype, out):
    """A sum in the tensor cores is cut off at each of its additions (16 tokens), by less than 2^-23 of itself: a part of
    8192 tokens loses less than 512 2^-23 = 6.2e-5, the parts' additions in fp32 next to nothing."""
    import paper_2211_15023_b200 as P
    g = torch.Generator("cuda").manual_seed(t)
    make = lambda c, scale: ((torch.rand((t, c), device="cuda", generator=g) + 1.0) * scale).to(TYPES[dtype])  # noqa: E731
    dy, (_, ckpt) = make(n, 0.125 * 16384.0 / t), P.ckpt_save(make(k, 1.0))
    dw, db = P.ckpt_weight_grad(dy, ckpt, k, out_dtype=TYPES[out])
    P.device_check()
    want, want_b = torch.zeros((n, k), device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda", dtype=torch.float64)
    x = P.ckpt_load(ckpt, k, TYPES[dtype])
    for i in range(0, t, 1 << 16):
        d = dy[i:i + (1 << 16)].double()
        want += d.t() @ x[i:i + (1 << 16)].double()
        want_b += d.sum(0)
    half = torch.finfo(TYPES[out]).eps / 2
    for got, w in ((dw, want), (db, want_b)):
        assert ((got.double() - w).abs() <= (half * 1.01 + 6.2e-5) * w.abs()).all()
