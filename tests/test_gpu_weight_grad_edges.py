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
    want, mag = sums(dy, ckpt, k)
    check((dw, db), want, mag, TYPES[out])
