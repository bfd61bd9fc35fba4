"""The Learner's operators refuse what their kernels could not read, on the host and before anything is launched."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")
INVALID = 1


@pytest.fixture(scope="module")
def P():
    from paper_2211_15023_b200 import build
    build.build()
    import paper_2211_15023_b200 as package
    return package


@pytest.fixture(scope="module")
def lib(P):
    return P.library()


BUF = np.zeros(1024, np.float32)
AT = (BUF.ctypes.data + 255) // 256 * 256  # a host address that is aligned like a device allocation; never read


def loss_args(**change):
    from paper_2211_15023_b200.binding import PolicyLossArgs
    a = dict(logits=AT, actions=AT, logp_old=AT, advantages=AT, ld_logits=8, ld_grad=8, rows=2, n_actions=8, clip_low=0.2,
             clip_high=0.2, grad=AT + 512, logp=AT, kl=AT, entropy=AT, stats=AT, terms=AT)
    a.update(change)
    return PolicyLossArgs(**a)


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(actions=None), dict(logp_old=None), dict(advantages=None), dict(logp=None), dict(kl=None),
    dict(entropy=None), dict(stats=None), dict(terms=None), dict(rows=0), dict(rows=-3), dict(rows=(1 << 26) + 1),
    dict(n_actions=0), dict(n_actions=262129, ld_logits=262129, ld_grad=262129), dict(ld_logits=7), dict(ld_grad=7),
    dict(logits_ref=AT, ld_logits_ref=7), dict(logits_ref=AT, ld_logits_ref=8, logp_ref=AT), dict(dtype=3), dict(dtype=-1),
    dict(clip_low=-0.1), dict(clip_high=float("nan")), dict(kl_coef=float("inf")), dict(entropy_coef=float("nan")),
    dict(logits=AT + 2), dict(grad=AT + 513), dict(dtype=1, logits=AT + 1), dict(actions=AT + 4, actions64=1),
    dict(actions=AT + 2), dict(terms=AT + 4), dict(weights=AT + 1), dict(stats=AT + 3), dict(grad=AT, ld_grad=9)])
def test_policy_loss_refuses(lib, change):
    assert lib.accerl_policy_loss(C.byref(loss_args(**change)), None) == INVALID
    assert lib.accerl_last_error().startswith(b"policy_loss")


def test_policy_loss_takes_no_null_description(lib):
    assert lib.accerl_policy_loss(None, None) == INVALID


def test_tensors_a_kernel_cannot_read_raise(P):
    z, a, f = torch.zeros((4, 6)), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for call in (lambda: P.policy_loss(z, a, f, f), lambda: P.policy_loss(z.double(), a, f, f),
                 lambda: P.policy_loss(z.int(), a, f, f)):
        with pytest.raises(AssertionError):
            call()
