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


def save_args(**change):
    a = dict(x=AT, ld_x=40, dtype=0, rows=2, cols=40, act=1, y=AT, ld_y=40, q=AT, ld_q=64, e=AT, ld_e=2, stream=None)
    a.update(change)
    return a


BAD_CKPT = [dict(q=None), dict(e=None), dict(q=AT + 8), dict(ld_q=63), dict(ld_q=72), dict(ld_q=48), dict(ld_e=1), dict(rows=0),
            dict(cols=0), dict(rows=1 << 40), dict(dtype=3), dict(dtype=-1)]


@pytest.mark.parametrize("change", BAD_CKPT + [dict(x=None), dict(x=AT + 2), dict(dtype=1, x=AT + 1), dict(ld_x=39),
                                               dict(ld_y=39), dict(y=AT + 1), dict(act=4), dict(act=-1)])
def test_ckpt_save_refuses(lib, change):
    assert lib.accerl_ckpt_save(*save_args(**change).values()) == INVALID
    assert lib.accerl_last_error().startswith(b"ckpt_save")


@pytest.mark.parametrize("change", BAD_CKPT + [dict(x=None), dict(x=AT + 2), dict(ld_x=39)])
def test_ckpt_load_refuses(lib, change):
    a = save_args(**change)
    args = [a[k] for k in ("q", "ld_q", "e", "ld_e", "rows", "cols", "x", "ld_x", "dtype", "stream")]
    assert lib.accerl_ckpt_load(*args) == INVALID
    assert lib.accerl_last_error().startswith(b"ckpt_load")


@pytest.mark.parametrize("change", BAD_CKPT + [dict(x=None), dict(x=AT + 2), dict(ld_x=39), dict(y=None), dict(ld_y=39),
                                               dict(act=4)])
def test_ckpt_act_backward_refuses(lib, change):
    a = save_args(**change)
    args = [a[k] for k in ("x", "ld_x", "dtype", "q", "ld_q", "e", "ld_e", "rows", "cols", "act", "y", "ld_y", "stream")]
    assert lib.accerl_ckpt_act_backward(*args) == INVALID
    assert lib.accerl_last_error().startswith(b"ckpt_act_backward")


def test_checkpoint_tensors_a_kernel_cannot_read_raise(P):
    x = torch.zeros((4, 40))
    ckpt = torch.zeros((4, 64), dtype=torch.int8), torch.zeros((4, 2), dtype=torch.uint8)
    for call in (lambda: P.ckpt_save(x), lambda: P.ckpt_save(x.double()), lambda: P.ckpt_load(ckpt, 40, torch.float32),
                 lambda: P.ckpt_act_backward(x, ckpt, "relu")):
        with pytest.raises(AssertionError):
            call()


@pytest.mark.parametrize("change", [dict(x=None), dict(q=None), dict(scale=None), dict(x=AT + 2), dict(dtype=1, x=AT + 1),
                                    dict(ld_x=39), dict(q=AT + 8), dict(ld_q=47), dict(ld_q=32), dict(rows=0), dict(cols=0),
                                    dict(rows=1 << 31), dict(rows=1 << 41), dict(dtype=3), dict(scale=AT + 2)])
def test_quant_rows_refuses(lib, change):
    a = dict(x=AT, ld_x=40, dtype=0, rows=2, cols=40, q=AT, ld_q=48, scale=AT, stream=None)
    a.update(change)
    assert lib.accerl_quant_rows(*a.values()) == INVALID
    assert lib.accerl_last_error().startswith(b"quant_rows")


def linear_args(**change):
    from paper_2211_15023_b200.binding import LinearI8Args
    a = dict(x=AT, w=AT, w_scale=AT, y=AT, workspace=AT, ld_x=40, ld_w=48, ld_y=8, workspace_bytes=1 << 20, tokens=2, n=8,
             k=40, x_dtype=0, y_dtype=0)
    a.update(change)
    return LinearI8Args(**a)


I8 = dict(x_dtype=3, x_scale=AT, ld_x=48, workspace=None)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(w=None), dict(w_scale=None), dict(y=None), dict(workspace=None), dict(workspace=AT + 128),
    dict(workspace_bytes=0), dict(tokens=0), dict(n=0), dict(k=0), dict(k=131073, ld_x=131073, ld_w=131088), dict(ld_x=39),
    dict(ld_w=47), dict(ld_w=32), dict(w=AT + 8), dict(ld_y=7), dict(y=AT + 2), dict(y_dtype=3), dict(x_dtype=4),
    dict(x_scale=AT), dict(bias=AT + 1), dict(w_scale=AT + 2), dict(I8, x_scale=None), dict(I8, x=AT + 8), dict(I8, ld_x=40),
    dict(I8, ld_x=32)])
def test_linear_i8_refuses(lib, change):
    assert lib.accerl_linear_i8(C.byref(linear_args(**change)), None) == INVALID
    assert lib.accerl_last_error().startswith(b"linear_i8")


def test_linear_i8_needs_no_workspace_for_quantised_tokens(lib):
    assert lib.accerl_linear_i8(None, None) == INVALID
    assert lib.accerl_linear_i8_workspace(5, 40, 3) == 0 and lib.accerl_linear_i8_workspace(5, 40, 1) == 256 + 256
    assert lib.accerl_linear_i8_workspace(1 << 20, 1 << 16, 0) == (1 << 36) + (1 << 22)


def test_int8_tensors_a_kernel_cannot_read_raise(P):
    x, q, s = torch.zeros((4, 40)), torch.zeros((8, 48), dtype=torch.int8)[:, :40], torch.zeros(8)
    for call in (lambda: P.quant_rows(x), lambda: P.linear_i8(x, (q, s)), lambda: P.linear_i8((q, s), (q, s)),
                 lambda: P.linear_i8(x.double(), (q, s))):
        with pytest.raises(AssertionError):
            call()


def grad_args(**change):
    from paper_2211_15023_b200.binding import WeightGradArgs
    a = dict(dy=AT, q=AT, e=AT, dw=AT, db=AT, ld_dy=16, ld_q=64, ld_e=2, ld_dw=40, tokens=4, n=16, k=40, dy_dtype=1,
             out_dtype=0)
    a.update(change)
    return WeightGradArgs(**a)


@pytest.mark.parametrize("change", [
    dict(dy=None), dict(q=None), dict(e=None), dict(dw=None), dict(tokens=0), dict(n=0), dict(k=0), dict(dy_dtype=3),
    dict(out_dtype=2), dict(out_dtype=1, accumulate=1), dict(q=AT + 8), dict(ld_q=63), dict(ld_q=72), dict(ld_e=1),
    dict(dy=AT + 1), dict(ld_dy=15), dict(ld_dw=39), dict(dw=AT + 2), dict(db=AT + 2), dict(ld_dy=17), dict(dy=AT + 2),
    dict(ld_dy=17, workspace=AT, workspace_bytes=64), dict(ld_dy=17, workspace=AT + 16, workspace_bytes=1 << 20),
    dict(n=1 << 27, ld_dy=1 << 27, k=1 << 27, ld_q=1 << 27, ld_e=1 << 22, ld_dw=1 << 27)])
def test_ckpt_weight_grad_refuses(lib, change):
    assert lib.accerl_ckpt_weight_grad(C.byref(grad_args(**change)), None) == INVALID
    assert lib.accerl_last_error().startswith(b"ckpt_weight_grad")


def test_ckpt_weight_grad_workspace_and_types(lib):
    assert lib.accerl_ckpt_weight_grad(None, None) == INVALID
    assert lib.accerl_ckpt_weight_grad(C.byref(grad_args(dy_dtype=0)), None) == 2  # fp32 gradients: unsupported
    assert lib.accerl_ckpt_weight_grad_workspace(None) == 0
    assert lib.accerl_ckpt_weight_grad_workspace(C.byref(grad_args())) == 0
    assert lib.accerl_ckpt_weight_grad_workspace(C.byref(grad_args(n=15, ld_dy=15))) == 256  # 4 rows of 16 16-bit values
    assert lib.accerl_ckpt_weight_grad_workspace(C.byref(grad_args(dy=AT + 2, tokens=1 << 20, n=1 << 14, ld_dy=1 << 14))) == 1 << 35
    # many tiles, five or more columns of channels: the checkpoint's values in 16 bits
    big = dict(n=2048, ld_dy=2048, k=4001, ld_q=4032, ld_e=126, ld_dw=4001, tokens=100)
    assert lib.accerl_ckpt_weight_grad_workspace(C.byref(grad_args(**big))) == (100 * 4008 * 2 + 255) // 256 * 256
