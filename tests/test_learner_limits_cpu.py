"""Sizes at the ends of int32 are refused by the Learner's operators before a kernel would count past them."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from test_learner_args_cpu import AT, INVALID, P, grad_args, lib, linear_args  # noqa: E402,F401

MOST = (1 << 31) - 1


@pytest.mark.parametrize("tokens,n", [(MOST, 1), (MOST - 200, 3), (1, MOST), (70, MOST - 4000), (1, MOST - 65535), (MOST - 65535, 1)])
def test_linear_i8_refuses_rows_whose_tiles_pass_int32(lib, tokens, n):  # noqa: F811
    a = linear_args(tokens=tokens, n=n, k=1, ld_y=n, workspace_bytes=1 << 40)
    assert lib.accerl_linear_i8(C.byref(a), None) == INVALID
    assert b"2^31 - 2^16" in lib.accerl_last_error() or b"too large" in lib.accerl_last_error()


@pytest.mark.parametrize("change", [dict(tokens=MOST), dict(tokens=MOST - 63), dict(tokens=MOST - 65535)])
def test_ckpt_weight_grad_refuses_tokens_whose_stages_pass_int32(lib, change):  # noqa: F811
    a = grad_args(workspace=AT, workspace_bytes=1 << 60, **change)
    assert lib.accerl_ckpt_weight_grad(C.byref(a), None) == INVALID
    assert b"2^31 - 2^16" in lib.accerl_last_error()


@pytest.mark.parametrize("n,k", [(MOST, 40), (16, MOST), (MOST - 6, MOST - 6)])
def test_the_workspace_of_the_largest_sizes_is_not_negative(lib, n, k):  # noqa: F811
    need = lib.accerl_ckpt_weight_grad_workspace(C.byref(grad_args(n=n, k=k, ld_dy=n + 1, dy=AT + 2)))
    assert need >= 2 * 4 * n


def test_checkpoints_in_place_need_the_same_row_distance(lib):  # noqa: F811
    from test_learner_args_cpu import save_args
    a = save_args(y=AT, ld_y=48)
    assert lib.accerl_ckpt_save(*a.values()) == INVALID and b"same ld" in lib.accerl_last_error()
    args = [a[k] for k in ("x", "ld_x", "dtype", "q", "ld_q", "e", "ld_e", "rows", "cols", "act", "y", "ld_y", "stream")]
    assert lib.accerl_ckpt_act_backward(*args) == INVALID and b"same ld" in lib.accerl_last_error()
