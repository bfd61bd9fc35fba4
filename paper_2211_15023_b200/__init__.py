"""B200-native int8 Actor policy inference (AcceRL's data-collection hot path).

The work happens in ``libaccerl.so`` (hand-written CUDA for sm_100a behind the C
ABI of ``include/accerl.h``).  This package only marshals arguments: torch is
used for device memory and streams, nothing is computed in Python, and there
is no CPU fallback -- importing :class:`Policy` without the built library
raises.
"""
from .binding import (AccerlError, Policy, act_mixed, ckpt_act_backward, ckpt_load, ckpt_save,  # noqa: F401
                      ckpt_weight_grad, device_check, kl, library, library_path, linear_i8, policy_loss, quant_rows,
                      tc_probe_i8, trim, vtrace, FLAG_FORCE_GENERIC, FLAG_KEEP_ACTIVATIONS, FLAG_TAP_FUSED,
                      FLAG_VALUE_HEAD, FLAG_TEST_NO_FASTDIV, FLAG_TEST_NO_AFFINE)
