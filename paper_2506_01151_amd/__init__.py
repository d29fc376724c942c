"""Python binding of the zapformat HIP library (argument marshalling only)."""
from .binding import (Engine, State, StateBatch, Twin, ZfError, load_library, compile, advance, compute_mask, compute_mask_async, compute_mask_apply_async, compute_mask_noalloc, mask_wait, apply_mask,  # noqa: F401
                      ZF_OK, ZF_ERR_INVALID_ARG, ZF_ERR_GRAMMAR, ZF_ERR_REJECTED, ZF_ERR_RANGE,
                      ZF_ERR_DEVICE, ZF_ERR_OOM, ZF_ERR_OVERFLOW)


_OPERATORS = ("quantize_blocks", "head_logits", "token_logprobs", "TokenLogprobs")
_LOSSES = ("distill_loss", "policy_loss", "preference_loss", "DistillLoss", "PolicyLoss", "PreferenceLoss")


def __getattr__(name):                         # they need torch, which the rest of the binding loads with the first tensor
    if name in _OPERATORS:
        from . import operators
        return getattr(operators, name)
    if name in _LOSSES:
        from . import losses
        return getattr(losses, name)
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted([*globals(), *_OPERATORS, *_LOSSES])
