"""Losses that a learner takes on logits under masks, each one number with the gradient of the logits.

    got = distill_loss(logits, teacher.top_ids, teacher.top_logprobs, mask, rest=True, weight=weight)     # a teacher's most probable tokens (token_logprobs(top=))
    got = policy_loss(logits, tokens, old_logprobs, advantages, mask, ref_logprobs=ref, kl_weight=0.05, weight=weight)
    got = preference_loss(logits, tokens, offsets, ref_logprobs, mask, beta=0.1)
    got.loss.backward()

logits: fp32 or bf16 [rows, V], rows without gaps; masks are those of compute_mask.  What a mask forbids, and what is -inf, has no gradient and is not looked at.  got.loss is the sum of
weight x got.losses (weight: fp32, one each where it is None; 1 / n makes a mean) and has a gradient, once, for the logits; everything else that comes back, and
every other tensor that goes in, is a constant (one that requires grad is refused).  distill_loss and policy_loss make the gradient beside the losses, in the
same pass over the logits: where the loss's own gradient is 1, as that of got.loss.backward(), the backward pass has nothing left to do; elsewhere, when it runs a
second time, and in a graph's capture it reads the logits again and makes the gradient anew: (0.5 * got.loss).backward() on 4,096 x 128,256 bf16 makes a step of policy_loss 817 us instead of 411, of distill_loss 867
instead of 438.  A coefficient, or the share of a micro-batch, is better given in `weight`.  (A weight of 0 does not leave out a row whose loss is infinite or NaN; negative tokens and ids do.)  As in operators.py calls are enqueued on torch's current stream, wait for nothing and allocate through torch
only, so that they can be captured into a graph (a backward pass from leaves made for the capture, no eager graph of theirs alive); what does not fit raises ZfError; forward-mode derivatives, torch.func and tracers are refused; a tensor that was written before the backward pass makes it raise.
"""
import ctypes
import math
from typing import NamedTuple, Optional

import torch

from . import _native_losses
from .binding import DistillArgs, PolicyArgs, PreferenceArgs, _check
from .operators import _DTYPES, _kept, _lib, _mask_ptr, _matrix, _need, _not_traced, _plain, _row_stride, _stream

_native_losses.bind({n: ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in (
    "zf_distill_loss", "zf_distill_loss_backward", "zf_policy_loss", "zf_policy_loss_backward", "zf_preference_loss", "zf_preference_loss_backward", "zf_last_error")}, _check)
# The ordinary call is _native_losses' (csrc/zf_py_losses.cpp); what it does not take it answers with None, and the code here, its definition, does or refuses it.

_IDS = (torch.int32, torch.int64)
_F32 = (torch.float32,)


class DistillLoss(NamedTuple):
    loss: torch.Tensor                             # fp32, one number
    losses: torch.Tensor                           # fp32 [rows]


class PolicyLoss(NamedTuple):
    loss: torch.Tensor                             # fp32, one number
    losses: torch.Tensor                           # fp32 [rows]
    logprobs: torch.Tensor                         # fp32 [rows]
    entropy: Optional[torch.Tensor]                # fp32 [rows], where it is part of the loss


class PreferenceLoss(NamedTuple):
    loss: torch.Tensor                             # fp32, one number
    losses: torch.Tensor                           # fp32 [pairs]
    chosen: torch.Tensor                           # fp32 [pairs]: beta times the preferred sequences' log ratios, a reward
    rejected: torch.Tensor                         # fp32 [pairs]


def _constant(t, what, dtypes, shape, device):
    _need(isinstance(t, torch.Tensor) and t.layout == torch.strided and t.device == device and t.dtype in dtypes, f"{what}: {' or '.join(str(d)[6:] for d in dtypes)} on the logits' device is wanted")
    _plain(t, what)
    _need(tuple(t.shape) == tuple(shape) and t.is_contiguous(), f"{what}: a contiguous {list(shape)} is wanted, not {tuple(t.shape)}")
    _need(not (torch.is_grad_enabled() and t.requires_grad), f"{what}: it is a constant here and requires grad (detach it)")


def _number(x, what, low=-math.inf, high=math.inf):
    _need(isinstance(x, (int, float)) and low <= x <= high, f"{what}: a number from {low} to {high} is wanted, not {x!r}")
    return float(x)


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _capturing(device):
    with torch.cuda.device(device):
        return torch.cuda.is_current_stream_capturing()


def _pop(held):
    """What is in the list, taken out, or None: two backward passes at once get it once."""
    try:
        return held.pop()
    except IndexError:
        return None


class _Loss:
    """One of the losses: `t` its tensors by name, `o` its numbers.  args() is given both and what the kernels write."""

    def __init__(self, t, o):
        self.t, self.o = t, o

    def rows(self, r, out):
        x = self.t["logits"]
        r.logits, r.dtype, r.V, r.rows, r.row_stride = x.data_ptr(), _DTYPES[x.dtype], x.shape[1], x.shape[0], _row_stride(x)
        r.mask, r.weight, r.temperature = _ptr(self.t["mask"]), _ptr(self.t["weight"]), self.o["temperature"]
        r.loss, r.losses = out["loss"].data_ptr(), out["losses"].data_ptr()

    def fresh(self, **shapes):
        dev = self.t["logits"].device
        return {n: torch.empty(s, dtype=torch.float32, device=dev) for n, s in shapes.items()}

    def grad(self):
        return torch.empty(self.t["logits"].shape, dtype=self.t["logits"].dtype, device=self.t["logits"].device)

    def forward(self, grad):
        """The results by name; writes `grad` beside them where it is given."""
        out, x = self.outputs(), self.t["logits"]
        _check(self.call(ctypes.byref(self.args(out)), _ptr(grad), x.shape[1], x.device.index, _stream(x.device)))
        return out

    def backward(self, out, g, held, grad):
        x = self.t["logits"]
        _check(self.call_back(ctypes.byref(self.args(out)), g.data_ptr(), held, grad.data_ptr(), x.shape[1], x.device.index, _stream(x.device)))


class _Distill(_Loss):
    call, call_back, at_once = _lib.zf_distill_loss, _lib.zf_distill_loss_backward, True
    saved = ()

    def outputs(self):
        return self.fresh(loss=(), losses=self.t["logits"].shape[:1])

    def args(self, out):
        a, t = DistillArgs(), self.t
        self.rows(a.r, out)
        a.ids, a.values, a.id_bytes, a.values_dtype = t["ids"].data_ptr(), t["values"].data_ptr(), t["ids"].element_size(), _DTYPES[t["values"].dtype]
        a.n_listed, a.rest = t["ids"].shape[1], self.o["rest"]
        return a

    def shapes(self, rows):
        n = self.o["listed"]
        return {"ids": (_IDS, (rows, n)), "values": (tuple(_DTYPES), (rows, n)), "weight": (_F32, (rows,))}


class _Policy(_Loss):
    call, call_back, at_once = _lib.zf_policy_loss, _lib.zf_policy_loss_backward, True
    saved = ()

    def outputs(self):
        n = self.t["logits"].shape[:1]
        return self.fresh(loss=(), losses=n, logprobs=n, **({"entropy": n} if self.o["entropy"] else {}))

    def args(self, out):
        a, t, o = PolicyArgs(), self.t, self.o
        self.rows(a.r, out)
        a.tokens, a.token_bytes, a.old_logprobs, a.advantages, a.ref_logprobs = t["tokens"].data_ptr(), t["tokens"].element_size(), t["old"].data_ptr(), t["advantages"].data_ptr(), _ptr(t["ref"])
        a.clip_low, a.clip_high, a.kl_weight, a.entropy_weight = o["clip"][0], o["clip"][1], o["kl_weight"], o["entropy_weight"]
        a.logprobs, a.entropy = out["logprobs"].data_ptr(), _ptr(out.get("entropy"))
        return a

    def shapes(self, rows):
        return {"tokens": (_IDS, (rows,)), "old": (_F32, (rows,)), "advantages": (_F32, (rows,)), "ref": (_F32, (rows,)), "weight": (_F32, (rows,))}


class _Preference(_Loss):
    at_once = False
    saved = ("stats", "slopes")                    # what the gradient is made from

    @staticmethod
    def call(a, grad, stride, device, stream):
        return _lib.zf_preference_loss(a, device, stream)

    @staticmethod
    def call_back(a, g, held, grad, stride, device, stream):
        return _lib.zf_preference_loss_backward(a, g, grad, stride, device, stream)

    def outputs(self):
        n, P = self.t["logits"].shape[0], self.o["pairs"]
        return self.fresh(loss=(), losses=(P,), chosen=(P,), rejected=(P,), stats=(n, 4), slopes=(2 * P,))

    def args(self, out):
        a, t, o = PreferenceArgs(), self.t, self.o
        self.rows(a.r, out)
        a.tokens, a.token_bytes, a.offsets, a.offset_bytes, a.ref_logprobs = t["tokens"].data_ptr(), t["tokens"].element_size(), t["offsets"].data_ptr(), t["offsets"].element_size(), _ptr(t["ref"])
        a.pairs, a.beta, a.label_smoothing, a.average = o["pairs"], o["beta"], o["label_smoothing"], o["average"]
        for n in ("chosen", "rejected", "stats", "slopes"):
            setattr(a, n, out[n].data_ptr())
        return a

    def shapes(self, rows):
        P = self.o["pairs"]
        return {"tokens": (_IDS, (rows,)), "offsets": (_IDS, (2 * P + 1,)), "ref": (_F32, (rows,)), "weight": (_F32, (P,)),
                "stats": (_F32, (rows, 4)), "slopes": (_F32, (2 * P,))}


def _returned(out):
    return tuple(t for n, t in out.items() if n not in ("stats", "slopes"))


class _LossOf(torch.autograd.Function):
    @staticmethod
    def forward(ctx, kind, o, names, *tensors):
        it = kind(dict(zip(names, tensors)), o)
        held = it.grad() if kind.at_once and not _capturing(it.t["logits"].device) else None
        out = it.forward(held)
        ctx.save_for_backward(*tensors, *(out[n] for n in kind.saved))
        x = it.t["logits"]
        ctx.like = x.shape, x.dtype, x.device
        ctx.kind, ctx.o, ctx.names, ctx.held = kind, o, names + kind.saved, [held]
        ctx.set_materialize_grads(False)
        returned = _returned(out)
        ctx.mark_non_differentiable(*returned[1:])
        return returned

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g, *_):
        none = (None,) * (3 + len(ctx.names) - len(ctx.kind.saved))
        tensors = ctx.saved_tensors                # (raises where one of them was written since)
        if g is None:
            return none
        t = dict(zip(ctx.names, tensors))
        (rows, V), dtype, device = ctx.like
        t["logits"] = _kept(t["logits"], "logits", (dtype,), (rows, V), device, rows_apart=True)
        if t["mask"] is not None:
            t["mask"] = _kept(t["mask"], "mask", (torch.int32,), (rows, (V + 31) // 32), device)
        it = ctx.kind(t, ctx.o)
        for n, (dtypes, shape) in it.shapes(rows).items():
            if t[n] is not None:
                t[n] = _kept(t[n], n, dtypes, shape, device)
        g = _kept(g.to(torch.float32), "gradient", _F32, (), device)
        # The gradient for g = 1 is handed out once: whoever has it may write it.  What a capture records may run again under another g.
        held = None if _capturing(device) else _pop(ctx.held)
        grad = held if held is not None else it.grad()
        out = it.outputs()
        out.update((n, t[n]) for n in ctx.kind.saved)
        it.backward(out, g, held is not None, grad)
        at = ctx.names.index("logits")
        return none[:3 + at] + (grad,) + none[4 + at:]


def _run(kind, t, o):
    if torch.is_grad_enabled() and t["logits"].requires_grad:
        return _LossOf.apply(kind, o, tuple(t), *t.values())
    return _returned(kind(t, o).forward(None))


def _checked(logits, mask, temperature):
    _not_traced()
    _matrix(logits, "logits", _DTYPES, contiguous=False)
    _need(logits.shape[1] > 0, "logits: no columns")
    _mask_ptr(mask, logits.shape[0], logits.shape[1], logits.device)
    return _number(temperature, "temperature", 2.0 ** -126, torch.finfo(torch.float32).max)


def distill_loss(logits, teacher_ids, teacher_values, mask=None, *, temperature=1.0, rest=False, weight=None):
    """Divergence of softmax(logits / temperature) over what the mask allows from a teacher of whom the most probable tokens are known, as DistillLoss.

    teacher_ids: int32 or int64 [rows, n], n up to 1024, negative where there is none; teacher_values: fp32 or bf16 [rows, n].  Of the listed tokens those count that the student allows.
    The teacher's shares are softmax(teacher_values / temperature) over them: logits, or log probabilities, of the teacher.  With rest=True they are e^teacher_values -- log probabilities, at that
    temperature, as token_logprobs reports them -- and what is missing from 1 is the share of all other tokens together, which the student's probability of these is held to
    (where there are none, or the listed shares are 1 or more, nothing is).  With rest=True the report is to be one under the same mask: what the teacher gave to tokens that `mask` forbids counts to what is
    missing, and so teaches the allowed tokens that are not listed, where rest=False shares it among the listed ones.  A row of which no token counts: loss 0, no gradient."""
    got = _native_losses.distill_loss(logits, teacher_ids, teacher_values, mask, temperature, bool(rest), weight)
    if got is not None:
        return DistillLoss(*got)
    temperature = _checked(logits, mask, temperature)
    _need(isinstance(teacher_ids, torch.Tensor) and teacher_ids.dim() == 2 and 1 <= teacher_ids.shape[1] <= 1024, "teacher_ids: [rows, 1..1024] is wanted")
    shape = (logits.shape[0], teacher_ids.shape[1])
    _constant(teacher_ids, "teacher_ids", _IDS, shape, logits.device)
    _constant(teacher_values, "teacher_values", tuple(_DTYPES), shape, logits.device)
    if weight is not None:
        _constant(weight, "weight", _F32, shape[:1], logits.device)
    t = {"logits": logits, "ids": teacher_ids, "values": teacher_values, "mask": mask, "weight": weight}
    return DistillLoss(*_run(_Distill, t, {"temperature": temperature, "rest": bool(rest), "listed": shape[1]}))


def policy_loss(logits, tokens, old_logprobs, advantages, mask=None, *, ref_logprobs=None, temperature=1.0, clip=(0.2, 0.2), kl_weight=0.0, entropy_weight=None, weight=None):
    """Clipped loss of a policy, as PolicyLoss: with lp the log probability of a row's token under softmax(logits / temperature) over what the mask allows, ratio = e^(lp - old_logprobs),
    - min(ratio A, clamp(ratio, 1 - clip[0], 1 + clip[1]) A), A the advantage; with ref_logprobs + kl_weight (e^(ref - lp) - (ref - lp) - 1); with entropy_weight (0.0 to
    have it reported alone) - entropy_weight x entropy.

    tokens: int32 or int64 [rows]; old_logprobs, advantages, ref_logprobs, weight: fp32 [rows].  A negative token is padding: loss, log probability and entropy 0, no gradient.  A token
    that is not allowed: log probability -inf, loss 0, no gradient.  An id beyond V: NaN."""
    if type(clip) is tuple and len(clip) == 2:
        got = _native_losses.policy_loss(logits, tokens, old_logprobs, advantages, mask, ref_logprobs, temperature, *clip, kl_weight, entropy_weight is not None, entropy_weight or 0.0, weight)
        if got is not None:
            return PolicyLoss(*got)
    temperature = _checked(logits, mask, temperature)
    shape, dev = (logits.shape[0],), logits.device
    _constant(tokens, "tokens", _IDS, shape, dev)
    for t, what in ((old_logprobs, "old_logprobs"), (advantages, "advantages"), (ref_logprobs, "ref_logprobs"), (weight, "weight")):
        if t is not None or what in ("old_logprobs", "advantages"):
            _constant(t, what, _F32, shape, dev)
    _need(isinstance(clip, (tuple, list)) and len(clip) == 2, "clip: two numbers are wanted")
    o = {"temperature": temperature, "clip": (_number(clip[0], "clip", 0.0), _number(clip[1], "clip", 0.0)), "kl_weight": _number(kl_weight, "kl_weight", -1e300, 1e300),
         "entropy": entropy_weight is not None, "entropy_weight": _number(entropy_weight or 0.0, "entropy_weight", -1e300, 1e300)}
    _need(ref_logprobs is not None or o["kl_weight"] == 0.0, "kl_weight: there are no ref_logprobs")
    t = {"logits": logits, "tokens": tokens, "old": old_logprobs, "advantages": advantages, "ref": ref_logprobs, "mask": mask, "weight": weight}
    got = _run(_Policy, t, o)
    return PolicyLoss(*got, *(None,) * (4 - len(got)))


def preference_loss(logits, tokens, offsets, ref_logprobs=None, mask=None, *, beta=0.1, label_smoothing=0.0, average=False, temperature=1.0, weight=None):
    """Loss of paired sequences, as PreferenceLoss: with D_s the sum (average=True: the mean) of lp - ref_logprobs over a sequence's tokens, chosen = beta D_2i, rejected = beta D_2i+1 and h = chosen - rejected,
    - (1 - label_smoothing) ln sigma(h) - label_smoothing ln sigma(-h), sigma(h) = 1 / (1 + e^-h).

    offsets: int32 or int64 [2 pairs + 1]: sequence s has the rows offsets[s] up to offsets[s + 1]; of each pair the preferred one comes first.  tokens: int32 or int64 [rows], ref_logprobs:
    fp32 [rows]; weight: fp32 [pairs].  Negative tokens (prompts) and rows of no sequence are passed over.  A token that is not allowed: log probability -inf, no gradient of its
    own.  (In both sequences of a pair: a loss of NaN.)  Offsets that descend or leave the rows, or give a row to two sequences: NaN for their pair."""
    got = _native_losses.preference_loss(logits, tokens, offsets, ref_logprobs, mask, beta, label_smoothing, bool(average), temperature, weight)
    if got is not None:
        return PreferenceLoss(*got)
    temperature = _checked(logits, mask, temperature)
    shape, dev = (logits.shape[0],), logits.device
    _constant(tokens, "tokens", _IDS, shape, dev)
    _need(isinstance(offsets, torch.Tensor) and offsets.dim() == 1 and offsets.shape[0] % 2 == 1, "offsets: [2 pairs + 1] is wanted")
    pairs = offsets.shape[0] // 2
    _constant(offsets, "offsets", _IDS, offsets.shape, dev)
    if ref_logprobs is not None:
        _constant(ref_logprobs, "ref_logprobs", _F32, shape, dev)
    if weight is not None:
        _constant(weight, "weight", _F32, (pairs,), dev)
    o = {"temperature": temperature, "pairs": pairs, "beta": _number(beta, "beta", -1e300, 1e300), "label_smoothing": _number(label_smoothing, "label_smoothing", 0.0, 1.0), "average": bool(average)}
    t = {"logits": logits, "tokens": tokens, "offsets": offsets, "ref": ref_logprobs, "mask": mask, "weight": weight}
    return PreferenceLoss(*_run(_Preference, t, o))
