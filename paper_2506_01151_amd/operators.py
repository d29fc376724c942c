"""The two ends of a step's logits: the head's product that makes them, the log probabilities that are read from them.

    q, q_scale = quantize_blocks(hidden)                          # activations to 8 bits, a scale for 128 columns
    logits = head_logits(q, q_scale, weight, weight_scale, mask)  # -inf where the mask does not allow the token
    got = token_logprobs(logits, tokens, mask, entropy=True, top=5)
    got.logprobs.sum().backward()                                 # the logits' gradient under the same mask

Masks are those of compute_mask.  Every call is enqueued on torch's current stream of the tensors' device, waits for nothing and
allocates through torch only, so it can be captured into a graph (a backward pass as any of torch's: from leaves made for the
capture, no eager graph of theirs alive).  Arguments that do not fit raise ZfError (ZF_ERR_INVALID_ARG), tensors with a tangent among them: there are no
forward-mode derivatives.  Nor can the calls be traced (torch.jit.trace, make_fx): they refuse.
"""
import ctypes
import sys
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import _native_ops
from .binding import ZF_ERR_INVALID_ARG, LogprobsArgs, ZfError, _check, load_library

BLOCK = 128                                        # columns that share a scale, and rows of a weight that do
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


_lib = load_library()
_native_ops.bind({n: ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in (
    "zf_quantize_blocks", "zf_head_logits", "zf_token_logprobs_workspace", "zf_token_logprobs", "zf_token_logprobs_backward", "zf_last_error")}, _check)
# The ordinary call is _native_ops' (csrc/zf_py_ops.cpp); what it does not take it answers with None, and the code here, its definition, does or refuses it.


class TokenLogprobs(NamedTuple):
    logprobs: Optional[torch.Tensor]               # fp32, the shape of tokens
    entropy: Optional[torch.Tensor]                # fp32 [rows]
    top_ids: Optional[torch.Tensor]                # int32 [rows, top]
    top_logprobs: Optional[torch.Tensor]           # fp32 [rows, top]


def _need(ok, why):
    if not ok:
        raise ZfError(ZF_ERR_INVALID_ARG, why)


def _plain(t, what):
    """A kernel is given the tensor's address: what else there is to a tensor would be lost."""
    _need(not t.is_neg(), f"{what}: a negated view is not taken (resolve_neg makes a tensor of it)")
    _need(not torch._C._functorch.is_functorch_wrapped_tensor(t) and forward_ad.unpack_dual(t).tangent is None, f"{what}: there is no forward-mode derivative, nor another of torch.func's transforms")


def _not_traced():
    """torch.jit.trace and make_fx see none of what these calls do, and would keep the results as constants."""
    proxies = sys.modules.get("torch.fx.experimental.proxy_tensor")
    _need(not torch.jit.is_tracing() and (proxies is None or proxies.get_proxy_mode() is None), "these calls cannot be traced")


def _matrix(t, what, dtypes, rows=None, cols=None, contiguous=True):
    _need(isinstance(t, torch.Tensor) and t.layout == torch.strided and t.is_cuda, f"{what}: a tensor on the GPU is wanted")
    _plain(t, what)
    _need(t.dtype in dtypes, f"{what}: {t.dtype} is none of {', '.join(map(str, dtypes))}")
    _need(t.dim() == 2 and (rows is None or t.shape[0] == rows) and (cols is None or t.shape[1] == cols),
          f"{what}: a matrix of {'any' if rows is None else rows} x {'any' if cols is None else cols} is wanted, not {tuple(t.shape)}")
    _need(t.is_contiguous() if contiguous else t.shape[1] <= 1 or t.stride(1) == 1, f"{what}: {'a contiguous matrix is' if contiguous else 'rows without gaps are'} wanted")


def _row_stride(t):
    """Elements between rows; what a matrix of one row says does not matter.  The library refuses rows that overlap."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _mask_ptr(mask, rows, V, device):
    if mask is None:
        return None
    _matrix(mask, "mask", (torch.int32,), rows, (V + 31) // 32)
    _need(mask.device == device, "mask: on another device")
    return mask.data_ptr()


def _stream(device):
    return torch._C._cuda_getCurrentRawStream(device.index)


def quantize_blocks(x, *, block_rows=1):
    """x (fp32 or bf16 [rows, cols]) as (q, scale): e4m3 [rows, cols padded with zeros to a multiple of 128] and fp32 scales, one for 128 columns
    of block_rows = 1 row (activations) or of 128 rows (a head's weight).  Both are constants to autograd, as those of x.detach(), also where x requires grad."""
    got = _native_ops.quantize_blocks(x, block_rows)
    if got is not None:
        return got
    _not_traced()
    _matrix(x, "x", _DTYPES, contiguous=False)
    _need(block_rows in (1, BLOCK), "block_rows must be 1 or 128")
    rows, cols = x.shape
    _need(cols > 0, "x: no columns")
    blocks = -(-cols // BLOCK)
    q = torch.empty((rows, blocks * BLOCK), dtype=torch.float8_e4m3fn, device=x.device)
    scale = torch.empty((-(-rows // block_rows), blocks), dtype=torch.float32, device=x.device)
    _check(_lib.zf_quantize_blocks(x.data_ptr(), _DTYPES[x.dtype], rows, cols, _row_stride(x), block_rows, q.data_ptr(), scale.data_ptr(), x.device.index, _stream(x.device)))
    return q, scale


class _NoDerivative(torch.autograd.Function):
    """The result of a call, tied to its operands by a node that raises when it is followed back."""

    @staticmethod
    def forward(ctx, call, *operands):
        return call()

    @staticmethod
    def backward(ctx, *g):
        raise ZfError(ZF_ERR_INVALID_ARG, "head_logits: there is no derivative; detach its operands, or take the product in another type")


def head_logits(q, q_scale, weight, weight_scale, mask=None, *, dtype=torch.bfloat16, out=None):
    """Logits [batch, V] of activations q [batch, K] against a head's weight [V, K], both e4m3 with K a multiple of 128, scales [batch, K / 128] and
    [ceil(V / 128), K / 128] (quantize_blocks makes all four).  Under a mask the logits of tokens that it does not allow are -inf, and
    rows of the weight that none of a batch of up to 64 allows are not read (a larger batch reads all: where its rows allow few tokens, calls of 64 rows each are quicker).  fp32 logits are sums in 32 bits; bf16 ones come from 8-bit matrix instructions, which are off by about 1.3e-5 of the norm of a logit's
    products (less than 7 x 2^-13 of the sum of their sizes) before they are rounded.  dtype: fp32 or bf16; out: rows of the result without gaps.  There is no derivative: where an operand requires grad the result does,
    and a backward pass that reaches it raises; out= is refused then, and an out that requires grad itself, as torch's own calls do."""
    if out is None:
        got = _native_ops.head_logits(q, q_scale, weight, weight_scale, mask, _DTYPES.get(dtype, -1))
        if got is not None:
            return got
    _not_traced()
    for t, what in ((q, "q"), (weight, "weight")):
        _matrix(t, what, (torch.float8_e4m3fn,), contiguous=False)
    batch, K, V = q.shape[0], q.shape[1], weight.shape[0]
    _need(K > 0 and K % BLOCK == 0 and weight.shape[1] == K, f"q and weight: the same number of columns, a multiple of {BLOCK}, is wanted, not {K} and {weight.shape[1]}")
    _need(V > 0, "weight: no rows")
    _matrix(q_scale, "q_scale", (torch.float32,), batch, K // BLOCK)
    _matrix(weight_scale, "weight_scale", (torch.float32,), -(-V // BLOCK), K // BLOCK)
    followed = torch.is_grad_enabled() and any(t.requires_grad for t in (q, q_scale, weight, weight_scale))
    if out is None:
        _need(dtype in _DTYPES, f"dtype: {dtype} is neither fp32 nor bf16")
    else:
        _matrix(out, "out", _DTYPES, batch, V, contiguous=False)
        _need(not followed and not (torch.is_grad_enabled() and out.requires_grad), "out: there is no derivative, and it or an operand requires grad")
    for t, what in ((q_scale, "q_scale"), (weight, "weight"), (weight_scale, "weight_scale"), (q if out is None else out, "out")):
        _need(t.device == q.device, f"{what}: on another device than q")
    mask_ptr = _mask_ptr(mask, batch, V, q.device)

    def call():
        y = torch.empty((batch, V), dtype=dtype, device=q.device) if out is None else out
        if out is not None:
            torch.autograd.graph.increment_version(out)    # written by its address: a backward pass that has kept it is told
        _check(_lib.zf_head_logits(q.data_ptr(), _row_stride(q), q_scale.data_ptr(), weight.data_ptr(), _row_stride(weight), weight_scale.data_ptr(),
                                   batch, V, K, mask_ptr, y.data_ptr(), _DTYPES[y.dtype], _row_stride(y), q.device.index, _stream(q.device)))
        return y

    return _NoDerivative.apply(call, q, q_scale, weight, weight_scale) if followed else call()


def _logprobs_args(logits, tokens, mask, temperature, top):
    a = LogprobsArgs()
    a.logits, a.dtype, a.V, a.rows, a.row_stride = logits.data_ptr(), _DTYPES[logits.dtype], logits.shape[1], logits.shape[0], _row_stride(logits)
    a.mask = _mask_ptr(mask, logits.shape[0], logits.shape[1], logits.device)
    a.temperature, a.top = temperature, top
    if tokens is not None:
        a.tokens, a.token_bytes, a.n_tokens = tokens.data_ptr(), tokens.element_size(), tokens.shape[1] if tokens.dim() == 2 else 1
    return a


def _forward(logits, tokens, mask, temperature, entropy, top, stats):
    """(logprobs, entropy, top_ids, top_logprobs, stats), each None where it is not wanted."""
    lib, rows, dev = _lib, logits.shape[0], logits.device
    a = _logprobs_args(logits, tokens, mask, temperature, top)
    f32 = dict(dtype=torch.float32, device=dev)
    out = (torch.empty(tokens.shape, **f32) if tokens is not None else None, torch.empty(rows, **f32) if entropy else None,
           torch.empty((rows, top), dtype=torch.int32, device=dev) if top else None, torch.empty((rows, top), **f32) if top else None,
           torch.empty((rows, 2), **f32) if stats else None)
    a.logprobs, a.entropy, a.top_ids, a.top_logprobs, a.stats = (t.data_ptr() if t is not None else None for t in out)
    size = lib.zf_token_logprobs_workspace(ctypes.byref(a))
    if size < 0:
        _check(size)
    work = torch.empty(size, dtype=torch.uint8, device=dev)
    _check(lib.zf_token_logprobs(ctypes.byref(a), work.data_ptr(), size, dev.index, _stream(dev)))
    return out


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, mask, temperature, entropy, top):
        lp, H, ids, top_lp, stats = _forward(logits, tokens, mask, temperature, entropy, top, True)
        ctx.save_for_backward(logits, tokens, mask, lp, H, ids, top_lp, stats)
        ctx.temperature = temperature
        if ids is not None:
            ctx.mark_non_differentiable(ids)
        ctx.set_materialize_grads(False)
        return lp, H, ids, top_lp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_lp, g_H, _, g_top):
        return _backward(*ctx.saved_tensors, ctx.temperature, g_lp, g_H, g_top), None, None, None, None, None


def _kept(t, what, dtypes, shape, device, rows_apart=False):
    """A saved tensor, or an incoming gradient, for a kernel to read: what hooks on saved tensors give back may lie anywhere, in any order."""
    _need(t.layout == torch.strided and t.device == device and t.dtype in dtypes and tuple(t.shape) == tuple(shape), f"saved {what}: {tuple(t.shape)} of {t.dtype} on {t.device} came back instead of {tuple(shape)} on {device}")
    t = t.resolve_neg()
    _plain(t, f"saved {what}")
    as_it_is = t.stride(1) == 1 and _row_stride(t) >= t.shape[1] if rows_apart else t.is_contiguous()
    return t if as_it_is else t.contiguous()


def _backward(logits, tokens, mask, lp, H, ids, top_lp, stats, temperature, g_lp, g_H, g_top):
    _need(logits.is_cuda and logits.dim() == 2, "saved logits: a matrix on the GPU is wanted")
    (rows, V), dev, f32 = logits.shape, logits.device, (torch.float32,)
    logits = _kept(logits, "logits", _DTYPES, (rows, V), dev, rows_apart=True)
    if tokens is not None:
        tokens = _kept(tokens, "tokens", (torch.int32, torch.int64), lp.shape, dev)
        lp = _kept(lp, "logprobs", f32, (rows, *lp.shape[1:2]), dev)
    if mask is not None:
        mask = _kept(mask, "mask", (torch.int32,), (rows, (V + 31) // 32), dev)
    if H is not None:
        H = _kept(H, "entropy", f32, (rows,), dev)
    if ids is not None:
        ids = _kept(ids, "top_ids", (torch.int32,), (rows, *ids.shape[1:2]), dev)
        top_lp = _kept(top_lp, "top_logprobs", f32, ids.shape, dev)
    stats = _kept(stats, "stats", f32, (rows, 2), dev)
    a = _logprobs_args(logits, tokens, mask, temperature, ids.shape[1] if ids is not None else 0)
    a.logprobs, a.entropy, a.top_ids, a.top_logprobs, a.stats = (t.data_ptr() if t is not None else None for t in (lp, H, ids, top_lp, stats))
    g = [_kept(t.to(torch.float32), "gradient", f32, of.shape, dev) if t is not None else None for t, of in ((g_lp, lp), (g_H, H), (g_top, top_lp))]
    grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _check(_lib.zf_token_logprobs_backward(ctypes.byref(a), *(t.data_ptr() if t is not None else None for t in g), grad.data_ptr(), grad.shape[1],
                                                     logits.device.index, _stream(logits.device)))
    return grad


def token_logprobs(logits, tokens=None, mask=None, *, temperature=1.0, entropy=False, top=0):
    """Log probabilities of tokens ([rows] or [rows, n], int32 or int64) under softmax(logits / temperature) over what the mask allows, the rows'
    entropies and their `top` (up to 64) most probable tokens, as TokenLogprobs.  logits: fp32 or bf16 [rows, V], rows without gaps.

    -inf for a token that the mask does not allow, 0 and no gradient for a negative id (padding), NaN for an id beyond V.  Alternatives that there are
    not: id -1, -inf.  temperature: 2^-126 at least.  logprobs, entropy and top_logprobs have gradients for the logits (once; not to be differentiated again).  The backward pass
    reads logits, tokens and mask again: written meanwhile by torch or by this package's calls on tensors, it raises; what is written by a raw address (Engine's methods, other libraries) torch does not see."""
    got = _native_ops.token_logprobs(logits, tokens, mask, float(temperature), bool(entropy), top)
    if got is not None:
        return TokenLogprobs(*got)
    _not_traced()
    _matrix(logits, "logits", _DTYPES, contiguous=False)
    rows, V = logits.shape
    _need(V > 0, "logits: no columns")
    if tokens is not None:
        _need(isinstance(tokens, torch.Tensor) and tokens.device == logits.device and tokens.dtype in (torch.int32, torch.int64), "tokens: int32 or int64 on the logits' device are wanted")
        _plain(tokens, "tokens")
        _need(tokens.dim() in (1, 2) and tokens.shape[0] == rows and tokens.is_contiguous(), f"tokens: a contiguous [{rows}] or [{rows}, n] is wanted, not {tuple(tokens.shape)}")
    _need(isinstance(top, int) and 0 <= top <= 64, "top must be 0..64")
    if torch.is_grad_enabled() and logits.requires_grad:
        return TokenLogprobs(*_TokenLogprobs.apply(logits, tokens, mask, float(temperature), bool(entropy), top))
    return TokenLogprobs(*_forward(logits, tokens, mask, float(temperature), bool(entropy), top, False)[:4])
