"""What torch is told, and asked, by the operators around the logits, which read and write by address: derivatives that there are not, buffers that are written
again, tensors whose address is not all there is to them.  Each by the extension module and by operators.py's own code, which defines the calls."""
import math

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

import paper_2506_01151_amd as zf

gpu = pytest.mark.gpu
INF = math.inf


@pytest.fixture(params=["native", "definition"])
def path(request, monkeypatch):
    """"definition": the extension module takes no call, so that operators.py's code does."""
    from paper_2506_01151_amd import operators as ops
    if request.param == "definition":
        class Untaken:
            quantize_blocks = head_logits = token_logprobs = staticmethod(lambda *a: None)
        monkeypatch.setattr(ops, "_native_ops", Untaken)
    return request.param


def refused(call, says=""):
    with pytest.raises(zf.ZfError) as e:
        call()
    assert e.value.code == zf.ZF_ERR_INVALID_ARG and says in str(e.value), str(e.value)


def operands(rows=3, V=300, cols=256, seed=1):
    """Hidden states, what they and a weight are in 8 bits, logits, tokens, all on the GPU."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g).cuda()
    q, s = zf.quantize_blocks(x)
    w, ws = zf.quantize_blocks(torch.randn((V, cols), generator=g).cuda(), block_rows=128)
    return x, q, s, w, ws, torch.randn((rows, V), generator=g).cuda(), torch.randint(V, (rows,), generator=g).cuda()


@gpu
def test_forward_mode_is_refused(path):
    """A tangent that comes in would be lost: no call of these has a forward-mode derivative.  Tensors without one are taken inside a level as outside."""
    x, q, s, w, ws, logits, tokens = operands()
    want = zf.token_logprobs(logits, tokens, entropy=True, top=2)
    with forward_ad.dual_level():
        def dual(t):
            return forward_ad.make_dual(t, torch.ones_like(t))

        for call in (lambda: zf.quantize_blocks(dual(x)), lambda: zf.quantize_blocks(dual(x), block_rows=128), lambda: zf.head_logits(q, dual(s), w, ws), lambda: zf.head_logits(q, s, w, dual(ws)),
                     lambda: zf.head_logits(q, s, w, ws, out=dual(logits.clone())), lambda: zf.token_logprobs(dual(logits), tokens), lambda: zf.token_logprobs(dual(logits), entropy=True),
                     lambda: zf.token_logprobs(dual(logits.clone().requires_grad_()), tokens, top=3)):
            refused(call, "forward-mode")
        got = zf.token_logprobs(logits, tokens, entropy=True, top=2)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        on = logits.clone().requires_grad_()
        lp = zf.token_logprobs(on, tokens).logprobs
        with pytest.raises(RuntimeError, match="forward-mode"):
            torch.autograd.grad(lp, on, dual(torch.ones_like(lp)))
    for f, at in ((lambda v: zf.token_logprobs(v, tokens).logprobs, logits), (lambda v: zf.quantize_blocks(v)[1], x), (lambda v: zf.head_logits(q, v, w, ws, dtype=torch.float32), s)):
        with pytest.raises(RuntimeError):
            torch.func.jvp(f, (at,), (torch.ones_like(at),))
