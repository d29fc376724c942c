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


@gpu
@pytest.mark.parametrize("by", ["position", "name"])       # by name: the binding's own code does it, not the extension module
def test_buffers_that_are_written_again_are_noticed(path, by):
    """A mask or logits that a backward pass still needs, written by this package's own calls: torch's error of such buffers, no gradient under another mask."""
    from workloads import configs
    cfg = configs.CONFIGS[1]
    engine = zf.Engine(cfg.grammar(), cfg.vocab())
    states = zf.StateBatch([engine.new_state() for _ in range(2)])
    x = torch.randn((2, engine.V), generator=torch.Generator().manual_seed(5)).cuda()
    tokens = torch.zeros(2, dtype=torch.int64, device="cuda")
    _, q, s, w, ws, _, _ = operands(rows=2, V=engine.V)

    def call(f, *args, **kw):
        names = {"compute_mask": ("engine", "states", "mask_tensor"), "compute_mask_noalloc": ("engine", "states", "mask_tensor"), "compute_mask_async": ("engine", "states", "mask_tensor"),
                 "compute_mask_apply_async": ("engine", "states", "mask_tensor", "logits"), "apply_mask": ("engine", "logits", "mask_tensor")}[f]
        getattr(zf, f)(**dict(zip(names, args)), **kw) if by == "name" else getattr(zf, f)(*args, **kw)
        if "async" in f:
            zf.mask_wait(engine)

    spare = torch.empty((2, engine.W), dtype=torch.int32, device="cuda")
    writers = {"mask": lambda mask, on: call("compute_mask", engine, states, mask), "noalloc": lambda mask, on: call("compute_mask_noalloc", engine, states, mask),
               "async": lambda mask, on: call("compute_mask_async", engine, states, mask), "apply_async": lambda mask, on: call("compute_mask_apply_async", engine, states, mask, torch.zeros_like(x)),
               "apply_async logits": lambda mask, on: call("compute_mask_apply_async", engine, states, spare, on.detach()),
               "apply_async out": lambda mask, on: call("compute_mask_apply_async", engine, states, spare, torch.zeros_like(x), out=on.detach()),
               "apply": lambda mask, on: call("apply_mask", engine, on.detach(), mask), "apply out": lambda mask, on: call("apply_mask", engine, torch.zeros_like(x), mask, out=on.detach()),
               "head": lambda mask, on: zf.head_logits(q, s, w, ws, out=on.detach())}
    for name, write in writers.items():
        for another in (False, True):                      # the buffers themselves, or others
            mask = torch.empty((2, engine.W), dtype=torch.int32, device="cuda")
            zf.compute_mask(engine, states, mask)
            on = x.clone().requires_grad_()
            loss = zf.token_logprobs(on, tokens, mask, entropy=True).entropy.sum()
            write(*(mask.clone(), on.detach().clone()) if another else (mask, on))
            if another:
                loss.backward()
                assert torch.isfinite(on.grad).all()
            else:
                with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                    loss.backward()
    # tensors of inference mode have no such count, inside it and outside
    with torch.inference_mode():
        mask, on = torch.empty((2, engine.W), dtype=torch.int32, device="cuda"), x.clone()
        call("compute_mask", engine, states, mask)
        call("apply_mask", engine, on, mask)
        zf.head_logits(q, s, w, ws, out=on)
    call("compute_mask", engine, states, mask)
    call("compute_mask_apply_async", engine, states, mask, on)
    zf.head_logits(q, s, w, ws, mask, out=on)
    assert torch.equal(on, zf.head_logits(q, s, w, ws, mask, dtype=torch.float32))


@gpu
def test_head_logits_has_no_derivative(path):
    """Operands that require grad: the result does too, and who follows it back is told.  A result's memory that requires grad, or has to for its operands, is refused.
    quantize_blocks rounds: its results are constants."""
    x, q, s, w, ws, logits, tokens = operands()
    want = zf.head_logits(q, s, w, ws, dtype=torch.float32)
    for k in range(4):
        args = [q, s, w, ws]
        args[k] = args[k].clone().requires_grad_()
        y = zf.head_logits(*args, dtype=torch.float32)
        assert y.requires_grad and torch.equal(y.detach(), want)
        with pytest.raises(RuntimeError, match="no derivative"):
            y.sum().backward()
        refused(lambda: zf.head_logits(*args, out=logits.clone()), "derivative")
        with torch.no_grad():
            assert not zf.head_logits(*args).requires_grad
            out = logits.clone().requires_grad_()
            assert zf.head_logits(*args, out=out) is out
        assert torch.equal(out.detach(), want)
    kept = logits.clone().requires_grad_()
    refused(lambda: zf.head_logits(q, s, w, ws, out=kept), "derivative")
    assert torch.equal(kept.detach(), logits)
    assert not any(t.requires_grad for t in zf.quantize_blocks(x.clone().requires_grad_()))


@gpu
def test_tracing_is_refused(path):
    """A traced program would hold the results of the example's inputs as constants."""
    from torch.fx.experimental.proxy_tensor import make_fx
    x, q, s, w, ws, logits, tokens = operands()
    for f, at in ((lambda v: zf.quantize_blocks(v)[1], x), (lambda v: zf.head_logits(q, v, w, ws), s), (lambda v: zf.token_logprobs(v, tokens).logprobs, logits)):
        refused(lambda: make_fx(f)(at), "trace")
        refused(lambda: make_fx(f, pre_dispatch=True)(at), "trace")
        refused(lambda: make_fx(f, tracing_mode="fake")(at), "trace")
        refused(lambda: torch.jit.trace(f, (at,), check_trace=False), "trace")
        f(at)


@gpu
def test_other_dispatch_modes_change_nothing(path):
    from torch.utils._python_dispatch import TorchDispatchMode

    class Through(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    x, q, s, w, ws, logits, tokens = operands()

    def calls():
        on = logits.clone().requires_grad_()
        got = zf.token_logprobs(on, tokens, entropy=True, top=3)
        grad, = torch.autograd.grad(got.logprobs.sum() + got.entropy.sum(), on)
        return [t.detach() for t in (*zf.quantize_blocks(x), zf.head_logits(q, s, w, ws), *got, grad)]

    want = calls()
    with Through():
        got = calls()
    assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want))


class Spread:
    """Saved tensors in every other place of a larger one, the places between filled with something else."""

    def __enter__(self):
        def pack(t):
            big = torch.full((*t.shape[:-1], 2 * t.shape[-1]), 77, dtype=t.dtype, device=t.device)
            big[..., ::2] = t
            return big
        self.hooks = torch.autograd.graph.saved_tensors_hooks(pack, lambda big: big[..., ::2])
        return self.hooks.__enter__()

    def __exit__(self, *e):
        return self.hooks.__exit__(*e)


@gpu
def test_saved_tensors_come_back_as_their_hooks_give_them(path):
    """In another layout, or by way of the host: the same gradient."""
    _, _, _, _, _, logits, tokens = operands(rows=4, V=1001)
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (4, 32), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()

    def grad():
        on = logits.clone().requires_grad_()
        got = zf.token_logprobs(on, tokens[:, None].repeat(1, 3), mask, entropy=True, top=4)
        return on, (got.logprobs.nan_to_num(0, 0, 0).sum() * 0.5 + got.entropy.square().sum() + got.top_logprobs.sum())

    on, loss = grad()
    want, = torch.autograd.grad(loss, on)
    for hooks in (Spread(), torch.autograd.graph.save_on_cpu(), torch.autograd.graph.save_on_cpu(pin_memory=True)):
        with hooks:
            on, loss = grad()
        got, = torch.autograd.grad(loss, on)
        assert torch.equal(got, want)


@gpu
def test_saved_tensors_that_came_back_as_others_are_refused(path):
    """Left on the host, of another type or shape: an error before anything is read."""
    _, _, _, _, _, logits, tokens = operands(rows=4, V=1001)
    mask = torch.full((4, 32), -1, dtype=torch.int32, device="cuda")

    def only(pick, change):
        return torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: change(t) if pick(t) else t)

    def lost(pick, change):
        on = logits.clone().requires_grad_()
        with only(pick, change):
            got = zf.token_logprobs(on, tokens, mask, entropy=True, top=4)
            loss = got.logprobs.sum() + got.entropy.sum() + got.top_logprobs.sum()
        with pytest.raises(RuntimeError, match="saved"):
            loss.backward()

    for pick in (lambda t: tuple(t.shape) == (4, 1001), lambda t: tuple(t.shape) == (4, 32), lambda t: t.dtype == torch.int64, lambda t: tuple(t.shape) == (4,) and t.dtype == torch.float32,
                 lambda t: tuple(t.shape) == (4, 4) and t.dtype == torch.int32, lambda t: tuple(t.shape) == (4, 4) and t.dtype == torch.float32, lambda t: tuple(t.shape) == (4, 2)):
        for change in (lambda t: t.cpu(), lambda t: t[:2], lambda t: t.to(torch.float16), lambda t: t.to_sparse(), lambda t: t[..., :1] if t.dim() > 1 else t[:1]):
            lost(pick, change)


@gpu
def test_negated_views_are_refused_or_resolved(path):
    """A view that stands for its memory's negative (torch's imaginary parts of conjugates are such): refused as an input, its values taken as a gradient."""
    x, q, s, w, ws, logits, tokens = operands()
    mask = torch.full((3, 10), -1, dtype=torch.int32, device="cuda")
    neg = torch._neg_view
    for call in (lambda: zf.quantize_blocks(neg(x)), lambda: zf.head_logits(q, neg(s), w, ws), lambda: zf.head_logits(q, s, w, neg(ws)), lambda: zf.head_logits(q, s, w, ws, neg(mask)), lambda: zf.head_logits(q, s, w, ws, out=neg(logits)),
                 lambda: zf.token_logprobs(neg(logits), tokens), lambda: zf.token_logprobs(logits, neg(tokens)), lambda: zf.token_logprobs(logits, tokens, neg(mask))):
        refused(call, "negated")
    on = logits.clone().requires_grad_()
    got = zf.token_logprobs(on, tokens, entropy=True, top=2)
    gs = [torch.randn(t.shape, generator=torch.Generator().manual_seed(9)).cuda() for t in (got.logprobs, got.entropy, got.top_logprobs)]
    outs = (got.logprobs, got.entropy, got.top_logprobs)
    want, = torch.autograd.grad(outs, on, [-g for g in gs], retain_graph=True)
    grad, = torch.autograd.grad(outs, on, [neg(g) for g in gs])
    assert torch.equal(grad, want)


@gpu
def test_no_memory_is_torch_s_own_error(path):
    """What torch's other calls raise then, which programs catch to try a smaller batch."""
    x, q, s, w, ws, logits, _ = operands()
    x, many = torch.zeros((1 << 22, 1), device="cuda"), torch.zeros((1 << 17, 128), device="cuda").to(torch.float8_e4m3fn)
    scale = torch.ones((1 << 17, 1), device="cuda")
    torch.cuda.empty_cache()
    free, total = torch.cuda.mem_get_info()
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (64 << 20)) / total)      # (a limit of torch's allocator: the device is not asked)
    try:
        for call in (lambda: zf.quantize_blocks(x), lambda: zf.head_logits(many, scale, many[:4096], scale[:32])):
            with pytest.raises(torch.OutOfMemoryError):
                call()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert zf.quantize_blocks(x[:128])[0].shape == (128, 128)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("grad", [False, True])
def test_the_extension_module_does_what_the_definition_does(monkeypatch, dtype, grad):
    """The same bits of every result and gradient, with everything asked for and with parts of it; the same refusals."""
    from paper_2506_01151_amd import operators as ops
    taken = ops._native_ops
    g = torch.Generator().manual_seed(31)

    class Untaken:
        quantize_blocks = head_logits = token_logprobs = staticmethod(lambda *a: None)

    def both(call):
        res = []
        for module in (taken, Untaken):
            monkeypatch.setattr(ops, "_native_ops", module)
            try:
                res.append([t if t is None else t.detach().float().cpu() for t in call()])
            except zf.ZfError as e:
                res.append((e.code, str(e)))
        monkeypatch.setattr(ops, "_native_ops", taken)
        assert len(res[0]) == len(res[1])
        for a, b in zip(*res):
            assert type(a) is type(b) and (torch.equal(a.nan_to_num(9.0, 8.0, 7.0), b.nan_to_num(9.0, 8.0, 7.0)) if isinstance(a, torch.Tensor) else a == b), (a, b)

    for rows, V, n, top, entropy, masked, layout in ((1, 1, 0, 1, True, False, "packed"), (5, 700, 1, 0, True, True, "padded"), (3, 40037, 4, 7, False, True, "odd"), (2, 9001, None, 3, True, True, "packed"), (33, 515, 0, 0, False, False, "odd"),
                                                     (4, 32768, 70, 64, True, False, "padded"), (6, 33, None, 0, True, False, "packed")):
        buf = torch.randn((rows * (V + 5) + 1,), generator=g).to(dtype).cuda()
        x = buf[1:].view(rows, V + 5)[:, :V] if layout != "packed" else buf[:rows * V].view(rows, V)
        if layout == "padded":
            x = torch.nn.functional.pad(x, (0, 64 - V % 64))[:, :V]
        tokens = None if n is None else torch.randint(-1, V + 1, (rows, n) if n else (rows,), generator=g).to(torch.int32 if V % 2 else torch.int64).cuda()
        mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, (V + 31) // 32), generator=g, dtype=torch.int32).cuda() if masked else None

        def call():
            on = x.detach().requires_grad_(grad)
            got = zf.token_logprobs(on, tokens, mask, temperature=0.7, entropy=entropy, top=top)
            if not grad:
                return got
            outs = [t for t in (got.logprobs, got.entropy, got.top_logprobs) if t is not None]
            res = list(got)
            for some in [outs] + ([[t] for t in outs] if outs else []):
                if some:
                    ws = [torch.linspace(-1, 2, t.numel(), device="cuda").view(t.shape) for t in some]
                    res += torch.autograd.grad(some, on, ws, retain_graph=True)
            return res

        both(call)
    for rows, cols in ((1, 1), (130, 300), (5, 4096), (257, 1000)):
        x = torch.randn((rows, cols), generator=g).to(dtype).cuda()
        for block_rows in (1, 128):
            both(lambda: [t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in zf.quantize_blocks(x, block_rows=block_rows)])
    for M, V, K in ((1, 300, 256), (33, 9001, 384), (130, 515, 128)):
        q, s = zf.quantize_blocks(torch.randn((M, K), generator=g).cuda())
        w, ws = zf.quantize_blocks(torch.randn((V, K), generator=g).cuda(), block_rows=128)
        mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (M, (V + 31) // 32), generator=g, dtype=torch.int32).cuda()
        both(lambda: [zf.head_logits(q, s, w, ws, dtype=dtype)])
        both(lambda: [zf.head_logits(q, s, w, ws, mask, dtype=dtype)])
    x = torch.zeros((2, 256), device="cuda", dtype=dtype, requires_grad=grad)
    t, m = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    for bad in (lambda: zf.quantize_blocks(x, block_rows=2), lambda: zf.quantize_blocks(x.half()), lambda: zf.quantize_blocks(x.t()), lambda: zf.quantize_blocks(x.detach()[:1].expand(3, 256)), lambda: zf.token_logprobs(x, t, m[:, :7]),
                lambda: zf.token_logprobs(x, t, top=65), lambda: zf.token_logprobs(x, t, temperature=0.0), lambda: zf.token_logprobs(x, t, temperature=1e-40), lambda: zf.token_logprobs(x, t, temperature=1e39), lambda: zf.token_logprobs(x, t.float()),
                lambda: zf.token_logprobs(x, t.cpu()), lambda: zf.token_logprobs(x, t[:1]), lambda: zf.token_logprobs(x, torch.zeros((2, 1025), dtype=torch.int64, device="cuda"))):
        both(bad)
