"""The operators' kernels by the rules that choose them: calls large enough, or laid out so, that variants run which smaller ones never reach."""
import math

import pytest
import torch

import paper_2506_01151_amd as zf
from tests.test_operators import DTYPES, U, bounds_of, check_head, check_logprobs, half_step, head_case, head_want, near, packed, quantized, rows_of, softmax_of, some_tokens

gpu = pytest.mark.gpu


# ---- the gradient in segments of four pieces a thread: 512 of them at least (4,096 fp32 or 8,192 bf16 logits each) ----
@gpu
@pytest.mark.parametrize("layout", ["packed", "odd"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,rows,V,n,top", [("f32", 300, 9001, 6, 5), ("bf16", 300, 16391, 6, 5), ("f32", 513, 4096, 1, 0), ("bf16", 520, 8192, 2, 0), ("f32", 520, 515, 40, 3), ("bf16", 257, 8193, 0, 2)])
def test_gradients_of_many_segments(dtype, rows, V, n, top, masked, layout):
    """Ends of rows inside a segment and at one's, masks across the pieces, repeated, padded and missing tokens in each segment."""
    g = torch.Generator().manual_seed(rows + V)
    x = (torch.randn((rows, V), generator=g) * 2).to(DTYPES[dtype])
    bits = None
    if masked:
        bits = torch.rand((rows, V), generator=g) < torch.rand((rows, 1), generator=g)
        bits[rows // 2] = False
        bits[0] = True
    tokens = some_tokens(rows, V, n, bits, g, torch.int64 if V % 2 else torch.int32)
    if n > 3:
        tokens[:, n - 1] = V - 1                           # the last one, where the segment is cut short
    check_logprobs(x, tokens, bits, 0.9, top, layout, padding=True)


# ---- tensors beyond 256 MiB, whose rows pass the cache by ----
@gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,rows,V", [("f32", 520, 131076), ("bf16", 1040, 131080), ("f32", 2100, 32764), ("f32", 4200, 16380), ("bf16", 4200, 32760), ("f32", 17000, 4092), ("bf16", 17000, 8184)])
def test_logits_that_pass_the_cache_by(dtype, rows, V, masked):
    """The same bits as in two calls of half the rows, which do not pass it by; some rows against 64 bits."""
    t = DTYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.empty((rows, V), dtype=t, device="cuda").normal_(0.0, 2.0, generator=g)
    half = rows // 2
    assert x.numel() * x.element_size() > 2 ** 28 >= x[half:].numel() * x.element_size() and x.stride(0) * x.element_size() % 16 == 0
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int32) if masked else None
    tokens = torch.randint(V, (rows,), generator=g, device="cuda")
    tokens[:2] = -1
    g_lp, g_H = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")

    def step(sel):
        on = x[sel].requires_grad_()
        got = zf.token_logprobs(on, tokens[sel], None if mask is None else mask[sel], temperature=0.8, entropy=True, top=3)
        plain = zf.token_logprobs(on.detach(), tokens[sel], None if mask is None else mask[sel], temperature=0.8)
        grad, = torch.autograd.grad((got.logprobs, got.entropy), on, (g_lp[sel], g_H[sel]))
        return [v.detach() for v in (*got, plain.logprobs, grad)]

    whole, parts = step(slice(0, rows)), [step(slice(0, half)), step(slice(half, rows))]
    for k, v in enumerate(whole):
        assert torch.equal(v, torch.cat([p[k] for p in parts])), k
    some = torch.tensor([0, 3, half, rows - 1])
    xs, ts = x[some.cuda()].cpu(), tokens[some.cuda()].cpu()
    bits = None
    if masked:
        words = mask[some.cuda()].cpu().view(len(some), -1, 1)
        bits = ((words >> torch.arange(32, dtype=torch.int32)) & 1).bool().reshape(len(some), -1)[:, :V]
    z, lp, p, any_ = softmax_of(xs, bits, 0.8)
    _, b_lp, b_H = bounds_of(z, lp, p, any_, 0.8)
    at = ts.clamp(min=0)[:, None]
    own_lp, H = torch.where(ts < 0, 0.0, lp.gather(1, at)[:, 0]), -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    near(whole[0][some.cuda()], own_lp, torch.where(ts < 0, 0.0, b_lp.gather(1, at)[:, 0]), "logprobs")
    near(whole[1][some.cuda()], H, b_H, "entropy")
    gl, gh = torch.where((ts >= 0) & (own_lp > -math.inf), g_lp[some.cuda()].cpu().double(), 0.0), g_H[some.cuda()].cpu().double()
    lp0, b0 = torch.where(p > 0, lp, 0.0), b_lp.nan_to_num(0.0, 0.0, 0.0)
    want = p * (-gl[:, None] - gh[:, None] * (lp0 + H[:, None]))
    size = p * (gl.abs()[:, None] + gh.abs()[:, None] * (lp0.abs() + H.abs()[:, None]))
    # p carries the bound of its logarithm and three roundings, the bracket those of lp and H, the whole some more
    bound = size * (b0 + 9 * U) + p * gh.abs()[:, None] * (b0 + b_H[:, None])
    want.scatter_add_(1, at, gl[:, None])
    bound.scatter_add_(1, at, 7 * U * gl.abs()[:, None])
    want, bound = want / 0.8, bound / 0.8
    near(whole[5][some.cuda()], want, bound + half_step(t) * (want.abs() + bound) + 2.0 ** -120, "gradient")


# ---- two blocks of bf16 at once: more than 32,768 blocks ----
@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", [(2051, 2300, "packed"), (32769, 100, "packed"), (2051, 2300, "odd"), (33001, 128, "padded"), (16385, 257, "odd")])
def test_quantize_many_blocks(rows, cols, layout, dtype):
    """Numbers of blocks that two at a time, or sixteen groups of two, do not divide: the bytes and scales themselves."""
    g = torch.Generator().manual_seed(rows)
    x = (torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g))).to(DTYPES[dtype])
    q, scale = zf.quantize_blocks(rows_of(x, layout))
    want_q, want_scale = quantized(x, 1)
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(q.cpu().view(torch.uint8), want_q.view(torch.uint8))


# ---- more than 64 rows whose operands' rows lie 2^24 bytes apart: groups of 64 rows past the weight ----
@gpu
@pytest.mark.parametrize("far", ["x", "w"])
@pytest.mark.parametrize("kind", [None, "few", "half"])
@pytest.mark.parametrize("M,V,K", [(70, 300, 384), (130, 257, 1280), (130, 66001, 128)])
def test_head_logits_operands_far_apart(M, V, K, kind, far):
    if far == "w" and V > 300:
        V = 130                                            # (2 GiB of addresses)
    q, qs, wq, ws = head_case(M, V, K, M + V)
    pitch = (1 << 24) + 16

    def apart(t):
        rows = t.shape[0]
        y = torch.empty(((rows - 1) * pitch + K,), dtype=torch.uint8, device="cuda").as_strided((rows, K), (pitch, 1))
        y.copy_(t.view(torch.uint8).cuda())
        return y.view(torch.float8_e4m3fn)

    q_on, w_on = (apart(q), wq.cuda()) if far == "x" else (q.cuda(), apart(wq))
    bits = None
    if kind:
        bits = torch.rand((M, V), generator=torch.Generator().manual_seed(K)) < {"few": 0.2 / M, "half": 0.5}[kind]
        bits[M - 1, V - 1] = True
    mask = None if bits is None else packed(bits, padding=True).cuda()
    want, bound = head_want(q, qs, wq, ws)
    for dtype in (torch.float32, torch.bfloat16):
        # (bf16 logits: less than 7 x 2^-13 of the sum of the products' sizes, which the 32-bit bound holds (2 * 128 + 2 + K / 128) U of)
        cut = bound if dtype == torch.float32 else bound * (1 + 7 * 2.0 ** -13 / ((2 * 128 + 2 + K // 128) * U))
        check_head(zf.head_logits(q_on, qs.cuda(), w_on, ws.cuda(), mask, dtype=dtype), want, cut, bits)


# ---- tiles of 128, 192 and 256 rows and tokens, those that a rule of sizes chooses, in one round of the compute units and in several ----
@gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(65, 191, 384), (65, 32953, 128), (65, 65887, 256), (65, 49420, 384), (260, 32953, 128), (130, 16486, 640), (130, 32953, 256), (130, 65887, 384), (130, 49420, 128), (260, 49420, 256),
                                   (385, 12494, 384), (385, 16486, 512), (385, 36945, 384), (580, 16486, 640), (385, 49420, 128)])
def test_head_logits_tiles_of_every_shape(M, V, K, dtype, masked):
    q, qs, wq, ws = (t.cuda() for t in head_case(M, V, K, M + V + K))
    x = q.double() * qs.double().repeat_interleave(128, dim=1)
    w = wq.double() * ws.double().repeat_interleave(128, dim=0)[:V].repeat_interleave(128, dim=1)
    want, sizes = x @ w.t(), x.abs() @ w.abs().t()
    # a block's sum in 32 bits, or as the 8-bit instructions make it; two products of scales and the sum over the blocks
    cut = ((2 * 128 + 2 + K // 128) * U + (7 * 2.0 ** -13 if dtype == "bf16" else 0.0)) * sizes
    bits = torch.rand((M, V), generator=torch.Generator().manual_seed(K)) < 0.5 if masked else None
    y = zf.head_logits(q, qs, wq, ws, packed(bits, padding=True).cuda() if masked else None, dtype=DTYPES[dtype])
    allowed = bits.cuda() if masked else torch.ones((M, V), dtype=torch.bool, device="cuda")
    assert (y[~allowed] == -math.inf).all()
    err, want, sizes, cut = ((y.double() - want).abs()[allowed], want[allowed], sizes[allowed], cut[allowed])
    assert (err <= cut + half_step(y.dtype) * (want.abs() + cut)).all()
    if dtype == "bf16":                                    # nearly all of them far within it, as a misplaced scale or block would not be
        assert (err > half_step(y.dtype) * want.abs() + 2.0 ** -13 * sizes).double().mean() < 1e-4
