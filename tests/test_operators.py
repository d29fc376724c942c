"""The calls at the two ends of a step's logits (quantize_blocks, head_logits, token_logprobs and its gradient) against their
definitions in 64 bits on the CPU, and their refusals.

Tolerances count roundings of u = 2^-24 (a 32-bit result is off by at most u relative to its value), and half a step of the result's type at the end."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2506_01151_amd as zf

gpu = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = math.inf


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- masks and rows ----------------------------------------------------------------------------------
def packed(bits, padding=False):
    """bool [rows, V] -> int32 [rows, ceil(V / 32)]; padding: the bits beyond V are set."""
    rows, V = bits.shape
    W = (V + 31) // 32
    b = np.zeros((rows, W * 32), dtype=bool)
    b[:, :V] = bits.numpy()
    b[:, V:] = padding
    return torch.from_numpy(np.packbits(b, axis=1, bitorder="little").view(np.int32).copy())


def rows_of(x, layout):
    """x on the GPU: its rows one behind the other; at the next multiple of 64 elements; from an odd element on, at odd distances, among other numbers; or 2^30
    elements (and a few) apart, so that the third begins beyond what 31 bits count."""
    rows, V = x.shape
    if layout == "far":
        pitch = 2 ** 30 + 24
        y = torch.empty(((rows - 1) * pitch + V,), dtype=x.dtype, device="cuda").as_strided((rows, V), (pitch, 1))
        y.copy_(x.cuda())
        return y
    if layout == "packed":
        return x.cuda()
    if layout == "padded":
        buf = torch.full((rows, (V + 63) // 64 * 64), 7.0, dtype=x.dtype, device="cuda")
        buf[:, :V] = x.cuda()
        return buf[:, :V]
    pitch = V + 3 - V % 2
    buf = torch.full((rows * pitch + 1,), 7.0, dtype=x.dtype, device="cuda")
    y = buf[1:].view(rows, pitch)[:, :V]
    y.copy_(x.cuda())
    return y


# ---- to 8 bits ---------------------------------------------------------------------------------------
def quantized(x, block_rows):
    """(q as numbers, scale) by the definition: the scale and the quotient in 32 bits, the quotient to the nearest e4m3 number."""
    rows, cols = x.shape
    R, C = -(-rows // block_rows) * block_rows, -(-cols // 128) * 128
    p = torch.zeros((R, C))
    p[:rows, :cols] = x.float()
    t = p.view(R // block_rows, block_rows, C // 128, 128)
    scale = torch.maximum(t.abs().amax(dim=(1, 3)).double().div(448.0).float(), torch.tensor(2.0 ** -126))
    q = (t / scale[:, None, :, None]).clamp(-448.0, 448.0).reshape(R, C)[:rows]
    return q.to(torch.float8_e4m3fn), scale


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", [(1, 1, "packed"), (1, 128, "packed"), (3, 127, "odd"), (127, 129, "odd"), (129, 256, "padded"), (300, 1000, "packed"), (5, 4096, "odd"), (257, 640, "packed")])
def test_quantize_bit_exact(rows, cols, layout, dtype, block_rows):
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g))
    x[0, 0] = 0.0
    x = x.to(DTYPES[dtype])
    q, scale = zf.quantize_blocks(rows_of(x, layout), block_rows=block_rows)
    want_q, want_scale = quantized(x, block_rows)
    assert q.dtype == torch.float8_e4m3fn and tuple(q.shape) == tuple(want_q.shape)
    assert torch.equal(scale.cpu(), want_scale)
    assert torch.equal(q.cpu().view(torch.uint8), want_q.view(torch.uint8))


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_zeros_tiny_infinite_and_nan(block_rows):
    x = torch.zeros((130, 512))
    x[0, 128:256] = 1e-42                                  # denormal: the scale stays at 2^-126
    x[1, 256] = INF
    x[1, 257] = 3.0
    x[2, 384] = math.nan
    x[2, 385] = -5.0
    x[129, 0] = 448.0                                      # the scale is one
    q, scale = (t.cpu() for t in zf.quantize_blocks(x.cuda(), block_rows=block_rows))
    v = q.float()
    assert scale[0, 0] == (2.0 ** -126) and scale[0, 1] == 2.0 ** -126 and torch.equal(v[0, 128:256], torch.full((128,), 1e-42 * 2.0 ** 126).to(torch.float8_e4m3fn).float())
    assert scale[0 if block_rows > 1 else 1, 2] == INF and math.isnan(v[1, 256]) and v[1, 257] == 0.0
    assert math.isnan(v[2, 384]) and v[2, 385] == -448.0 and scale[0 if block_rows > 1 else 2, 3] == torch.tensor(5.0) / torch.tensor(448.0)
    assert v[129, 0] == 448.0 and scale[1 if block_rows > 1 else 129, 0] == 1.0
    assert zf.quantize_blocks(torch.empty((0, 256), device="cuda"))[0].shape == (0, 256)


# ---- the head's product ------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_next_to_ties(block_rows):
    """Scales of all sizes, elements within three steps of e4m3's numbers and of the middles between them, zeros of both signs: the bytes themselves."""
    g = torch.Generator().manual_seed(21)
    rows, cols = 512, 2048
    e = torch.randint(-126, 119, (rows // block_rows, 1, cols // 128, 1), generator=g).double()
    scale = (1 + torch.rand(e.shape, generator=g, dtype=torch.float64)) * 2.0 ** e
    few = torch.randint(16, 32, (rows // block_rows, block_rows, cols // 128, 128), generator=g) * 2.0 ** torch.randint(-15, 4, (rows // block_rows, block_rows, cols // 128, 128), generator=g)
    x = (few.double() * scale).float()
    x = (x.view(torch.int32) + torch.randint(-3, 4, x.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    x = torch.where(torch.rand(x.shape, generator=g) < 0.5, -x, x)
    x[..., 5], x[..., 77] = 0.0, -0.0
    x[..., 0:1, :, 9] = (448.0 * scale[..., 0]).float()                       # the largest, so that the scale is near what it was made with
    x = x.reshape(rows, cols)
    want_q, want_scale = quantized(x, block_rows)
    got_q, got_scale = zf.quantize_blocks(x.cuda(), block_rows=block_rows)
    assert torch.equal(got_scale.cpu(), want_scale)
    assert torch.equal(got_q.cpu().view(torch.uint8), want_q.to(torch.float8_e4m3fn).view(torch.uint8))


def head_case(M, V, K, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g) * torch.exp(torch.randn((M, 1), generator=g))
    w = torch.randn((V, K), generator=g) * torch.exp(torch.randn((V, 1), generator=g) / 2) / math.sqrt(K)
    q, qs = quantized(x, 1)
    wq, ws = quantized(w, 128)
    return q, qs, wq, ws


def head_want(q, qs, wq, ws):
    """(logits, bound of their error in 32 bits): a block's 128 products are exact and their sum at most 128 additions, each off by a step (u rounded, 2 u cut off);
    the scales' product, its product with the sum and the sum over the blocks are a rounding each."""
    V, n = wq.shape[0], qs.shape[1]
    x = q.double() * qs.double().repeat_interleave(128, dim=1)
    w = wq.double() * ws.double().repeat_interleave(128, dim=0)[:V].repeat_interleave(128, dim=1)
    return x @ w.t(), (2 * 128 + 2 + n) * U * (x.abs() @ w.abs().t())


def check_head(y, want, bound, bits=None):
    y = y.cpu()
    err = (y.double() - want).abs()
    bound = bound + half_step(y.dtype) * (want.abs() + bound)
    if bits is not None:
        assert (y[~bits] == -INF).all()
        err, bound = err[bits], bound[bits]
    assert (err <= bound).all(), f"off by {(err / bound).max():.3g} of the bound"


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(1, 1, 128), (1, 2048, 1024), (3, 15, 256), (5, 129, 384), (16, 1000, 640), (17, 128, 128), (33, 300, 2048), (64, 257, 896), (65, 1025, 256), (130, 515, 1024), (300, 777, 512), (257, 2048, 768)])
def test_head_logits(M, V, K, dtype):
    q, qs, wq, ws = head_case(M, V, K, M * 7 + V)
    y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), dtype=DTYPES[dtype])
    check_head(y, *head_want(q, qs, wq, ws))


@gpu
@pytest.mark.parametrize("kind", ["few", "half", "nothing", "one", "all", "range"])
@pytest.mark.parametrize("M,V,K", [(1, 1000, 256), (4, 333, 1152), (16, 4096, 128), (40, 515, 640), (100, 1025, 256), (200, 2049, 384)])
def test_head_logits_under_masks(M, V, K, kind):
    """Every share of allowed tokens; weights of tokens that nothing allows are NaN and must not show, nor may those that other rows allow."""
    q, qs, wq, ws = head_case(M, V, K, M + V + len(kind))
    g = torch.Generator().manual_seed(V)
    bits = torch.rand((M, V), generator=g) < {"few": 0.01, "half": 0.5, "nothing": 0.0, "one": 0.0, "all": 1.0, "range": 0.0}[kind]
    if kind == "one":
        bits[M // 2, V - 1] = True
    if kind == "range":
        bits[:, V // 3:V // 3 + 40] = True
    bits[0, 0] = kind == "all"
    wq = wq.clone()
    dead = ~bits.any(dim=0)
    wq.view(torch.uint8)[dead] = 0x7F
    want, bound = head_want(q, qs, wq, ws)
    for padding in (False, True):
        y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), packed(bits, padding).cuda(), dtype=torch.float32)
        check_head(y, want, bound, bits)
    if M > 1 and kind == "half":
        wq.view(torch.uint8)[V // 2] = 0x7F
        y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), packed(bits).cuda(), dtype=torch.float32).cpu()
        assert y[bits[:, V // 2], V // 2].isnan().all() and (y[~bits[:, V // 2], V // 2] == -INF).all()


@gpu
@pytest.mark.parametrize("kind", [None, "few", "some", "half", "mixed"])
@pytest.mark.parametrize("M,V,K", [(1, 8192, 256), (2, 8200, 4224), (7, 9001, 640), (20, 8321, 1152), (33, 8193, 2304), (64, 8320, 384), (5, 70001, 256), (18, 66000, 128), (40, 200003, 128), (3, 300000, 256)])
def test_head_logits_vocabularies_of_many_ranges(M, V, K, kind):
    """Vocabularies that workgroups of few rows take in ranges of 128 tokens, several of them: lists of all lengths, long ones beside empty ones."""
    q, qs, wq, ws = head_case(M, V, K, M + K)
    g = torch.Generator().manual_seed(V)
    bits = None
    if kind:
        bits = torch.rand((M, V), generator=g) < {"few": 2.0 / 128 / M, "some": 0.2 / M, "half": 0.5, "mixed": 0.02}[kind]
        if kind == "mixed":                                # dense ranges, and runs that nothing allows
            bits[:, 128 * 5:128 * 8] = True
            bits[0, V // 2:V // 2 + 300] = True
            bits[:, V - 2000:] = False
        bits[M - 1, V - 1] = True
    want, bound = head_want(q, qs, wq, ws)
    y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), packed(bits, True).cuda() if kind else None, dtype=torch.float32)
    check_head(y, want, bound, bits)


@gpu
@pytest.mark.parametrize("kind", [None, "few", "half", "mixed"])
@pytest.mark.parametrize("M,V,K", [(2, 16384, 256), (17, 16385, 384), (50, 16321, 640), (40, 16449, 256), (3, 28737, 4224), (30, 32768, 4096), (20, 30001, 4224), (1, 32769, 4096), (9, 33000, 4352), (18, 33000, 4096), (64, 28800, 4096)])
def test_head_logits_where_ranges_change(M, V, K, kind):
    """Vocabularies on both sides of where ranges of tokens get wider, rows of an odd number of blocks where they are taken in pairs; "mixed": some ranges are allowed whole."""
    q, qs, wq, ws = head_case(M, V, K, M + V)
    want, bound = head_want(q, qs, wq, ws)
    bits = None
    if kind:
        g = torch.Generator().manual_seed(K)
        bits = torch.rand((M, V), generator=g) < {"few": 0.002, "half": 0.5, "mixed": 0.0005}[kind]
        if kind == "mixed":
            for v in (0, 320, 8192, V - 200):
                bits[:, v:v + 200] = True
        bits[M // 2] = False
    mask = None if bits is None else packed(bits, padding=True).cuda()
    for dtype in (torch.float32, torch.bfloat16):
        check_head(zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), mask, dtype=dtype), want, bound, bits)


@gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(70, 70001, 128), (150, 70001, 384), (200, 66049, 256), (300, 66000, 128), (513, 40037, 256)])
def test_head_logits_more_tiles_than_compute_units(M, V, K, dtype, masked):
    """Batches whose workgroups take several tiles, one after the other: one block of columns and several, an odd number and an even one."""
    q, qs, wq, ws = head_case(M, V, K, M + K)
    bits = torch.rand((M, V), generator=torch.Generator().manual_seed(K)) < 0.5 if masked else None
    y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), packed(bits).cuda() if masked else None, dtype=DTYPES[dtype])
    want, bound = head_want(q, qs, wq, ws)
    check_head(y, want, bound, bits)


@gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(70, 65000, 128), (180, 60001, 256), (256, 50257, 384), (100, 40037, 256), (185, 49001, 128), (250, 33001, 384), (128, 32768, 256), (520, 20003, 128), (700, 24001, 256), (66, 191, 640), (66, 193, 128)])
def test_head_logits_tiles_of_all_sizes(M, V, K, dtype, masked):
    """Batches and vocabularies that tiles of 128, 192 and 256 tokens are chosen for, in one round of the compute units and in several."""
    q, qs, wq, ws = head_case(M, V, K, M + V)
    bits = torch.rand((M, V), generator=torch.Generator().manual_seed(K)) < 0.5 if masked else None
    y = zf.head_logits(q.cuda(), qs.cuda(), wq.cuda(), ws.cuda(), packed(bits, padding=True).cuda() if masked else None, dtype=DTYPES[dtype])
    want, bound = head_want(q, qs, wq, ws)
    check_head(y, want, bound, bits)


@gpu
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("M,V", [(2, 515), (70, 300), (260, 515)])
def test_head_logits_strides(M, V, masked):
    """Operands among others, a result at odd elements and distances that leaves what is around it alone, a result of the other type."""
    K = 256
    q, qs, wq, ws = head_case(M, V, K, 5)
    big_q = torch.zeros((M, K + 48), dtype=torch.uint8, device="cuda")
    big_w = torch.full((V, K + 128), 0x7F, dtype=torch.uint8, device="cuda")
    big_q[:, 16:16 + K] = q.view(torch.uint8).cuda()
    big_w[:, :K] = wq.view(torch.uint8).cuda()
    q_on, w_on = big_q.view(torch.float8_e4m3fn)[:, 16:16 + K], big_w.view(torch.float8_e4m3fn)[:, :K]
    bits = torch.rand((M, V), generator=torch.Generator().manual_seed(1)) < 0.5 if masked else None
    want, bound = head_want(q, qs, wq, ws)
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.full((M * (V + 2) + 1,), 7.0, dtype=dtype, device="cuda")
        out = buf[1:].view(M, V + 2)[:, :V]
        assert zf.head_logits(q_on, qs.cuda(), w_on, ws.cuda(), packed(bits).cuda() if masked else None, out=out) is out
        check_head(out, want, bound, bits)
        assert buf[0] == 7.0 and (buf[1:].view(M, V + 2)[:, V:] == 7.0).all()
    assert zf.head_logits(q_on[:0], qs.cuda()[:0], w_on, ws.cuda()).shape == (0, V)


@gpu
@pytest.mark.parametrize("M", [3, 70])
def test_head_logits_weight_of_more_than_two_gibibytes(M):
    """The last rows of the weight lie beyond 2^31 bytes, the last rows of the result beyond 2^31 elements."""
    V, K = 300001, 7424
    q, qs, wq, ws = head_case(M, 384, K, M)                # (its scales are the last three blocks of the weight's, whose last one is not full)
    first = V - 1 - (V - 1) % 128 - 256
    weight = torch.zeros((V, K), dtype=torch.float8_e4m3fn, device="cuda")
    weight[first:] = wq[:V - first].cuda()
    scales = torch.full((-(-V // 128), K // 128), math.nan, device="cuda")
    scales[-3:] = ws.cuda()
    bits = torch.zeros((M, V), dtype=torch.bool)
    bits[:, first:] = True
    out = None
    if M == 3:
        out = torch.empty(((M - 1) * (2 ** 30 + 24) + V,), dtype=torch.bfloat16, device="cuda").as_strided((M, V), (2 ** 30 + 24, 1))
    want, bound = head_want(q, qs, wq, ws)
    y = zf.head_logits(q.cuda(), qs.cuda(), weight, scales, packed(bits).cuda(), out=out)
    assert (y[:, :first] == -INF).all()
    n = V - first
    check_head(y[:, first:], want[:, :n], bound[:, :n])


# ---- log probabilities -------------------------------------------------------------------------------
def softmax_of(x, bits, temperature):
    """In 64 bits: logits with -inf where forbidden, log probabilities, probabilities, rows that have anything."""
    z = x.double()
    if bits is not None:
        z = z.masked_fill(~bits, -INF)
    some = (z > -INF).any(dim=1)
    lp = torch.where(some[:, None], torch.log_softmax(torch.where(some[:, None], z, 0.0) / temperature, dim=1), -INF)
    return z, lp, torch.where(some[:, None], lp.exp(), 0.0), some


def bounds_of(z, lp, p, some, temperature):
    """Bounds for a row's ln S, a log probability, the entropy.  e^z of a term is off by (3 |z| + 3) u (the difference, its product with log2 e / T, 2^x), a sum
    of 2^24 terms goes through at most 100 additions (64 in a lane, then trees over lanes, wavefronts and segments, with two products each): p-weighted
    |z| of a softmax is below ln S + 1, so ln S is off by less than (3 (ln S + 1) + 3 + 100) u, and a rounding of its own."""
    most = torch.where(some, z.amax(dim=1), 0.0)
    d = torch.where(z > -INF, (z - most[:, None]) / temperature, 0.0)
    ln_S = torch.where(some, -lp.amax(dim=1), 0.0)
    b_S = (3 * (ln_S + 1) + 103 + 2 * ln_S) * U
    b_lp = b_S[:, None] + 3 * U * (d.abs() + ln_S[:, None])
    mean, square = (p * d.abs()).sum(dim=1), (p * d * d).sum(dim=1)
    b_H = b_S * (1 + mean) + (3 * square + 110 * mean + 2 * (ln_S + mean)) * U
    return b_S, b_lp, b_H


def top_of(z, k):
    ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    ids = torch.where(z.gather(1, ids) > -INF, ids, -1)
    return torch.nn.functional.pad(ids, (0, k - ids.shape[1]), value=-1)


def near(got, want, bound, what):
    got, want = got.detach().cpu().double(), want.double()
    most = torch.finfo(torch.float32).max                  # a finite result beyond 32 bits is the largest number
    want = torch.where(torch.isfinite(want), want.clamp(-most, most), want)
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(9.0, 8.0, 7.0), want[~fine].nan_to_num(9.0, 8.0, 7.0)), what
    off = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    assert (off <= 0).all(), f"{what}: beyond its bound by {off.max():.3g}"


def check_logprobs(x, tokens, bits, temperature, top, layout="packed", padding=False, mask=None):
    """Everything of one call, and the gradient, against the definitions."""
    rows, V = x.shape
    z, lp, p, some = softmax_of(x, bits, temperature)
    _, b_lp, b_H = bounds_of(z, lp, p, some, temperature)
    if bits is not None and mask is None:
        mask = packed(bits, padding).cuda()
    x_on = rows_of(x, layout).requires_grad_()
    t2 = tokens.long().view(rows, -1)
    inside = (t2 >= 0) & (t2 < V)
    at = t2.clamp(0, V - 1)
    want_lp = torch.where(inside, lp.gather(1, at), torch.where(t2 < 0, 0.0, math.nan))
    want_H = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    for grad in (False, True):
        got = zf.token_logprobs(x_on if grad else x_on.detach(), tokens.cuda(), mask, temperature=temperature, entropy=True, top=top)
        assert got.logprobs.shape == tokens.shape
        near(got.logprobs.view(rows, -1), want_lp, torch.where(inside, b_lp.gather(1, at), 0.0), "logprobs")
        near(got.entropy, want_H, b_H, "entropy")
        if top:
            ids = top_of(z, top)
            assert torch.equal(got.top_ids.cpu().long(), ids), "top_ids"
            near(got.top_logprobs, torch.where(ids >= 0, lp.gather(1, ids.clamp(min=0)), -INF), b_lp.gather(1, ids.clamp(min=0)), "top_logprobs")
    # the gradient: given tokens (those with a log probability), alternatives and entropy together
    g = torch.Generator().manual_seed(V)
    g_lp, g_H, g_top = torch.randn((rows, t2.shape[1]), generator=g), torch.randn((rows,), generator=g), torch.randn((rows, top), generator=g)
    outs = [got.logprobs, got.entropy] + ([got.top_logprobs] if top else [])
    gs = [g_lp.view(tokens.shape).cuda(), g_H.cuda()] + ([g_top.cuda()] if top else [])
    grad, = torch.autograd.grad(outs, x_on, gs)
    assert grad.shape == x.shape and grad.dtype == x.dtype
    own = torch.zeros((rows, V), dtype=torch.float64)
    own_abs = torch.zeros((rows, V), dtype=torch.float64)
    G, G_abs = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    for ids, gg in ((t2, g_lp), (top_of(z, top), g_top)) if top else ((t2, g_lp),):
        c = ids.clamp(0, V - 1)
        gg = torch.where((ids >= 0) & (ids < V) & (lp.gather(1, c) > -INF), gg.double(), 0.0)
        own.scatter_add_(1, c, gg)
        own_abs.scatter_add_(1, c, gg.abs())
        G, G_abs = G + gg.sum(dim=1), G_abs + gg.abs().sum(dim=1)
    lp0 = torch.where(p > 0, lp, 0.0)
    want = (p * (-G[:, None] - g_H.double()[:, None] * (lp0 + want_H[:, None])) + own) / temperature
    n = t2.shape[1] + top
    size = p * (G_abs[:, None] + g_H.double().abs()[:, None] * (lp0.abs() + want_H[:, None].abs()))
    # p carries the bound of its logarithm (and 3 roundings for 2^x), the bracket those of lp, H and the sum of n gradients, the whole a few roundings more
    bound = size * (b_lp.nan_to_num(0.0, 0.0, 0.0) + 3 * U) + p * (g_H.double().abs()[:, None] * (b_lp.nan_to_num(0.0, 0.0, 0.0) + b_H[:, None]) + n * U * G_abs[:, None]) + 6 * U * size + (n + 6) * U * own_abs
    bound = bound / temperature
    near(grad, want, bound + half_step(x.dtype) * (want.abs() + bound) + 2.0 ** -120, "gradient")
    if bits is not None:
        assert (grad.cpu()[~bits] == 0).all()


def some_tokens(rows, V, n, bits, g, dtype):
    """Given tokens: any, allowed ones, a repeated one, padding, one beyond V."""
    t = torch.randint(V, (rows, n) if n else (rows,), generator=g)
    flat = t.view(rows, -1)
    if bits is not None:
        flat[:, 0] = torch.where(bits.any(dim=1), bits.float().argmax(dim=1), flat[:, 0])
    if flat.shape[1] > 3:
        flat[:, 1] = flat[:, 0]
        flat[:, 2] = -1
        flat[0, 3] = V + 5
    elif rows > 2:
        flat[1] = -7
    return t.to(dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,n,top,kind,layout,temperature", [
    (1, 1, 0, 1, None, "packed", 1.0), (3, 2, 4, 5, "half", "odd", 0.7), (5, 31, 1, 31, "half", "packed", 1.0), (4, 33, 6, 64, "few", "odd", 2.0), (130, 1000, 0, 3, "half", "padded", 1.0),
    (2, 4095, 5, 20, None, "odd", 1.0), (3, 4097, 0, 0, "few", "packed", 0.5), (2, 8193, 70, 64, "half", "packed", 1.3), (17, 16391, 0, 7, "few", "odd", 1.0), (2, 40037, 0, 20, "half", "odd", 1.0),
    (33, 32000, 2, 5, None, "packed", 1.0), (1, 152064, 0, 64, "few", "packed", 0.9), (1, 300007, 3, 20, None, "packed", 1.0)])
def test_token_logprobs(rows, V, n, top, kind, layout, temperature, dtype):
    g = torch.Generator().manual_seed(rows + V)
    x = (torch.randn((rows, V), generator=g) * 3).to(DTYPES[dtype])
    bits = None
    if kind:
        bits = torch.rand((rows, V), generator=g) < {"half": 0.5, "few": 0.004}[kind]
        bits[0, V // 2] = True
        if rows > 1:
            bits[rows - 1] = False                         # a row that allows nothing
    tokens = some_tokens(rows, V, n, bits, g, torch.int64 if rows % 2 else torch.int32)
    check_logprobs(x, tokens, bits, temperature, top, layout, padding=V % 2 == 1)


@gpu
@pytest.mark.parametrize("V", [37, 5000, 33000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprobs_values_that_meet_limits(dtype, V):
    """Rows by kind: all equal; all at the type's lowest; lowest but for one; -inf among others; all -inf; large ones; rising; falling; one far above all."""
    t = DTYPES[dtype]
    low = torch.finfo(t).min
    g = torch.Generator().manual_seed(V)
    x = torch.randn((10, V), generator=g)
    x[0] = 3.0
    x[1] = low
    x[2] = low
    x[2, V // 2] = 0.5
    x[3, ::2] = -INF
    x[4] = -INF
    x[5] *= 1e4
    x[6] = torch.arange(V) / V * 8
    x[7] = torch.arange(V, 0, -1) / V * 8
    x[8, V - 1] = 200.0
    x[9, 1:] = -INF
    x = x.to(t)
    tokens = torch.tensor([0, 1, V // 2, 1, 2, int(x[5].float().argmax()), V - 1, 0, V - 1, 0])
    check_logprobs(x, tokens, None, 1.0, 20)
    bits = torch.rand((10, V), generator=g) < 0.5
    bits[torch.arange(10), tokens] = True
    check_logprobs(x, tokens, bits, 0.8, 20, "odd")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprobs_forbidden_values_are_not_looked_at(dtype):
    """NaN, infinities and the lowest value behind a mask change nothing, in either direction; among the allowed ones they show."""
    V, rows = 9001, 6
    g = torch.Generator().manual_seed(3)
    x = torch.randn((rows, V), generator=g).to(DTYPES[dtype])
    bits = torch.rand((rows, V), generator=g) < 0.3
    bits[5] = False
    tokens = torch.where(bits.any(dim=1), bits.float().argmax(dim=1), 0)
    dirty = x.clone()
    for k, v in enumerate((math.nan, INF, -INF, torch.finfo(DTYPES[dtype]).min, torch.finfo(DTYPES[dtype]).max)):
        dirty[:, k::5] = torch.where(bits[:, k::5], x[:, k::5], torch.tensor(v, dtype=x.dtype))
    mask = packed(bits).cuda()
    res = []
    for v in (x, dirty):
        on = v.cuda().requires_grad_()
        got = zf.token_logprobs(on, tokens.cuda(), mask, entropy=True, top=9)
        grad, = torch.autograd.grad((got.logprobs.sum() + got.entropy.sum() * 0.3,), on)
        res.append([t.detach().cpu() for t in got] + [grad.cpu()])
    assert all(torch.equal(a, b) for a, b in zip(*res))
    # a NaN or +inf among the allowed: that row's numbers are NaN, the others stay
    for bad in (math.nan, INF):
        y = x.clone()
        y[2, tokens[2]] = bad
        got = zf.token_logprobs(y.cuda(), tokens.cuda(), mask, entropy=True, top=3)
        assert got.logprobs[2].isnan() and got.entropy[2].isnan()
        keep = torch.arange(rows) != 2
        assert torch.equal(got.logprobs.cpu()[keep], res[0][0][keep]) and torch.equal(got.entropy.cpu()[keep], res[0][1][keep])
        assert torch.equal(got.top_ids.cpu()[keep], res[0][2][keep][:, :3])
    alone = torch.full((1, 40), math.nan, dtype=x.dtype)
    got = zf.token_logprobs(alone.cuda(), torch.tensor([3]).cuda(), entropy=True, top=2)
    assert got.logprobs.isnan().all() and got.entropy.isnan().all() and (got.top_ids == -1).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 9001, 40037])
def test_gradient_of_forbidden_tokens_is_zero_whatever_comes_in(V, dtype):
    """Rows with a NaN, with +inf, with NaN alone, of logits far out, and ordinary ones with infinite and NaN gradients: what the mask forbids has gradient 0, given or not; the row
    beside them is what it is without them."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn((7, V), generator=g).to(DTYPES[dtype])
    bits = torch.rand((7, V), generator=g) < 0.4
    tokens = torch.stack([bits.float().argmax(dim=1), (~bits).float().argmax(dim=1)], dim=1)      # an allowed one and one that is not
    x[0, tokens[0, 0]] = math.nan
    x[1, tokens[1, 0]] = INF
    x[2] = torch.where(bits[2], math.nan, x[2].float()).to(x.dtype)
    x[3] = x[3] * 1e30
    g_lp, g_H = torch.randn((7, 2), generator=g), torch.randn(7, generator=g)
    g_lp[4, 0], g_H[5], g_lp[6, 1] = INF, math.nan, INF    # the last one's token is not allowed: nobody takes it
    grads = []
    for rows in (torch.arange(7), torch.tensor([6])):
        on = x[rows].cuda().requires_grad_()
        got = zf.token_logprobs(on, tokens[rows].cuda(), packed(bits[rows]).cuda(), entropy=True)
        grad, = torch.autograd.grad((got.logprobs, got.entropy), on, (g_lp[rows].cuda(), g_H[rows].cuda()))
        grads.append(grad.cpu())
    assert (grads[0][~bits] == 0).all()
    assert torch.equal(grads[0][6:], grads[1]) and torch.isfinite(grads[1]).all()
    assert grads[0][0][bits[0]].isnan().all() and grads[0][2][bits[2]].isnan().all() and torch.isfinite(grads[0][3]).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 9001, 40037])
@pytest.mark.parametrize("exponent", [-120, -20, 20, 120])
def test_token_logprobs_temperatures_far_from_one(exponent, V, dtype):
    g = torch.Generator().manual_seed(V)
    x = torch.randn((3, V), generator=g).to(DTYPES[dtype])
    bits = torch.rand((3, V), generator=g) < 0.5
    bits[:, 1] = True
    check_logprobs(x, torch.tensor([1, 1, -1]), bits, 2.0 ** exponent, 3)


def test_library_refuses_temperatures_whose_reciprocal_is_infinite():
    from paper_2506_01151_amd.binding import LogprobsArgs
    a = LogprobsArgs()
    a.logits, a.V, a.rows, a.row_stride = 4096, 10, 2, 10                     # (an address that nothing reads)
    for t, code in ((2.0 ** -149, zf.ZF_ERR_INVALID_ARG), (2.0 ** -126 - 2.0 ** -149, zf.ZF_ERR_INVALID_ARG), (2.0 ** -126, 0), (3e38, 0)):
        a.temperature = t
        assert min(zf.load_library().zf_token_logprobs_workspace(ctypes.byref(a)), 0) == code, t


@gpu
@pytest.mark.parametrize("top", [1, 20, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_with_many_equal_logits(dtype, top):
    """Few distinct values, both zeros, the largest ones all in one place or spread thin: by the lower id among equals."""
    V = 50001
    g = torch.Generator().manual_seed(top)
    x = torch.randint(-2, 3, (6, V), generator=g).float()
    x[1] = 0.0
    x[1, ::3] = -0.0
    x[2] = -5.0
    x[2, 20000:20100] = torch.arange(100.0)
    x[3] = -5.0
    x[3, ::777] = torch.arange(len(x[3, ::777])).float() % 40
    x[4] = -INF
    x[4, 17::9001] = 1.0
    x[5] = torch.arange(V).float()
    x = x.to(DTYPES[dtype])
    got = zf.token_logprobs(x.cuda(), top=top)
    assert got.logprobs is None and got.entropy is None
    assert torch.equal(got.top_ids.cpu().long(), top_of(x.double() + 0.0, top))


@gpu
@pytest.mark.parametrize("top", [1, 5, 64])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8193, 20000, 32768])
def test_alternatives_of_equal_logits_in_rows_of_one_workgroup(V, dtype, top):
    """Rows that are all one value, two values, the smaller first, or rise: more candidates than a list holds."""
    x = torch.zeros((5, V))
    x[1, V // 2:] = 1.0
    x[2] = torch.arange(V).float() / 256
    x[3] = -torch.arange(V).float()
    x[4, -1] = -0.0
    bits = torch.ones((5, V), dtype=torch.bool)
    bits[4, :-3] = False
    x = x.to(DTYPES[dtype])
    got = zf.token_logprobs(x.cuda(), mask=packed(bits).cuda(), top=top)
    assert torch.equal(got.top_ids.cpu().long(), top_of(x.double().masked_fill(~bits, -INF) + 0.0, top))


@gpu
@pytest.mark.parametrize("V,top", [(40037, 20), (9001, 3), (511, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprobs_rows_far_apart(V, top, dtype):
    g = torch.Generator().manual_seed(V + 1)
    x = torch.randn((4, V), generator=g).to(DTYPES[dtype])
    bits = torch.rand((4, V), generator=g) < 0.5
    check_logprobs(x, some_tokens(4, V, 5, bits, g, torch.int64), bits, 0.9, top, layout="far")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_rows_far_apart(dtype):
    x = torch.randn((4, 300), generator=torch.Generator().manual_seed(9)).to(DTYPES[dtype])
    for block_rows in (1, 128):
        q, scale = zf.quantize_blocks(rows_of(x, "far"), block_rows=block_rows)
        want_q, want_scale = quantized(x, block_rows)
        assert torch.equal(q.cpu().float(), want_q.float()) and torch.equal(scale.cpu(), want_scale)


@gpu
def test_calls_with_nothing_to_do():
    """No rows, no given tokens in a row, neither tokens nor anything else."""
    x = torch.randn((3, 50)).cuda()
    for grad in (False, True):
        on = x.clone().requires_grad_(grad)
        got = zf.token_logprobs(on, torch.empty((3, 0), dtype=torch.int64, device="cuda"), entropy=True)
        assert got.logprobs.shape == (3, 0) and got.entropy.shape == (3,)
        if grad:
            (got.entropy.sum() + got.logprobs.sum()).backward()
            want = zf.token_logprobs(on.detach(), entropy=True).entropy
            assert torch.equal(got.entropy.detach(), want) and on.grad.shape == on.shape
        got = zf.token_logprobs(on[:0], torch.empty(0, dtype=torch.int64, device="cuda"), entropy=True, top=2)
        assert got.logprobs.shape == got.entropy.shape == (0,) and got.top_ids.shape == got.top_logprobs.shape == (0, 2)
        assert zf.token_logprobs(on) == (None, None, None, None)
    q, scale = zf.quantize_blocks(x[:0])
    assert q.shape == (0, 128) and scale.shape == (0, 1)


@gpu
def test_gradient_against_differences():
    """The forward call's own differences in 32 bits: a step of h = 2^-5 leaves h^2 / 6 times the third derivative (each factor's share of it is below 1, times what the
    gradients add up to), and twice a value's error over 2 h."""
    rows, V, h, T = 4, 45, 2.0 ** -5, 0.8
    g = torch.Generator().manual_seed(11)
    x = torch.randn((rows, V), generator=g)
    bits = torch.rand((rows, V), generator=g) < 0.8
    tokens = torch.stack([bits[r].nonzero()[:3, 0] for r in range(rows)])
    mask = packed(bits).cuda()
    w_lp, w_H, w_top = torch.randn((rows, 3), generator=g), torch.randn((rows,), generator=g), torch.randn((rows, 2), generator=g)

    def loss(v, with_top):
        got = zf.token_logprobs(v, tokens.cuda(), mask, temperature=T, entropy=True, top=2)
        s = (got.logprobs * w_lp.cuda()).sum(dim=1) + got.entropy * w_H.cuda()
        return s + (got.top_logprobs * w_top.cuda()).sum(dim=1) if with_top else s

    for with_top in (False, True):
        if with_top:                                       # the two largest stay the two largest under a step
            x[:, 7], x[:, 9], bits[:, 7], bits[:, 9] = 4.0, 5.0, True, True
            mask = packed(bits).cuda()
        on = x.cuda().requires_grad_()
        grad, = torch.autograd.grad(loss(on, with_top).sum(), on)
        steps = torch.eye(V).cuda() * h
        size = w_lp.abs().sum(dim=1) + (w_top.abs().sum(dim=1) if with_top else 0) + 8 * w_H.abs()       # |ln p| < 8 at these logits
        for v in range(V):
            with torch.no_grad():
                d = (loss(on + steps[v], with_top) - loss(on - steps[v], with_top)).cpu().double() / (2 * h)
            assert ((grad[:, v].cpu().double() - d).abs() <= size.double() * ((h / T) ** 2 / 6 / T * 8 + 150 * U / h)).all()


@gpu
def test_operators_on_streams_and_in_graphs():
    """On a stream of its own behind other work, and captured: every replay gives the eager results of what the inputs then hold; eager calls in between."""
    M, V, K = 20, 5003, 512
    q, qs, wq, ws = (t.cuda() for t in head_case(M, V, K, 2))
    hidden = (q.float() * qs.repeat_interleave(128, dim=1)).to(torch.bfloat16)
    bits = torch.rand((M, V), generator=torch.Generator().manual_seed(4)) < 0.2
    mask, tokens, g = packed(bits).cuda(), torch.randint(V, (M,)).cuda(), torch.randn(M).cuda()

    def chain(h):
        a, b = zf.quantize_blocks(h)
        y = zf.head_logits(a, b, wq, ws, mask)
        y.requires_grad_()
        got = zf.token_logprobs(y, tokens, mask, entropy=True, top=6)
        grad, = torch.autograd.grad((got.logprobs, got.entropy), y, (g, g))
        return [t.detach() for t in (a.view(torch.uint8), b, y, *got, grad)]

    want = [t.clone() for t in chain(hidden)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain(hidden)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    at = hidden.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs = chain(at)
    for r in range(4):
        fresh = hidden * (r + 1) / 2
        at.copy_(fresh)
        graph.replay()
        eager = chain(fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)), r


@gpu
def test_gradient_may_overwrite_the_logits():
    """The C call with d_grad = the logits: the same bits as into memory of its own."""
    from paper_2506_01151_amd import operators as ops
    rows, V = 3, 20011
    x = torch.randn((rows, V), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).cuda()
    tokens, g = torch.tensor([1, 19999, 7]).cuda(), torch.randn(rows).cuda()
    lp, H, ids, top_lp, stats = ops._forward(x, tokens, None, 1.0, True, 0, True)
    want = ops._backward(x, tokens, None, lp, H, None, None, stats, 1.0, g, g, None)
    a = ops._logprobs_args(x, tokens, None, 1.0, 0)
    a.logprobs, a.entropy, a.stats = lp.data_ptr(), H.data_ptr(), stats.data_ptr()
    assert zf.load_library().zf_token_logprobs_backward(ctypes.byref(a), g.data_ptr(), g.data_ptr(), None, x.data_ptr(), V, 0, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(x, want)


@gpu
def test_example_draws_under_the_grammar_and_learns():
    """examples/decode_and_train.py: what it draws parses, what it reports is what the definitions say of the logits' own product, the gradient is that of its loss."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_and_train.py")
    spec = importlib.util.spec_from_file_location("decode_and_train", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    from workloads import configs
    cfg = configs.CONFIGS[1]
    engine = zf.Engine(cfg.grammar(), cfg.vocab())
    model = example.Model(engine.V, 256, "cuda:0")
    steps = example.decode(engine, model, 3, 12)
    assert len(steps) == 12
    for r in range(3):
        state = engine.new_state()
        for _, mask, tokens, got in steps:
            bits = np.unpackbits(mask[r].cpu().numpy().view(np.uint8), bitorder="little")[:engine.V]
            token = int(tokens[r])
            if token < 0:
                assert not bits.any() and float(got.logprobs[r]) == 0.0
                state.reset()
                continue
            assert bits[token]
            state.advance(token)                           # (raises where the grammar does not go on so)
            assert 0 <= float(got.entropy[r]) <= math.log(bits.sum()) + 1e-3 and float(got.logprobs[r]) <= 0
            best = [i for i in got.top_ids[r].tolist() if i >= 0]
            assert len(best) == min(5, int(bits.sum())) and all(bits[i] for i in best)
    served = torch.cat([s[3].logprobs for s in steps])
    advantage = torch.linspace(-1, 1, len(served)).cuda()
    loss, g_hidden, g_head, learnt = example.train_step(model, steps, advantage)
    # the loss in 64 bits from the same logits, and its gradient for them by torch
    hidden = torch.cat([s[0] for s in steps]).to(torch.bfloat16)
    head = model.head.to(torch.bfloat16)
    logits = (hidden @ head.t()).cpu().double().requires_grad_()
    mask, tokens = torch.cat([s[1] for s in steps]).cpu(), torch.cat([s[2] for s in steps]).cpu().long()
    bits = torch.from_numpy(np.unpackbits(mask.numpy().view(np.uint8), axis=1, bitorder="little")[:, :engine.V].astype(bool))
    drawn = tokens >= 0
    z = torch.where(drawn[:, None], logits.masked_fill(~bits, -INF), 0.0) / 0.8
    lp = torch.log_softmax(z, dim=1)
    own = torch.where(drawn, lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = -(lp.exp() * lp.masked_fill(lp == -INF, 0.0)).sum(dim=1) * drawn
    want = -(advantage.cpu().double() * own + 0.01 * entropy).sum() / drawn.sum()
    grad, = torch.autograd.grad(want, logits)
    assert (learnt.cpu().double() - own.detach()).abs().max() < 1e-4 and abs(float(loss) - float(want.detach())) < 1e-4
    # the logits' gradient is in bf16, and so are its two products with the model: three roundings of half a step relative to the terms
    for got, by_hand, terms in ((g_hidden, grad @ head.cpu().double(), grad.abs() @ head.cpu().double().abs()), (g_head, grad.t() @ hidden.cpu().double(), grad.abs().t() @ hidden.cpu().double().abs())):
        assert ((got.cpu().double() - by_hand.detach()).abs() <= 3 * half_step(torch.bfloat16) * terms + 1e-6).all()


# ---- refusals ----------------------------------------------------------------------------------------
def refused(call, says=""):
    with pytest.raises(zf.ZfError) as e:
        call()
    assert e.value.code == zf.ZF_ERR_INVALID_ARG and says in str(e.value), str(e.value)


def test_library_refuses_before_it_touches_a_device():
    """The C calls with arguments that do not fit: ZF_ERR_INVALID_ARG and a text, with no device there at all; no rows: ZF_OK."""
    from paper_2506_01151_amd.binding import LogprobsArgs
    L = zf.load_library()
    one = 4096                                             # an address that nothing reads
    ok = dict(x=one, dtype=0, rows=2, cols=10, stride=10, br=1, q=one, s=one)

    def quant(**kw):
        a = {**ok, **kw}
        return L.zf_quantize_blocks(a["x"], a["dtype"], a["rows"], a["cols"], a["stride"], a["br"], a["q"], a["s"], 0, None)

    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 24) + 1), dict(stride=9), dict(br=2), dict(br=0), dict(x=one + 2), dict(q=one + 8), dict(x=one + 1, dtype=1)):
        assert quant(**bad) == zf.ZF_ERR_INVALID_ARG and L.zf_last_error(), bad
    assert quant(rows=0, x=None, q=None, s=None) == 0
    ok_h = dict(x=one, xst=256, xs=one, w=one, wst=256, ws=one, M=2, V=10, K=256, mask=None, y=one, dtype=1, yst=10)

    def head(**kw):
        a = {**ok_h, **kw}
        return L.zf_head_logits(a["x"], a["xst"], a["xs"], a["w"], a["wst"], a["ws"], a["M"], a["V"], a["K"], a["mask"], a["y"], a["dtype"], a["yst"], 0, None)

    for bad in (dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(y=None), dict(M=-1), dict(M=(1 << 20) + 1), dict(V=0), dict(V=(1 << 24) + 1, yst=1 << 25), dict(K=0), dict(K=100), dict(K=384), dict(xst=264),
                dict(wst=257), dict(wst=128), dict(yst=9), dict(dtype=3), dict(x=one + 4), dict(w=one + 8), dict(y=one + 1), dict(y=one + 2, dtype=0)):
        assert head(**bad) == zf.ZF_ERR_INVALID_ARG and L.zf_last_error(), bad
    assert head(M=0, x=None, xs=None, y=None) == 0
    ok_l = dict(logits=one, dtype=0, V=10, rows=2, row_stride=10, mask=None, tokens=one, token_bytes=8, n_tokens=1, top=1, temperature=1.0, logprobs=one, entropy=one, top_ids=one, top_logprobs=one, stats=one)

    def args(**kw):
        a = LogprobsArgs()
        for k, v in {**ok_l, **kw}.items():
            setattr(a, k, v)
        return ctypes.byref(a)

    def logprobs(**kw):
        assert L.zf_token_logprobs_workspace(args(**kw)) < 0
        back = L.zf_token_logprobs_backward(args(**kw), one, one, one, one, 10, 0, None)
        assert back == zf.ZF_ERR_INVALID_ARG
        return L.zf_token_logprobs(args(**kw), one, 1 << 40, 0, None)

    for bad in (dict(logits=None), dict(dtype=2), dict(V=0), dict(V=(1 << 24) + 1, row_stride=1 << 25), dict(rows=-1), dict(rows=1 << 31), dict(rows=1 << 30), dict(row_stride=9), dict(row_stride=0), dict(tokens=None), dict(token_bytes=2), dict(n_tokens=-1),
                dict(n_tokens=1025), dict(top=-1), dict(top=65), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=INF), dict(logprobs=None), dict(top_ids=None), dict(top_logprobs=None),
                dict(logits=one + 2)):
        assert logprobs(**bad) == zf.ZF_ERR_INVALID_ARG and L.zf_last_error(), bad
    wide = dict(V=100000, row_stride=100000)               # rows that one workgroup does not take
    need = L.zf_token_logprobs_workspace(args(**wide))
    assert need > 0
    assert L.zf_token_logprobs(args(**wide), one, need - 1, 0, None) == zf.ZF_ERR_INVALID_ARG
    assert L.zf_token_logprobs(args(**wide), None, need, 0, None) == zf.ZF_ERR_INVALID_ARG
    assert L.zf_token_logprobs(args(**wide), one + 8, need, 0, None) == zf.ZF_ERR_INVALID_ARG
    assert L.zf_token_logprobs(None, one, 1 << 40, 0, None) == zf.ZF_ERR_INVALID_ARG and L.zf_token_logprobs_workspace(None) == zf.ZF_ERR_INVALID_ARG
    assert L.zf_token_logprobs(args(rows=0, logits=None), None, 0, 0, None) == 0 and L.zf_token_logprobs_workspace(args(rows=0)) == 0
    for kw, g in ((dict(stats=None), (one, one, one, one, 10)), ({}, (one, one, one, None, 10)), ({}, (one, one, one, one, 9)), ({}, (one, one, one, one + 2, 10)), (dict(entropy=None), (one, one, one, one, 10))):
        assert L.zf_token_logprobs_backward(args(**kw), *g, 0, None) == zf.ZF_ERR_INVALID_ARG, (kw, g)


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    x = torch.zeros((2, 256))
    refused(lambda: zf.quantize_blocks(x), "on the GPU")
    refused(lambda: zf.quantize_blocks(3), "on the GPU")
    refused(lambda: zf.head_logits(x.to(torch.float8_e4m3fn), x, x, x), "on the GPU")
    refused(lambda: zf.token_logprobs(x), "on the GPU")
    refused(lambda: zf.token_logprobs(x.to_sparse()), "on the GPU")
    assert "token_logprobs" in dir(zf)
    with pytest.raises(AttributeError):
        zf.token_logprob


@gpu
def test_binding_refuses_what_does_not_fit():
    x = torch.zeros((2, 256), device="cuda")
    q, s = zf.quantize_blocks(x)
    w, ws = zf.quantize_blocks(torch.zeros((300, 256), device="cuda"), block_rows=128)
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    m = torch.zeros((2, 8), dtype=torch.int32, device="cuda")
    for call in (lambda: zf.quantize_blocks(x.half()), lambda: zf.quantize_blocks(x[0]), lambda: zf.quantize_blocks(x.t()), lambda: zf.quantize_blocks(x, block_rows=64), lambda: zf.quantize_blocks(x[:, :0]),
                 lambda: zf.quantize_blocks(x[:1].expand(3, 256)),
                 lambda: zf.head_logits(q, s[:1], w, ws), lambda: zf.head_logits(q, s, w, ws[:2]), lambda: zf.head_logits(q, s, w[:, :128], ws), lambda: zf.head_logits(q, s.half(), w, ws),
                 lambda: zf.head_logits(q, s, w, ws, m), lambda: zf.head_logits(q, s, w, ws, dtype=torch.float16), lambda: zf.head_logits(q, s, w, ws, out=x), lambda: zf.head_logits(q[:, :64], s, w[:, :64], ws),
                 lambda: zf.head_logits(q.view(torch.uint8), s, w, ws), lambda: zf.head_logits(q, s, w, ws, out=torch.zeros((300, 2), device="cuda").t()), lambda: zf.head_logits(q, s.cpu(), w, ws), lambda: zf.head_logits(q[:, 8:136], s[:, :1].contiguous(), w[:, :128], ws[:, :1].contiguous()),
                 lambda: zf.token_logprobs(x.half(), t), lambda: zf.token_logprobs(x, t[:1]), lambda: zf.token_logprobs(x, t.float()), lambda: zf.token_logprobs(x, t.cpu()), lambda: zf.token_logprobs(x, t, m[:, :7]),
                 lambda: zf.token_logprobs(x, t, m.long()), lambda: zf.token_logprobs(x, t, m[:1]), lambda: zf.token_logprobs(x, t, torch.zeros((2, 16), dtype=torch.int32, device="cuda")[:, ::2]),
                 lambda: zf.token_logprobs(x, t, top=65), lambda: zf.token_logprobs(x, t, top=-1), lambda: zf.token_logprobs(x, t, top=1.0), lambda: zf.token_logprobs(x, t, temperature=0.0), lambda: zf.token_logprobs(x, t, temperature=math.nan),
                 lambda: zf.token_logprobs(x[:, :0], t), lambda: zf.token_logprobs(x.t()), lambda: zf.token_logprobs(x[:1].expand(2, 256), t), lambda: zf.token_logprobs(x, torch.zeros((2, 1025), dtype=torch.int64, device="cuda")),
                 lambda: zf.token_logprobs(x, torch.zeros((2, 4), dtype=torch.int64, device="cuda")[:, ::2])):
        refused(call)
    got = zf.token_logprobs(x[:0], t[:0], m[:0], entropy=True, top=2)
    assert got.logprobs.shape == (0,) and got.top_ids.shape == (0, 2) and got.entropy.shape == (0,)
    y = x.clone().requires_grad_()
    lp = zf.token_logprobs(y, t, top=2)
    assert not lp.top_ids.requires_grad and lp.entropy is None
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(lp.logprobs.sum(), y, create_graph=True)[0].sum(), y)
