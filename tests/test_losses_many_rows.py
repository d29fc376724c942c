"""The losses on logits (distill_loss, policy_loss, preference_loss) in calls whose workgroups take several rows in turn, whose logits and gradients pass the last-level cache by, and the ways of
preference_loss that other tests leave out.

Two comparisons.  A row's results and gradient do not depend on the rows around it where as many threads take a row: a call of all rows has the same bits as calls of parts that are so small that each
workgroup takes one row, and whose logits and gradient fit the cache.  And a sample of the rows -- the first and last, those on either side of a workgroup's step from row to row, and of each kind of row -- is compared with the
definition in 64 bits, with the tolerances of tests/test_losses.py."""
import math

import pytest
import torch

import paper_2506_01151_amd as zf
from tests.test_losses import IDS, INF, PREFERENCE, U, Rows, close, distill_want, loss_bound, policy_want, preference_want
from tests.test_operators import DTYPES

gpu = pytest.mark.gpu
T = 0.9
KINDS = 37                                         # a row's kind is its number modulo this
NAN, FAR, PADDING, EMPTY, SINGLE, NOT_ALLOWED = (5,), (11,), (17, 18, 19), (23,), (29,), (7, 20)


class Batch:
    """Rows of all kinds on the GPU: logits and mask, allowed, tokens."""

    def __init__(self, dtype, rows, V, masked, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.V, self.dtype = rows, V, dtype
        self.x = torch.randn((rows, V), generator=self.g, device="cuda").mul_(3.0)
        self.kind = torch.arange(rows, device="cuda") % KINDS
        self.of(FAR, lambda at: self.x.index_add_(0, at, torch.full((len(at), V), 8000.0, device="cuda")))
        self.x = self.x.to(DTYPES[dtype])
        self.mask, self.allowed = None, torch.ones((rows, V), dtype=torch.bool, device="cuda")
        if masked:
            share = torch.rand((rows, 1), generator=self.g, device="cuda") ** 2
            self.allowed = torch.rand((rows, V), generator=self.g, device="cuda") < share
            self.allowed[:, V // 3] = True
            self.of(EMPTY + SINGLE, lambda at: self.allowed.index_fill_(0, at, False))
            self.allowed[self.where(SINGLE), V - 1] = True
        self.x[self.where(NAN), V // 3] = math.nan
        if masked:
            W = (V + 31) // 32
            bits = torch.ones((rows, W * 32), dtype=torch.bool, device="cuda")      # those beyond V are set
            bits[:, :V] = self.allowed
            words = (bits.view(rows, W, 32).to(torch.int64) << torch.arange(32, device="cuda")).sum(-1)
            self.mask = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
        z = torch.where(self.allowed, self.x.float().nan_to_num(), -INF)
        self.some = (z > -INF).any(dim=1)
        self.lse = torch.where(self.some, torch.logsumexp(z / T, dim=1), 0.0)
        self.tokens = torch.where(torch.rand((rows, V), generator=self.g, device="cuda") < 0.1, z, -INF).argmax(dim=1)
        self.tokens[self.where(SINGLE)] = V - 1
        self.tokens[self.where(NOT_ALLOWED)] = torch.randint(V, (len(self.where(NOT_ALLOWED)),), generator=self.g, device="cuda")
        self.tokens[self.where(PADDING)] = -1
        self.z = z

    def where(self, kinds):
        return torch.isin(self.kind, torch.tensor(kinds, device="cuda")).nonzero()[:, 0]

    def of(self, kinds, do):
        at = self.where(kinds)
        if len(at):
            do(at)

    def random(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def sample(self, places):
        """Rows to look at in 64 bits, where a workgroup's second and third may begin and of all kinds, and these as tests/test_losses.py has them."""
        n = self.rows
        some = [0, n - 1] + [k * places + d for k in range(1, n // places + 1) for d in (0, 1, -1)] + [places // 2 + k for k in range(KINDS)]
        some = [i for i in dict.fromkeys(some) if 0 <= i < n and i % KINDS not in NAN]
        at = torch.tensor(sorted(some[:max(12, 2_000_000 // self.V)]), device="cuda")
        r = Rows.__new__(Rows)
        r.n, r.V, r.T, r.x, r.bits = len(at), self.V, T, self.x[at].detach().cpu(), self.allowed[at].cpu()
        r.update()
        return at, r

    def normal_to(self, t, V):
        """Log probabilities of tokens, about."""
        return torch.where(t >= 0, self.z.gather(1, t.clamp(min=0)[:, None])[:, 0] / T - self.lse, 0.0).nan_to_num(neginf=-9.0)


def same_bits(a, b, what):
    assert a.dtype == b.dtype and a.shape == b.shape, what
    kind = {torch.float32: torch.int32, torch.bfloat16: torch.int16}[a.dtype]
    nan = torch.isnan(a)
    assert torch.equal(nan, torch.isnan(b)), f"{what}: NaN elsewhere"
    assert torch.equal(torch.where(nan, 0, a.view(kind)), torch.where(nan, 0, b.view(kind))), what


# rows, V, and how many workgroups there are at most for rows of that length (threads a row: 64, 192, 256, 960, 1,024 ...); 16 or 20 pieces of 16 bytes a thread from the fourth on
MANY = [("f32", 9000, 261, 4096), ("bf16", 9000, 261, 4096), ("bf16", 2700, 9000, 1280), ("bf16", 2100, 32000, 1024), ("f32", 600, 60001, 256), ("bf16", 1100, 130000, 256), ("bf16", 600, 131071, 256),
        ("f32", 600, 80000, 256), ("bf16", 600, 152065, 256), ("bf16", 900, 152064, 256)]
# from memory: no mask, one a compute unit; rows shorter than 16 bytes; under masks as many as there may be
FROM_MEMORY = [("f32", 600, 90001, 256), ("bf16", 300, 170001, 256), ("f32", 3000, 3, 256), ("f32", 66000, 3, 40000)]


def compare(batch, call, beside, slots, want, names):
    """`call(logits, mask, rows)` for a slice of rows; want(r, at, got): the comparison with 64 bits."""
    x = batch.x.requires_grad_()
    whole = call(x, batch.mask, slice(None))
    weight = beside["weight"]
    total = (weight.double() * whole.losses.double()).sum()
    assert torch.isnan(whole.loss) == torch.isnan(total)          # the rows that are not a number
    grads = [torch.autograd.grad(whole.loss, x, retain_graph=True)[0], torch.autograd.grad(whole.loss * 2.0, x)[0]]
    with torch.no_grad():
        alone = call(x, batch.mask, slice(None))
        for n in names:
            same_bits(getattr(alone, n), getattr(whole, n), f"{n} without a gradient")
    nan = batch.where(NAN)
    nan = nan[torch.isnan(whole.losses[nan])]
    assert len(nan) or batch.rows < KINDS
    step = -(-batch.rows // -(-batch.rows // slots))           # parts of equal size: a row of a much smaller call is taken by twice as many threads, which sum in another order
    parts = [slice(a, min(a + step, batch.rows)) for a in range(0, batch.rows, step)]
    assert len(parts) > 1
    for part in parts:
        leaf = batch.x[part].detach().requires_grad_()
        got = call(leaf, batch.mask[part] if batch.mask is not None else None, part)
        for n in names:
            same_bits(getattr(got, n), getattr(whole, n)[part], n)
        for grad, factor in zip(grads, (1.0, 2.0)):
            g, = torch.autograd.grad(got.loss * factor, leaf, retain_graph=True)
            same_bits(g, grad[part], f"gradient for {factor}")
    at, r = batch.sample(slots)
    want(r, at, whole, grads[0][at], grads[1][at])


@gpu
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,rows,V,slots", MANY + FROM_MEMORY)
def test_policy_of_many_rows(dtype, rows, V, slots, masked, entropy):
    b = Batch(dtype, rows, V, masked, rows + V)
    old = b.normal_to(b.tokens, V) + 0.6 * b.random(rows) - 0.3
    beside = {"old": old, "adv": b.random(rows) - 0.5, "ref": old + 0.2, "weight": b.random(rows)}
    e, kl = (0.01, 0.05) if entropy else (None, 0.0)

    def call(x, mask, part):
        return zf.policy_loss(x, b.tokens[part], beside["old"][part], beside["adv"][part], mask, ref_logprobs=beside["ref"][part] if entropy else None, temperature=T, clip=(0.2, 0.3), kl_weight=kl,
                              entropy_weight=e, weight=beside["weight"][part])

    def want(r, at, got, once, twice):
        t, old, adv, ref, weight = (y[at].cpu() for y in (b.tokens, beside["old"], beside["adv"], beside["ref"], beside["weight"]))
        losses, bound, lp, H, H_off, grad, off = policy_want(r, t, old, adv, ref if entropy else None, (0.2, 0.3), kl, e, weight)
        close(got.losses[at], losses, bound, "losses")
        close(got.logprobs[at], lp, torch.where(lp > -INF, r.slack[:, 0], 0.0), "log probabilities")
        if entropy:
            close(got.entropy[at], H, H_off, "entropy")
        close(once, grad, off, "gradient", DTYPES[dtype])
        close(twice, 2 * grad, 2 * off, "gradient made again", DTYPES[dtype])

    compare(b, call, beside, slots, want, ["losses", "logprobs"] + (["entropy"] if entropy else []))


@gpu
@pytest.mark.parametrize("rest,K", [(False, 3), (True, 70)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,rows,V,slots", MANY + FROM_MEMORY)
def test_distill_of_many_rows(dtype, rows, V, slots, masked, rest, K):
    b = Batch(dtype, rows, V, masked, rows + V + 1)
    n = min(K, V)
    best, at = torch.topk(b.z + torch.rand((rows, 1), generator=b.g, device="cuda"), n, dim=1)
    ids = torch.full((rows, K), -1, device="cuda")
    ids[:, :n] = torch.where(best > -INF, at, -1)
    values = torch.full((rows, K), -INF, device="cuda")
    values[:, :n] = (best / T - b.lse[:, None]).clamp(max=0.0) - 0.2 * b.random(rows, n) - 1.5 if rest else 0.8 * best
    other = torch.randint(V, (rows,), generator=b.g, device="cuda")
    kind = torch.arange(rows, device="cuda") % 5
    ids[:, K // 2] = torch.where(kind == 2, ids[:, 0], torch.where(kind == 3, other, ids[:, K // 2]))       # listed twice; whatever it is
    values[:, K // 2] = torch.where(kind == 3, -4.0, values[:, K // 2])
    values[:, K - 1] = torch.where(kind == 4, -INF, values[:, K - 1])
    ids[b.where(PADDING)] = -1
    ids = ids.to(IDS[4 if masked else 8])
    beside = {"weight": b.random(rows) - 0.2}

    def call(x, mask, part):
        return zf.distill_loss(x, ids[part], values[part], mask, temperature=T, rest=rest, weight=beside["weight"][part])

    def want(r, at, got, once, twice):
        losses, bound, grad, off = distill_want(r, ids[at].cpu(), values[at].cpu(), rest, beside["weight"][at].cpu(), dtype)
        close(got.losses[at], losses, bound, "losses")
        close(once, grad, off, "gradient", DTYPES[dtype])
        close(twice, 2 * grad, 2 * off, "gradient made again", DTYPES[dtype])

    compare(b, call, beside, slots, want, ["losses"])


# ---- preferences --------------------------------------------------------------------------------------
def preferences(r, lengths, before, dtype, average, s, beta, layout, ids=8, weighed=False, masked=False):
    """Against 64 bits: all rows."""
    P, rows = len(lengths) // 2, r.n
    t = r.tokens(ids, padding=0.3)
    lp, counts = r.at(t)
    t = torch.where(counts, t, -1).to(t.dtype)
    lp, counts = r.at(t)
    ref = (lp + 0.3 * torch.randn((rows,), generator=r.g)).float()
    weight = torch.rand((P,), generator=r.g) + 0.1 if weighed else None
    offsets = torch.tensor([before] + [before + sum(lengths[:i + 1]) for i in range(len(lengths))]).to(IDS[ids])
    losses, bound, chosen, rejected, D_off, grad, off = preference_want(r, t, offsets, ref, beta, s, average, weight)
    x, m = r.on_gpu(layout)
    assert (m is not None) == masked
    x.requires_grad_()
    got = zf.preference_loss(x, t.cuda(), offsets.cuda(), ref.cuda(), m, beta=beta, label_smoothing=s, average=average, temperature=r.T, weight=weight.cuda() if weighed else None)
    close(got.chosen, chosen, D_off[0::2], "chosen")
    close(got.rejected, rejected, D_off[1::2], "rejected")
    close(got.losses, losses, bound, "losses")
    close(got.loss, *loss_bound(weight, losses, bound), "loss")
    g, = torch.autograd.grad(got.loss, x)
    close(g, grad, off, "gradient", x.dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("average,s,beta", [(False, 0.0, 0.1), (True, 0.1, 2.5), (False, 1.0, -0.3)])
@pytest.mark.parametrize("case", range(len(PREFERENCE)))
def test_preference_without_a_mask(case, average, s, beta, dtype):
    lengths, before, behind, V = PREFERENCE[case]
    rows = before + sum(lengths) + behind
    r = Rows(rows, V, dtype, "none", (1.0, 0.7, 1.3)[case % 3], 1000 + case)
    preferences(r, lengths, before, dtype, average, s, beta, ("packed", "padded", "odd")[case // 2 % 3], ids=(4, 8)[case % 2], weighed=case % 3 == 1)


@gpu
@pytest.mark.parametrize("dtype,V", [("bf16", 8200), ("f32", 4101)])
@pytest.mark.parametrize("masked", [False, True])
def test_preference_of_many_rows(dtype, V, masked):
    """2,048 rows and more of more than 16 KB are taken by workgroups of another size."""
    r = Rows(2100, V, dtype, "share" if masked else "none", 1.0, V)
    if masked:
        r.bits[:, V // 2] = True
        r.update()
    preferences(r, [130] * 15 + [1], 3, dtype, True, 0.1, 0.5, "packed", masked=masked)


@gpu
@pytest.mark.parametrize("masked", [False, True])
def test_preference_that_passes_the_cache_by(masked):
    """1,100 rows, 286 MB: the same bits as its pairs in parts that fit the cache; a sample of the gradient against 64 bits."""
    rows, V, pairs = 1100, 130000, 10
    b = Batch("bf16", rows, V, masked, 77)
    b.x[b.where(NAN), V // 3] = 0.5
    t = b.tokens.clone()
    t[b.where(EMPTY)] = -1
    t[~b.allowed.gather(1, t.clamp(min=0)[:, None])[:, 0]] = -1
    length = torch.arange(2 * pairs) % 7 + 50
    offsets = torch.cat([torch.tensor([4]), 4 + torch.cumsum(length, 0)])
    ref = b.normal_to(t, V) + 0.3 * b.random(rows)
    x = b.x.requires_grad_()
    got = zf.preference_loss(x, t, offsets.cuda(), ref, b.mask, temperature=T)
    grad, = torch.autograd.grad(got.loss, x)
    assert torch.isfinite(got.losses).all() and torch.isfinite(grad).all()
    for i in range(0, pairs, 2):
        lo, hi = int(offsets[2 * i]), int(offsets[2 * i + 4])
        leaf = b.x[lo:hi].detach().requires_grad_()
        part = zf.preference_loss(leaf, t[lo:hi], (offsets[2 * i:2 * i + 5] - lo).cuda(), ref[lo:hi], b.mask[lo:hi] if masked else None, temperature=T)
        for n in ("losses", "chosen", "rejected"):
            same_bits(getattr(part, n), getattr(got, n)[i:i + 2], n)
        same_bits(torch.autograd.grad(part.loss, leaf)[0], grad[lo:hi], "gradient")
    assert not grad[:4].any() and not grad[int(offsets[-1]):].any()
    at = torch.tensor([4, int(offsets[1]), int(offsets[5]) - 1, int(offsets[-1]) - 1] + list(range(300, 300 + KINDS, 3)))
    r = Rows.__new__(Rows)
    r.n, r.V, r.T, r.x, r.bits = len(at), V, T, b.x[at].detach().cpu(), b.allowed[at].cpu()
    r.update()
    # d loss / d x = c (onehot - p) on a row, c from the call's own log ratios: beta sigma(-h), off by the 32 bits that these are rounded to
    h = got.chosen.double() - got.rejected.double()
    c = -0.1 * torch.sigmoid(-h).cpu() / T
    tokens = t[at].cpu()
    s = torch.searchsorted(offsets[1:], at, right=True)
    f = torch.where(tokens >= 0, c[s // 2] * (1 - 2 * (s % 2)), 0.0)
    f_off = f.abs() * 2 * U * (1 + (got.chosen.abs() + got.rejected.abs()).double().cpu()[s // 2])
    want = -r.p * f[:, None]
    want[torch.arange(len(at)), tokens.clamp(min=0)] += f
    off = r.p * (f.abs()[:, None] * (r.weighed + r.slack + 8 * U) + f_off[:, None])
    off[torch.arange(len(at)), tokens.clamp(min=0)] += f_off + 2 * U * f.abs()
    close(grad[at], torch.where(r.allowed, want, 0.0), torch.where(r.allowed, off, 0.0), "gradient", torch.bfloat16)


@gpu
@pytest.mark.parametrize("masked", [False, True])
def test_preference_of_rows_far_apart(masked):
    """Rows 2^30 elements apart, every one with a token that is allowed: results and gradient are those of the same rows side by side, and not zero."""
    r = Rows(3, 5000, "bf16", "share" if masked else "none", 1.0, 9)
    if masked:
        r.bits[:, 1:4] = True
        r.update()
    x, m = r.on_gpu("far")
    near = r.x.cuda().requires_grad_()
    x.requires_grad_()
    t, offsets = torch.tensor([1, 2, 3], device="cuda"), torch.tensor([0, 1, 3], device="cuda")
    ref = torch.tensor([-1.0, -2.0, -3.0], device="cuda")
    a, b = zf.preference_loss(x, t, offsets, ref, m), zf.preference_loss(near, t, offsets, ref, m)
    for p, q in zip(a, b):
        assert torch.isfinite(p).all()
        same_bits(p, q, "results")
    grad, = torch.autograd.grad(a.loss, x)
    same_bits(grad, torch.autograd.grad(b.loss, near)[0], "gradient")
    assert torch.isfinite(grad).all() and all(grad[i].any() for i in range(3))
    losses, bound, chosen, rejected, D_off, want, off = preference_want(r, t.cpu(), offsets.cpu(), ref.cpu(), 0.1, 0.0, False, None)
    close(a.losses, losses, bound, "losses")
    close(grad, want, off, "gradient", torch.bfloat16)
