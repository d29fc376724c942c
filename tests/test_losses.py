"""The losses on logits under masks (distill_loss, policy_loss, preference_loss) and their gradients against their definitions in 64 bits on the CPU, and their refusals.

Tolerances count roundings of u = 2^-24.  An element's 2^y, y = (x - m) c, is off by 3 u |z - max z| relative (the difference, c and the product) and 2 u (the instruction); a sum over
a row by as much on the mean, weighted with p, and u for each addition in a chain: V / 256 elements of a thread, eight at a time, and 20 over the threads.  That is
`slack`, the error of a log probability but for its last rounding.  What follows of a row is in 64 bits; results and gradients are rounded once, by half a step of their type."""
import ctypes
import math

import pytest
import torch

import paper_2506_01151_amd as zf
from tests.test_operators import DTYPES, half_step, packed, rows_of

gpu = pytest.mark.gpu
U, INF, TINY = 2.0 ** -24, math.inf, 2.0 ** -126
IDS = {4: torch.int32, 8: torch.int64}


@pytest.fixture(params=["module", "definition"])
def by(request, monkeypatch):
    """The extension module's way, and losses.py's own, which takes what the module does not."""
    if request.param == "definition":
        from paper_2506_01151_amd import losses

        class Nothing:
            distill_loss = policy_loss = preference_loss = staticmethod(lambda *args: None)

        monkeypatch.setattr(losses, "_native_losses", Nothing)
    return request.param


# ---- rows, and what is known of them in 64 bits -----------------------------------------------------
class Rows:
    """logits [rows, V] of a type, a mask of a kind, and in 64 bits: lp, p (0 where nothing is allowed), what is allowed, slack [rows, 1]."""

    def __init__(self, rows, V, dtype, mask, temperature, seed, sigma=3.0):
        self.g = torch.Generator().manual_seed(seed)
        self.n, self.V, self.T = rows, V, temperature
        self.x = (torch.randn((rows, V), generator=self.g) * sigma).to(DTYPES[dtype])
        self.bits = None
        if mask == "share":
            self.bits = torch.rand((rows, V), generator=self.g) < torch.rand((rows, 1), generator=self.g)
        elif mask == "few":
            self.bits = torch.rand((rows, V), generator=self.g) < 20.0 / V
        if self.bits is not None and rows > 2:
            self.bits[rows // 2] = False           # nothing is left
            self.bits[0] = False
            self.bits[0, V - 1] = True             # a single token
        self.update()

    def update(self):
        x = self.x.double()
        self.allowed = (x > -INF) if self.bits is None else (x > -INF) & self.bits
        z = torch.where(self.allowed, x / self.T, -INF)
        most = z.amax(dim=1, keepdim=True)
        self.some = most > -INF
        self.z = torch.where(self.some, z - most, -INF)
        total = torch.exp(self.z).sum(dim=1, keepdim=True)
        self.lp = torch.where(self.some, self.z - torch.log(total), -INF)
        self.p = torch.exp(self.lp)
        self.weighed = 3 * U * torch.where(self.allowed, -self.z, 0.0) + 2 * U            # of an element, relative
        self.slack = (self.p * self.weighed).sum(dim=1, keepdim=True) + U * (self.V / 256 + 28)
        self.H = -torch.where(self.p > 0, self.p * self.lp, 0.0).sum(dim=1)

    def on_gpu(self, layout="packed"):
        return rows_of(self.x, layout), None if self.bits is None else packed(self.bits, padding=True).cuda()

    def tokens(self, ids, padding=0.15):
        """Allowed tokens, some forbidden ones where there are such, some padding."""
        score = torch.where(self.allowed, torch.rand((self.n, self.V), generator=self.g), -1.0)
        t = score.argmax(dim=1)
        other = torch.rand((self.n,), generator=self.g)
        t = torch.where(other > 0.9, torch.randint(self.V, (self.n,), generator=self.g), t)
        return torch.where(torch.rand((self.n,), generator=self.g) < padding, torch.tensor(-7), t).to(IDS[ids])

    def at(self, t):
        """(lp of the tokens, 0 for padding; whether a row counts)"""
        i = t.long().clamp(min=0)[:, None]
        return torch.where(t >= 0, self.lp.gather(1, i)[:, 0], 0.0), (t >= 0) & self.allowed.gather(1, i)[:, 0]


def close(got, want, bound, what, dtype=torch.float32):
    """got, of a type, is within `bound` and half a step of its type of want; infinities and NaN are where they are wanted."""
    got = got.detach().cpu().double()
    want = want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), f"{what}: infinities elsewhere"
    limit = bound * (1 + 2.0 ** -7) + want.abs() * half_step(dtype) * (1 + 2.0 ** -7) + TINY
    off = torch.where(finite, (got - want).abs() - limit, 0.0)
    off = torch.nan_to_num(off, nan=0.0, posinf=0.0, neginf=0.0) if not finite.all() else off
    worst = int(off.argmax()) if off.numel() else 0
    assert not off.numel() or off.max() <= 0, f"{what}: {got.reshape(-1)[worst]} instead of {want.reshape(-1)[worst]}, which is {limit.expand_as(got).reshape(-1)[worst]} off at most ({int((off > 0).sum())} of them)"


def loss_bound(weight, losses, bound):
    """Of the sum: its terms' errors and half a step of each (the result is made from the rounded losses)."""
    w = weight.double() if weight is not None else torch.ones_like(losses)
    return (w * losses).sum(), (w.abs() * (bound + U * losses.abs())).sum()


# ---- distillation -----------------------------------------------------------------------------------
def teacher(r, K, ids, values, rest, seed, twice=False):
    """A teacher near the student: its K most probable allowed tokens, -1 where there are no more; a token that the student does not allow among them."""
    g = torch.Generator().manual_seed(seed)
    t = torch.where(r.allowed, 0.8 * r.x.double() / r.T + torch.randn(r.x.shape, generator=g), -INF)
    lp = t - torch.where(r.some, torch.logsumexp(t, dim=1, keepdim=True), 0.0)
    n = min(K, r.V)
    best, at = torch.topk(lp, n, dim=1)
    got = torch.full((r.n, K), -1).long()
    got[:, :n] = torch.where(best > -INF, at, -1)
    v = torch.full((r.n, K), -INF, dtype=torch.float64)
    v[:, :n] = best if rest else best * r.T + 3.0
    for i in range(r.n):
        if i % 5 == 4 and not r.allowed[i].all():
            got[i, K // 2] = int((~r.allowed[i]).nonzero()[0])
            v[i, K // 2] = -0.5
        if i % 7 == 3:
            got[i] = -1
        if i % 7 == 5:
            v[i, K - 1] = -INF
        if twice and K > 2:
            got[i, 2], got[i, K - 1] = got[i, 0], got[i, 0]
    return got.to(IDS[ids]), v.to(DTYPES[values])


def distill_want(r, ids, values, rest, weight, dtype):
    """(losses, their bound, gradient, its bound) by the definition, row by row."""
    losses, bound = torch.zeros(r.n, dtype=torch.float64), torch.zeros(r.n, dtype=torch.float64)
    grad, off = torch.zeros((r.n, r.V), dtype=torch.float64), torch.zeros((r.n, r.V), dtype=torch.float64)
    for i in range(r.n):
        entries = [(int(v), float(t)) for v, t in zip(ids[i], values[i].double()) if v >= 0 and r.allowed[i, int(v)]]
        if not entries:
            continue
        at = torch.tensor([e[0] for e in entries])
        t = torch.tensor([e[1] for e in entries], dtype=torch.float64)
        ln_q = t if rest else (t / r.T if (t == -INF).all() else t / r.T - torch.logsumexp(t / r.T, dim=0))
        q = torch.exp(ln_q)
        slack, lp, p = float(r.slack[i]), r.lp[i], r.p[i]
        losses[i] = torch.where(q > 0, q * (ln_q - lp[at]), 0.0).sum()
        bound[i] = q.sum() * slack
        coefficient, spread = q.sum() * torch.ones(r.V, dtype=torch.float64), torch.zeros(r.V, dtype=torch.float64)
        if rest:
            outside = torch.ones(r.V, dtype=torch.bool)
            outside[at] = False
            p_rest = p[outside].sum()
            q_rest = max(0.0, 1.0 - float(q.sum())) if p_rest > 0 else 0.0
            if q_rest > 0:
                losses[i] += q_rest * (math.log(q_rest) - math.log(p_rest))
                rest_slack = slack + float((p * r.weighed[i])[outside].sum() / p_rest) + U * (r.V / 256 + 28)
                bound[i] += q_rest * rest_slack
                coefficient = coefficient + q_rest
                coefficient[outside] -= q_rest / p_rest
                spread[outside] = q_rest / p_rest * (rest_slack + U)   # a difference: each side's own error
        f = torch.zeros(r.V, dtype=torch.float64).index_add_(0, at, q)
        w = float(weight[i]) / r.T
        grad[i] = w * (coefficient * p - f)
        off[i] = abs(w) * (p * ((q.sum() + 1) * (r.weighed[i] + slack + 6 * U) + spread) + 2 * U * len(entries) * f)
        grad[i, ~r.allowed[i]] = 0.0
        off[i, ~r.allowed[i]] = 0.0
    return losses, bound, grad, off


DISTILL = [                                        # rows, V, K
    (1, 1, 1), (3, 2, 2), (1, 2048, 5), (7, 31, 3), (9, 33, 64), (20, 1000, 20), (5, 8193, 200), (16, 40037, 64), (4, 131073, 7), (3, 300001, 1024), (600, 257, 4),
]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,V,K", DISTILL)
def test_distill(rows, V, K, rest, dtype):
    seed = rows * 7919 + V + K
    mask, T, ids, values, layout = ("none", "share", "few")[seed % 3], (1.0, 2.0, 0.7)[seed % 3], (4, 8)[seed % 2], ("f32", "bf16")[seed // 2 % 2], ("packed", "padded", "odd")[seed // 3 % 3]
    r = Rows(rows, V, dtype, mask, T, seed)
    listed, v = teacher(r, K, ids, values, rest, seed + 1, twice=seed % 4 == 1)
    weight = torch.rand((rows,), generator=r.g) + 0.5
    losses, bound, grad, off = distill_want(r, listed, v, rest, weight, dtype)
    x, m = r.on_gpu(layout)
    x.requires_grad_()
    got = zf.distill_loss(x, listed.cuda(), v.cuda(), m, temperature=T, rest=rest, weight=weight.cuda())
    close(got.losses, losses, bound, "losses")
    close(got.loss, *loss_bound(weight, losses, bound), "loss")
    g, = torch.autograd.grad(got.loss, x)
    assert g.dtype == x.dtype
    close(g, grad, off, "gradient", x.dtype)
    with torch.no_grad():
        alone = zf.distill_loss(x, listed.cuda(), v.cuda(), m, temperature=T, rest=rest, weight=weight.cuda())
    assert torch.equal(alone.losses, got.losses) and torch.equal(alone.loss, got.loss) and not alone.loss.requires_grad


@gpu
def test_distill_what_is_sure():
    """A student whose rest is 1e-9 of it, a teacher whose rest is 1e-8: differences from 1 would be noise."""
    x = torch.zeros((2, 5000))
    x[:, 17] = 30.0
    x[1, 23] = 29.0
    ids = torch.tensor([[17, 23, 4], [17, 23, 4]])
    v = torch.tensor([[-2e-8, -30.0, -40.0], [-0.3132617, -1.3132617, -20.0]])
    r = Rows(2, 5000, "f32", "none", 1.0, 1)
    r.x = x
    r.update()
    weight = torch.ones(2)
    losses, bound, grad, off = distill_want(r, ids, v, True, weight, "f32")
    xg = x.cuda().requires_grad_()
    got = zf.distill_loss(xg, ids.cuda(), v.cuda(), rest=True)
    close(got.losses, losses, bound, "losses")
    g, = torch.autograd.grad(got.loss, xg)
    close(g, grad, off, "gradient")
    outside = torch.ones(5000, dtype=torch.bool)
    outside[ids[0]] = False
    assert (g.cpu()[0, outside].double() - grad[0, outside]).abs().max() < 1e-4 * grad[0, outside].abs().max()


@gpu
def test_distill_the_rest_that_underflows():
    """All that is not listed lies 200 below: its share of the student is 0 in 32 bits, its logarithm is not."""
    x = torch.full((1, 3000), -200.0)
    x[0, :3] = 0.0
    r = Rows(1, 3000, "f32", "none", 1.0, 1)
    r.x = x
    r.update()
    ids, v = torch.tensor([[0, 1, 2]]), torch.log(torch.tensor([[0.2, 0.3, 0.4]]))
    losses, bound, grad, off = distill_want(r, ids, v, True, torch.ones(1), "f32")
    xg = x.cuda().requires_grad_()
    got = zf.distill_loss(xg, ids.cuda(), v.cuda(), rest=True)
    assert losses[0] > 15
    close(got.losses, losses, bound, "losses")
    close(torch.autograd.grad(got.loss, xg)[0], grad, off, "gradient")


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 900, 40037, 170001])
@pytest.mark.parametrize("K", [1, 3, 64, 65, 200])
def test_distill_values_that_are_all_minus_infinity(K, V, dtype, by):
    """Rows whose teacher gives nothing to any listed token that the student allows: loss 0 and no gradient at all, the forward call's or one made again; with `rest` all is the other tokens'.
    Beside them rows of which a whole 64 entries, the first or the last, are so, and rows whose only finite value is of a forbidden token."""
    n, T = 7, 0.7
    r = Rows(n, V, dtype, "none", T, 31 + K)
    r.bits = torch.rand((n, V), generator=r.g) < 0.6
    r.bits[:, 0] = True
    r.bits[3:5, V - 1] = False
    r.bits[5, V - 1] = True
    r.update()
    ids = torch.randint(V - 1, (n, K), generator=r.g)
    ids[:, 0] = 0
    v = torch.full((n, K), -INF)
    ids[3:6, K - 1] = V - 1                        # the only finite one: forbidden in rows 3 and 4, allowed in row 5
    v[3:6, K - 1] = -0.25
    v[6] = -1.0 - torch.rand((K,), generator=r.g)
    v[6, :64 if K > 64 else 0] = -INF
    ids[2, 1:] = -1                                # (one entry counts)
    weight = torch.rand((n,), generator=r.g) + 0.5
    x, m = r.on_gpu()
    x.requires_grad_()
    for rest in (False, True):
        losses, bound, grad, off = distill_want(r, ids, v, rest, weight, dtype)
        got = zf.distill_loss(x, ids.cuda(), v.cuda(), m, temperature=T, rest=rest, weight=weight.cuda())
        close(got.losses, losses, bound, "losses")
        first, = torch.autograd.grad(got.loss, x, retain_graph=True)
        again, = torch.autograd.grad(got.loss * -2.0, x)
        close(first, grad, off, "gradient", x.dtype)
        close(again, -2 * grad, 2 * off, "gradient made again", x.dtype)
        if not rest:
            without = [0, 1, 2] + ([3, 4] if K > 1 else [])        # (of one entry, rows 3 and 4 have none that counts)
            assert (got.losses[without] == 0).all() and (first[without] == 0).all() and (again[without] == 0).all()
        with torch.no_grad():
            assert torch.equal(zf.distill_loss(x, ids.cuda(), v.cuda(), m, temperature=T, rest=rest, weight=weight.cuda()).losses, got.losses)


# ---- the policy's loss ------------------------------------------------------------------------------
def policy_want(r, t, old, adv, ref, clip, kl, e, weight):
    lp, counts = r.at(t)
    safe = torch.where(counts, lp, 0.0)
    slack = r.slack[:, 0]
    a = adv.double()
    ratio = torch.exp(safe - old.double())
    kept = ratio.clamp(1 - clip[0], 1 + clip[1])
    losses = -torch.minimum(ratio * a, kept * a)
    clipped = kept * a < ratio * a
    f = torch.where(clipped, 0.0, -ratio * a)
    df = f.abs()
    if ref is not None:
        d = ref.double() - safe
        losses = losses + kl * (torch.expm1(d) - d)
        f = f - kl * torch.expm1(d)
        df = df + abs(kl) * torch.exp(d)
    H = torch.where(t >= 0, r.H, 0.0)
    # entropy: ln S - ln 2 T / S, both sums off by their elements and additions; T's elements by |y| u more
    span = (r.p * torch.where(r.allowed, -r.z, 0.0)).sum(dim=1)
    H_off = slack * (2 + 2 * span) + (r.p * torch.where(r.allowed, r.z ** 2, 0.0)).sum(dim=1) * 4 * U + 4 * U * span
    bound = f.abs() * slack + df * slack ** 2
    if e is not None:
        losses = losses - e * H
        bound = bound + abs(e) * (H_off + U * H)
    losses, f, df, bound = (torch.where(counts, y, 0.0) for y in (losses, f, df, bound))
    w = (weight.double() if weight is not None else torch.ones(r.n, dtype=torch.float64))[:, None] / r.T
    grad = -r.p * f[:, None]
    off = r.p * f.abs()[:, None] * (r.weighed + r.slack + 6 * U) + r.p * (df * slack)[:, None]
    rows = torch.arange(r.n)
    at = t.long().clamp(min=0)
    grad[rows, at] += f
    off[rows, at] += df * slack + 2 * U * f.abs()
    if e is not None:
        plp = torch.where(r.p > 0, r.p * r.lp, 0.0)
        grad = grad + torch.where(counts, e, 0.0)[:, None] * (plp + r.p * H[:, None])
        size = torch.where(r.p > 0, r.p * (r.lp.abs() + H[:, None]), 0.0)
        off = off + torch.where(counts, abs(e), 0.0)[:, None] * (size * (r.weighed + 2 * r.slack + 8 * U) + r.p * (H_off[:, None] + r.weighed * 2))
    grad, off = torch.where(r.allowed, grad, 0.0), torch.where(r.allowed, off, 0.0)
    return losses, bound, lp, H, H_off, w * grad, w.abs() * off


POLICY = [(1, 1), (1, 2048), (3, 5), (33, 127), (16, 32000), (5, 40037), (700, 300), (3, 152064), (4, 131073), (2, 600001), (9, 65536)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kl,e", [(None, None), (0.05, None), (None, 0.01), (0.1, -0.5), (0.02, 0.0)])
@pytest.mark.parametrize("rows,V", POLICY)
def test_policy(rows, V, kl, e, dtype):
    seed = rows * 7919 + V + int(1000 * ((kl or 0) + (e or 0)))
    mask, T, ids, layout = ("none", "share", "few")[seed % 3], (1.0, 0.7, 1.3)[seed // 3 % 3], (4, 8)[seed % 2], ("packed", "padded", "odd")[seed // 2 % 3]
    r = Rows(rows, V, dtype, mask, T, seed)
    t = r.tokens(ids)
    lp, counts = r.at(t)
    safe = torch.where(counts, lp, 0.0)
    old = (safe + 0.3 * torch.randn((rows,), generator=r.g)).float()
    ref = (safe + 0.5 * torch.randn((rows,), generator=r.g)).float() if kl is not None else None
    adv = torch.randn((rows,), generator=r.g)
    weight = torch.rand((rows,), generator=r.g) if seed % 2 else None
    losses, bound, lp, H, H_off, grad, off = policy_want(r, t, old, adv, ref, (0.2, 0.3), kl or 0.0, e, weight)
    x, m = r.on_gpu(layout)
    x.requires_grad_()
    cuda = [y.cuda() if y is not None else None for y in (t, old, adv, ref, weight)]
    got = zf.policy_loss(x, *cuda[:3], m, ref_logprobs=cuda[3], temperature=T, clip=(0.2, 0.3), kl_weight=kl or 0.0, entropy_weight=e, weight=cuda[4])
    close(got.logprobs, lp, torch.where(lp > -INF, r.slack[:, 0], 0.0), "log probabilities")
    if e is None:
        assert got.entropy is None
    else:
        close(got.entropy, H, H_off, "entropy")
    close(got.losses, losses, bound, "losses")
    close(got.loss, *loss_bound(weight, losses, bound), "loss")
    g, = torch.autograd.grad(got.loss, x)
    close(g, grad, off, "gradient", x.dtype)
    alone = zf.policy_loss(x.detach(), *cuda[:3], m, ref_logprobs=cuda[3], temperature=T, clip=(0.2, 0.3), kl_weight=kl or 0.0, entropy_weight=e, weight=cuda[4])
    assert torch.equal(alone.losses, got.losses) and torch.equal(alone.logprobs, got.logprobs) and torch.equal(alone.loss, got.loss)


@gpu
def test_policy_sides_of_the_clipping():
    """Ratios below, between and above the borders, advantages of both signs and zero, an infinite border."""
    V = 64
    x = torch.zeros((9, V), device="cuda", requires_grad=True)
    t = torch.arange(9, device="cuda")
    ratios = torch.tensor([0.5, 1.0, 2.0] * 3, dtype=torch.float64)
    old = (-math.log(V) - torch.log(ratios)).float().cuda()
    adv = torch.tensor([1.0] * 3 + [-1.0] * 3 + [0.0] * 3)
    for clip, kept in (((0.2, 0.3), [0.5, 1.0, 1.3, 0.8, 1.0, 2.0, 0, 0, 0]), ((0.2, INF), [0.5, 1.0, 2.0, 0.8, 1.0, 2.0, 0, 0, 0])):
        got = zf.policy_loss(x, t, old, adv.cuda(), clip=clip)
        want = -torch.tensor(kept, dtype=torch.float64) * adv
        assert (got.losses.cpu().double() - want).abs().max() < 1e-6
        slope = torch.autograd.grad(got.loss, x)[0].cpu()[torch.arange(9), torch.arange(9)] / (1 - 1 / V)
        free = torch.tensor([abs(k - float(q)) < 1e-6 for k, q in zip(kept, ratios)])
        assert (slope - torch.where(free, -(ratios * adv), 0.0)).abs().max() < 1e-5


# ---- masks that leave few tokens, from none to all, of long rows: of up to 16 and 20 pieces a thread, and longer ones ----
def few_rows(dtype, seed, rows, V):
    r = Rows(rows, V, dtype, "few", 0.8, seed)
    for i, n in enumerate((0, 1, 2, 64, 300, 2047, 2048, 2049, 2050, V)):
        where = torch.randperm(V, generator=r.g)[:n]
        r.bits[i] = False
        r.bits[i, where] = True
    r.bits[10] = False
    r.bits[10, V - 2048:] = True                   # at the row's end
    r.bits[11] = False
    r.bits[11, :2048] = True
    r.bits[11, V - 1] = True                       # one too many, which comes last
    r.bits[12, :40] = True
    r.x[12, :40] = -INF                            # allowed and -inf
    r.update()
    return r


@gpu
@pytest.mark.parametrize("dtype,rows,V", [("f32", 280, 30011), ("bf16", 300, 60001), ("bf16", 131, 131072), ("f32", 64, 152064), ("bf16", 150, 152065), ("f32", 33, 262144), ("f32", 33, 262176)])
@pytest.mark.parametrize("e", [None, 0.05])
def test_policy_of_few_tokens(dtype, rows, V, e):
    r = few_rows(dtype, rows + V, rows, V)
    t = r.tokens(8)
    lp, counts = r.at(t)
    old = torch.where(counts, lp, 0.0).float() + 0.1
    adv = torch.randn((rows,), generator=r.g)
    losses, bound, lp, H, H_off, grad, off = policy_want(r, t, old, adv, None, (0.2, 0.2), 0.0, e, None)
    x, m = r.on_gpu("odd" if V % 2 else "packed")
    x.requires_grad_()
    got = zf.policy_loss(x, t.cuda(), old.cuda(), adv.cuda(), m, temperature=0.8, entropy_weight=e)
    close(got.logprobs, lp, torch.where(lp > -INF, r.slack[:, 0], 0.0), "log probabilities")
    close(got.losses, losses, bound, "losses")
    if e is not None:
        close(got.entropy, H, H_off, "entropy")
    g, = torch.autograd.grad(got.loss, x, retain_graph=True)
    close(g, grad, off, "gradient", x.dtype)
    g, = torch.autograd.grad(got.loss, x, torch.tensor(-2.0, device="cuda"))
    close(g, -2 * grad, 2 * off, "gradient", x.dtype)
    assert all(torch.equal(p, q) for p, q in zip(zf.policy_loss(x.detach(), t.cuda(), old.cuda(), adv.cuda(), m, temperature=0.8, entropy_weight=e), got) if p is not None)


@gpu
@pytest.mark.parametrize("dtype,rows,V,K", [("f32", 280, 30011, 3), ("bf16", 131, 131072, 70), ("f32", 64, 152064, 1024)])
@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_few_tokens(dtype, rows, V, K, rest):
    r = few_rows(dtype, rows + V, rows, V)
    listed, v = teacher(r, K, 4, "f32", rest, 5, twice=rows % 3 == 1)
    weight = torch.rand((rows,), generator=r.g)
    losses, bound, grad, off = distill_want(r, listed, v, rest, weight, dtype)
    x, m = r.on_gpu()
    x.requires_grad_()
    got = zf.distill_loss(x, listed.cuda(), v.cuda(), m, temperature=0.8, rest=rest, weight=weight.cuda())
    close(got.losses, losses, bound, "losses")
    g, = torch.autograd.grad(got.loss, x)
    close(g, grad, off, "gradient", x.dtype)


# ---- preferences ------------------------------------------------------------------------------------
def preference_want(r, t, offsets, ref, beta, s, average, weight):
    lp, counts = r.at(t)
    o = [int(y) for y in offsets]
    P = len(o) // 2
    D, D_off, n = torch.zeros(2 * P, dtype=torch.float64), torch.zeros(2 * P, dtype=torch.float64), [1.0] * (2 * P)
    for i in range(2 * P):
        mine = [j for j in range(o[i], o[i + 1]) if t[j] >= 0]
        if average:
            n[i] = max(1, len(mine))
        for j in mine:
            D[i] += (lp[j] - (float(ref[j]) if ref is not None else 0.0)) / n[i]
            D_off[i] += ((r.slack[j, 0] + U * abs(lp[j])) / n[i]) if lp[j] > -INF else 0.0       # the log probabilities are rounded before they are added
    chosen, rejected = beta * D[0::2], beta * D[1::2]
    h, h_off = chosen - rejected, abs(beta) * (D_off[0::2] + D_off[1::2])
    losses = -(1 - s) * torch.nn.functional.logsigmoid(h) - (s * torch.nn.functional.logsigmoid(-h) if s else 0.0)
    dh = (s * torch.sigmoid(h) if s else 0.0) - (1 - s) * torch.sigmoid(-h)
    bound = dh.abs() * h_off + 0.25 * h_off ** 2
    w = weight.double() if weight is not None else torch.ones(P, dtype=torch.float64)
    f, f_off = torch.zeros(r.n, dtype=torch.float64), torch.zeros(r.n, dtype=torch.float64)
    for i in range(2 * P):
        c = beta * w[i // 2] / n[i] / r.T
        for j in range(o[i], o[i + 1]):
            if counts[j]:
                f[j] = c * dh[i // 2] * (1 - 2 * (i % 2))
                f_off[j] = abs(c) * (0.25 * h_off[i // 2] + 3 * U * abs(dh[i // 2]))
    grad = torch.where(r.allowed, -r.p * f[:, None], 0.0)
    off = torch.where(r.allowed, r.p * (f.abs()[:, None] * (r.weighed + r.slack + 8 * U) + f_off[:, None]), 0.0)
    rows, at = torch.arange(r.n), t.long().clamp(min=0)
    grad[rows, at] += f
    off[rows, at] += f_off + 2 * U * f.abs()
    return losses, bound, chosen, rejected, abs(beta) * D_off, grad, off


PREFERENCE = [                                     # lengths of the sequences, rows before and behind them, V
    ([1, 1], 0, 0, 1), ([3, 0], 0, 1, 7), ([0, 0], 1, 0, 40), ([5, 4, 1, 9], 2, 3, 257), ([12, 12], 0, 0, 2048), ([300, 129, 1, 64], 5, 1, 33),
    ([6, 3], 1, 1, 40037), ([2, 2], 0, 1, 152064), ([1, 2], 0, 0, 300001), ([2] * 200, 0, 7, 65), ([], 0, 3, 9), ([20, 30, 10, 7, 8, 9], 0, 2, 9000),
]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("average,s,beta", [(False, 0.0, 0.1), (True, 0.1, 2.5), (False, 1.0, -0.3)])
@pytest.mark.parametrize("case", range(len(PREFERENCE)))
def test_preference(case, average, s, beta, dtype):
    lengths, before, behind, V = PREFERENCE[case]
    rows, P, seed = before + sum(lengths) + behind, len(lengths) // 2, case * 100 + int(10 * abs(beta))
    mask, T, ids, layout = ("none", "share")[seed % 2], (1.0, 0.7, 1.3)[seed // 3 % 3], (4, 8)[seed // 2 % 2], ("packed", "padded", "odd")[case % 3]
    r = Rows(rows, V, dtype, mask, T, seed)
    if r.bits is not None:
        r.bits[:, V // 2] = True                   # (rows that allow nothing are in the test of what is not allowed)
        r.update()
    t = r.tokens(ids, padding=0.3)
    lp, counts = r.at(t)
    t = torch.where(counts, t, -1).to(t.dtype)
    lp, counts = r.at(t)
    ref = (lp + 0.3 * torch.randn((rows,), generator=r.g)).float() if case % 4 else None
    weight = torch.rand((P,), generator=r.g) + 0.1 if case % 2 else None
    offsets = torch.tensor([before] + [before + sum(lengths[:i + 1]) for i in range(len(lengths))]).to(IDS[(4, 8)[case % 2]])
    losses, bound, chosen, rejected, D_off, grad, off = preference_want(r, t, offsets, ref, beta, s, average, weight)
    x, m = r.on_gpu(layout)
    x.requires_grad_()
    cuda = [y.cuda() if y is not None else None for y in (t, offsets, ref, weight)]
    got = zf.preference_loss(x, *cuda[:3], m, beta=beta, label_smoothing=s, average=average, temperature=T, weight=cuda[3])
    close(got.chosen, chosen, D_off[0::2], "chosen")
    close(got.rejected, rejected, D_off[1::2], "rejected")
    close(got.losses, losses, bound, "losses")
    close(got.loss, *loss_bound(weight, losses, bound), "loss")
    g, = torch.autograd.grad(got.loss, x)
    close(g, grad, off, "gradient", x.dtype)
    alone = zf.preference_loss(x.detach(), *cuda[:3], m, beta=beta, label_smoothing=s, average=average, temperature=T, weight=cuda[3])
    assert all(torch.equal(a, b) for a, b in zip(alone, got))


@gpu
def test_preference_of_tokens_that_are_not_allowed():
    """The preferred sequence has one: its sum is -inf, the loss infinite, and the other rows' gradients as they are where sigma is at its end; the other has one: nothing is left to learn."""
    V = 50
    x = torch.randn((8, V), generator=torch.Generator().manual_seed(3)).cuda().requires_grad_()
    bits = torch.ones((8, V), dtype=torch.bool)
    bits[1, 9], bits[6, 9] = False, False
    t = torch.full((8,), 9, device="cuda")
    offsets = torch.tensor([0, 2, 4, 6, 8], device="cuda")
    got = zf.preference_loss(x, t, offsets, mask=packed(bits).cuda())
    assert got.losses.tolist() == [INF, 0.0] and got.chosen[0] == -INF and got.rejected[1] == -INF
    g, = torch.autograd.grad(got.loss, x)
    p = torch.softmax(x.detach().double(), dim=1).cpu()
    want = 0.1 * p
    want[:, 9] -= 0.1
    want[2:4] *= -1
    want[1], want[4:] = 0.0, 0.0
    assert (g.cpu().double() - want).abs().max() < 1e-7


@gpu
@pytest.mark.parametrize("s,want", [(0.0, [INF, 0.0]), (1.0, [0.0, INF]), (0.5, [INF, INF])])
def test_preference_shares_of_infinite_terms(s, want):
    """Of pairs that are infinitely far apart: the term that has no share does not make the loss NaN."""
    x = torch.zeros((4, 40), device="cuda").requires_grad_()
    bits = torch.ones((4, 40), dtype=torch.bool)
    bits[0, 9], bits[3, 9] = False, False
    got = zf.preference_loss(x, torch.full((4,), 9, device="cuda"), torch.arange(5, device="cuda"), mask=packed(bits).cuda(), label_smoothing=s)
    assert got.losses.tolist() == want and got.chosen[0] == -INF and got.rejected[1] == -INF
    g, = torch.autograd.grad(got.loss, x)
    # lp of row 1 counts -beta, of row 2 beta; d loss / d h is s - 1 for h = -inf, s for h = inf.  Three roundings of 0.1 at most: the slope's, p f's together, their sum's.
    for row, f in ((1, 0.1 * (1 - s)), (2, 0.1 * s)):
        at = torch.full((40,), -f / 40, dtype=torch.float64)
        at[9] += f
        assert (g[row].double().cpu() - at).abs().max() <= 0.3 * U
    assert not g[0].any() and not g[3].any()


@gpu
@pytest.mark.parametrize("offsets,bad", [([0, 5, 3, 6, 8], [True, True]), ([0, 2, 4, 6, 9], [False, True]), ([-1, 2, 4, 6, 8], [True, False]), ([0, 2 ** 40, 4, 6, 8], [True, True])])
def test_preference_offsets_that_do_not_fit(offsets, bad):
    x = torch.randn((8, 30), generator=torch.Generator().manual_seed(4)).cuda().requires_grad_()
    t = torch.arange(8, device="cuda")
    got = zf.preference_loss(x, t, torch.tensor(offsets, device="cuda"))
    assert torch.isnan(got.losses).tolist() == bad and torch.isnan(got.chosen).tolist() == bad
    g, = torch.autograd.grad(got.loss, x)
    assert g.shape == x.shape


@gpu
@pytest.mark.parametrize("offsets,may_be", [([0, 5, 3, 6, 8], [1]), ([4, 8, 2, 3, 6, 7, 8], [1, 2]), ([0, 4, 8, 0, 8], [0]), (list(range(0, 130)) + [5, 9, 130], list(range(0, 64)))])
def test_preference_offsets_that_overlap(offsets, may_be):
    """A pair is either right, as it is alone, or NaN: a row that the offsets give to two sequences is not left out without a word."""
    n = max(offsets) + 1
    x = torch.randn((n, 30), generator=torch.Generator().manual_seed(4)).cuda()
    t = torch.arange(n, device="cuda") % 30
    got = zf.preference_loss(x, t, torch.tensor(offsets, device="cuda"))
    nan = torch.isnan(got.losses).tolist()
    assert nan == torch.isnan(got.chosen).tolist() == torch.isnan(got.rejected).tolist()
    for i, (a, b, c) in enumerate(zip(offsets[0::2], offsets[1::2], offsets[2::2])):
        assert nan[i] or (i in may_be and a <= b <= c)
        if not nan[i]:
            alone = zf.preference_loss(x, t, torch.tensor([a, b, c], device="cuda"))
            assert float(got.losses[i]) == float(alone.losses[0]) and float(got.chosen[i]) == float(alone.chosen[0])


# ---- what rows can hold -----------------------------------------------------------------------------
def beside(x):
    """What the losses need beside rows: token 1 of each, tokens 1 and 2 of a teacher, two sequences."""
    n = x.shape[0]
    return (torch.ones((n,), dtype=torch.int64, device=x.device), torch.zeros((n,), device=x.device), torch.tensor([[1, 2]], device=x.device).expand(n, 2).contiguous(),
            torch.tensor([[-0.5, -1.5]], device=x.device).expand(n, 2).contiguous(), torch.tensor([0, n // 2, n], device=x.device))


def three(x, mask=None, needs=None, **more):
    """The three losses (distillation twice) on the same rows."""
    t, zeros, ids, v, half = needs or beside(x)
    return [zf.distill_loss(x, ids, v, mask, rest=False, **more), zf.distill_loss(x, ids, v, mask, rest=True, **more), zf.policy_loss(x, t, zeros - 2, zeros + 1, mask, entropy_weight=0.1, **more),
            zf.preference_loss(x, t, half, None, mask, **more)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_forbidden_is_not_looked_at(dtype, by):
    """NaN, infinities and the type's largest numbers in forbidden places change nothing, and their gradient is 0; -inf in allowed places is as forbidden."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn((6, 3000), generator=g).to(DTYPES[dtype])
    bits = torch.rand((6, 3000), generator=g) < 0.3
    bits[:, 1:3] = True
    bits[4] = False
    plain = torch.where(bits, x, torch.tensor(-INF).to(x.dtype))
    wild = x.clone()
    wild[~bits] = torch.tensor([math.nan, INF, -INF, torch.finfo(x.dtype).max])[torch.randint(4, (int((~bits).sum()),), generator=g)].to(x.dtype)
    a, b = wild.cuda().requires_grad_(), plain.cuda().requires_grad_()
    for i, (of_a, of_b) in enumerate(zip(three(a, packed(bits, padding=True).cuda()), three(b))):
        for p, q in zip(of_a, of_b):
            assert torch.equal(p, q) and (i == 3 or torch.isfinite(p).logical_or(p == -INF).all())
        ga, gb = torch.autograd.grad(of_a.loss, a)[0], torch.autograd.grad(of_b.loss, b)[0]
        assert torch.equal(ga, gb) and (ga.cpu()[~bits] == 0).all() and (i == 3 or torch.isfinite(ga).all())


@gpu
@pytest.mark.parametrize("bad", [math.nan, INF])
def test_what_is_not_a_number_makes_its_row_nan(bad):
    g = torch.Generator().manual_seed(6)
    x = torch.randn((4, 500), generator=g)
    x[2, 400] = bad
    bits = torch.rand((4, 500), generator=g) < 0.5
    bits[:, 1:3], bits[2, 400] = True, True
    xg = x.cuda().requires_grad_()
    for i, got in enumerate(three(xg, packed(bits).cuda())):
        nan = [False, False, True, False] if i < 3 else [True]
        assert torch.isnan(got.losses).tolist() == nan and torch.isnan(got.loss)
        d = torch.autograd.grad(got.loss, xg)[0].cpu()
        if i < 3:
            assert torch.isnan(d[2][bits[2]]).all() and (d[2][~bits[2]] == 0).all() and torch.isfinite(d[[0, 1, 3]]).all()


@gpu
def test_ids_beyond_the_vocabulary(by):
    x = torch.randn((4, 100), generator=torch.Generator().manual_seed(7)).cuda().requires_grad_()
    t = torch.tensor([3, 100, 2 ** 40, 99], device="cuda")
    one = torch.ones((4,), device="cuda")
    got = zf.policy_loss(x, t, one, one)
    assert torch.isnan(got.losses).tolist() == [False, True, True, False] and torch.isnan(got.logprobs).tolist() == [False, True, True, False]
    got = zf.distill_loss(x, torch.stack([t, t * 0 + 5], dim=1), torch.zeros((4, 2), device="cuda"))
    assert torch.isnan(got.losses).tolist() == [False, True, True, False]
    got = zf.preference_loss(x, t, torch.tensor([0, 1, 2, 3, 4], device="cuda"))
    assert torch.isnan(got.losses).tolist() == [True, True]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lowest_values_and_far_temperatures(dtype):
    """Rows that a program masked with the type's lowest value; temperatures whose reciprocals are near 32 bits' ends."""
    x = torch.randn((4, 700), generator=torch.Generator().manual_seed(8)).to(DTYPES[dtype])
    low = torch.finfo(x.dtype).min
    x[0, 3:] = low
    x[1] = low
    x[2, ::2] = low
    r = Rows(4, 700, dtype, "none", 1.0, 1)
    r.x = x
    r.update()
    t, zeros = torch.full((4,), 2), torch.zeros(4)
    losses, bound, lp, H, H_off, grad, off = policy_want(r, t, zeros - 3, zeros + 1, None, (0.2, 0.2), 0.0, None, None)
    xg = x.cuda().requires_grad_()
    got = zf.policy_loss(xg, t.cuda(), zeros.cuda() - 3, zeros.cuda() + 1)
    close(got.losses, losses, torch.nan_to_num(bound, nan=0.0), "losses")
    close(torch.autograd.grad(got.loss, xg)[0], grad, torch.nan_to_num(off, nan=0.0), "gradient", xg.dtype)
    for T in (2.0 ** -126, 1e30):
        for got in three(xg, temperature=T):
            assert not torch.isnan(got.losses[0])
            d = torch.autograd.grad(got.loss, xg)[0]
            assert not torch.isnan(d[0]).any()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,by,offset", [(0.02, 3.0, 400.0), (1.0, 3000.0, -9000.0), (50.0, 1.0, 0.0)])
def test_logits_far_from_zero(dtype, T, by, offset):
    """Logits over temperature in the thousands, of either sign, where a gradient of bf16 takes another way: all three losses."""
    r = Rows(9, 3001, dtype, "share", T, 20, sigma=by)
    r.x = (r.x.float() + offset).to(r.x.dtype)
    r.bits[:, 5:7] = True
    r.update()
    t = torch.where(r.at(torch.full((9,), 5))[1], r.x[:, :].float().masked_fill(~r.allowed, -INF).argmax(dim=1), -1)
    lp, counts = r.at(t)
    x, m = r.on_gpu()
    x.requires_grad_()
    old, adv = lp.float() + 0.05, torch.randn((9,), generator=r.g)
    losses, bound, lp, H, H_off, grad, off = policy_want(r, t, old, adv, None, (0.2, 0.2), 0.0, None, None)
    got = zf.policy_loss(x, t.cuda(), old.cuda(), adv.cuda(), m, temperature=T)
    close(got.losses, losses, bound, "losses")
    close(torch.autograd.grad(got.loss, x)[0], grad, off, "gradient", x.dtype)
    listed, v = teacher(r, 4, 8, "f32", False, 3)
    v = (v * (1.0 / by)).float()
    losses, bound, grad, off = distill_want(r, listed, v, False, torch.ones(9), dtype)
    got = zf.distill_loss(x, listed.cuda(), v.cuda(), m, temperature=T)
    close(got.losses, losses, bound, "losses")
    close(torch.autograd.grad(got.loss, x)[0], grad, off, "gradient", x.dtype)
    offsets = torch.tensor([0, 3, 9])
    losses, bound, chosen, rejected, D_off, grad, off = preference_want(r, t, offsets, old, 0.1, 0.0, False, None)
    got = zf.preference_loss(x, t.cuda(), offsets.cuda(), old.cuda(), m, temperature=T)
    close(got.losses, losses, bound, "losses")
    close(torch.autograd.grad(got.loss, x)[0], grad, off, "gradient", x.dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,V", [(5, 900), (300, 5000), (3, 170000)])
def test_distill_all_that_is_allowed_is_listed(rows, V, rest, dtype):
    r = Rows(rows, V, dtype, "few", 1.0, 21)
    listed, v = teacher(r, 64, 4, "f32", rest, 22)
    losses, bound, grad, off = distill_want(r, listed, v, rest, torch.ones(rows), dtype)
    x, m = r.on_gpu()
    x.requires_grad_()
    got = zf.distill_loss(x, listed.cuda(), v.cuda(), m, rest=rest)
    close(got.losses, losses, bound, "losses")
    close(torch.autograd.grad(got.loss, x)[0], grad, off, "gradient", x.dtype)


@gpu
def test_two_backward_passes_at_once(by):
    """Of one graph, by two threads: both gradients are whole, and neither is the other's memory."""
    import threading
    r = Rows(64, 9000, "f32", "none", 1.0, 23)
    x, _ = r.on_gpu()
    x.requires_grad_()
    for i in range(3):
        want, = torch.autograd.grad(three(x)[i].loss, x)
        for _ in range(5):
            got, out = three(x)[i], [None, None]
            torch.cuda.synchronize()

            def run(k):
                out[k], = torch.autograd.grad(got.loss, x, retain_graph=True)

            threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
            for th in threads:
                th.start()
            for th in threads:
                th.join()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want) and torch.equal(out[1], want) and out[0].data_ptr() != out[1].data_ptr()


@gpu
def test_no_rows():
    x = torch.empty((0, 40), device="cuda", requires_grad=True)
    e = torch.empty((0,), device="cuda")
    i = torch.empty((0,), dtype=torch.int64, device="cuda")
    for got in (zf.distill_loss(x, i.view(0, 1).expand(0, 3).contiguous(), e.view(0, 1).expand(0, 3).contiguous()), zf.policy_loss(x, i, e, e, entropy_weight=1.0), zf.preference_loss(x, i, torch.zeros(1, dtype=torch.int64, device="cuda")),
                zf.preference_loss(x, i, torch.zeros(3, dtype=torch.int64, device="cuda"))):
        assert got.loss.item() == (0.0 if got.losses.numel() == 0 else got.losses.item())
        assert torch.autograd.grad(got.loss, x)[0].shape == (0, 40)


@gpu
def test_one_row_with_a_weight():
    """The sum of a single row's call is made by the row itself."""
    for t in (3, -1):
        x = torch.randn((1, 50), generator=torch.Generator().manual_seed(2)).cuda()
        w, one = torch.tensor([0.37], device="cuda"), torch.ones((1,), device="cuda")
        for got in (zf.policy_loss(x, torch.tensor([t], device="cuda"), one, one, entropy_weight=0.3, weight=w), zf.distill_loss(x, torch.tensor([[t, 4]], device="cuda") if t > 0 else torch.tensor([[-1, -1]], device="cuda"), torch.zeros((1, 2), device="cuda"), weight=w)):
            assert float(got.loss) == float(torch.tensor(float(w.double()[0] * got.losses.double()[0]), dtype=torch.float64).float()) and (t > 0) == (float(got.loss) != 0)


@gpu
def test_rows_far_apart():
    """Rows 2^30 elements apart: the third begins beyond what 31 bits count."""
    r = Rows(3, 5000, "bf16", "share", 1.0, 9)
    t, zeros = r.tokens(8, padding=0.0), torch.zeros(3)
    x, m = r.on_gpu("far")
    near = r.x.cuda().requires_grad_()
    x.requires_grad_()
    for a, b in zip(three(x, m), three(near, m)):
        assert all(torch.equal(p, q) or torch.isnan(p).any() for p, q in zip(a, b))
        assert torch.equal(torch.autograd.grad(a.loss, x)[0].nan_to_num(), torch.autograd.grad(b.loss, near)[0].nan_to_num())


@gpu
@pytest.mark.parametrize("loss", ["policy", "entropy", "distill", "rest"])
@pytest.mark.parametrize("dtype,rows,V", [("bf16", 64, 32000), ("f32", 48, 32000), ("f32", 300, 7700), ("bf16", 24, 123680), ("f32", 16, 78224)])
def test_a_last_piece_that_several_wavefronts_write(dtype, rows, V, loss, by):
    """A row's last 16 bytes are written by the wavefront that has them and, once more, by those that have no pieces left.  Where none of their tokens is allowed all write the same zero, of the sign that
    other forbidden tokens of the row have: the bits are the same every time.  (Zeros are negative here: the factor of the tokens that were not drawn is.)"""
    r = Rows(rows, V, dtype, "none", 1.0, rows + V)
    r.bits = torch.ones((rows, V), dtype=torch.bool)
    r.bits[:, V - 16:] = False                     # the last pieces, and one among others
    r.bits[:, 4000:4008] = False
    x, m = rows_of(r.x, "packed"), packed(r.bits, padding=True).cuda()
    x.requires_grad_()
    t, zeros = torch.full((rows,), 7, device="cuda"), torch.zeros((rows,), device="cuda")
    weight = zeros - 1.0
    ids, v = torch.tensor([[7, 4001]], device="cuda").expand(rows, 2).contiguous(), torch.tensor([[-3.0, -1.0]], device="cuda").expand(rows, 2).contiguous()

    def gradient(factor):
        if loss in ("policy", "entropy"):
            got = zf.policy_loss(x, t, zeros - 9.0, zeros + 1.0, m, clip=(0.2, INF), entropy_weight=-0.01 if loss == "entropy" else None, weight=weight)
        else:                                      # (of the rest the share that the teacher leaves is the smaller one: its tokens' factor has the sign of the others')
            got = zf.distill_loss(x, ids, torch.cat([v[:, :1] + 2.9, v[:, 1:]], dim=1) if loss == "rest" else v, m, rest=loss == "rest", weight=weight)
        return torch.autograd.grad(got.loss * factor, x)[0]

    bits = lambda g: g.view(torch.int32 if dtype == "f32" else torch.int16)
    for factor in (1.0, 2.0):
        first = gradient(factor)
        forbidden = first[~r.bits.cuda()]
        assert (forbidden == 0).all() and torch.signbit(forbidden).all()
        for _ in range(3):
            assert torch.equal(bits(gradient(factor)), bits(first))


# ---- autograd, streams, graphs ----------------------------------------------------------------------
def same_twice(x, mask):
    return [lambda i=i: three(x, mask)[i] for i in range(4)]


@gpu
@pytest.mark.parametrize("V", [900, 40037])
def test_gradients_of_any_factor_and_twice(V, by):
    """A factor other than one; a second backward pass, with another factor, leaves what the first gave; a gradient that was written is not given again."""
    r = Rows(5, V, "f32", "share", 1.0, 10)
    r.bits[:, 1:3] = True
    r.update()
    x, m = r.on_gpu()
    x.requires_grad_()
    for make in same_twice(x, m):
        one, = torch.autograd.grad(make().loss, x)
        got = make()
        three_times, = torch.autograd.grad(got.loss * 3.0, x, retain_graph=True)
        # Not relative to the gradient: an element is e (base + slope y) or e a + f, each factor and each step of either side rounded once (8 in all), and the terms may cancel.
        # They are at most p (2 + 0.1 (|ln p| + H)), and 1.2 for a listed token.
        size = r.p * (2 + 0.1 * (torch.where(r.allowed, r.lp.abs(), 0.0) + r.H[:, None]))
        size[:, 1:3] += 1.2
        assert ((three_times - 3 * one).abs().cpu().double() <= 8 * U * 3 * size).all()
        three_times.zero_()
        again, = torch.autograd.grad(got.loss, x, retain_graph=True)
        assert torch.equal(again, one) and again.data_ptr() != three_times.data_ptr()
        again.zero_()
        zero, = torch.autograd.grad(got.loss * 0.0, x, retain_graph=True)
        assert (zero == 0).all()
        assert torch.equal(torch.autograd.grad(got.loss, x)[0], one)


@gpu
def test_gradients_against_differences():
    """(L(x + h) - L(x - h)) / 2 h for each of a row's logits: off by h^2 / 6 times the third derivative (4 at most for these losses of weight one and temperature one) and the
    losses' own rounding, some 30 u of their size, over h."""
    g = torch.Generator().manual_seed(11)
    V, h = 24, 2.0 ** -6
    x = torch.randn((4, V), generator=g)
    steps = torch.cat([torch.eye(V), -torch.eye(V)]) * h
    base = x.cuda().requires_grad_()
    for i in range(4):
        d = torch.autograd.grad(three(base)[i].loss, base)[0].cpu()
        for row in range(4):
            losses = []
            for s in steps:
                y = x.clone()
                y[row] += s
                losses.append(float(three(y.cuda())[i].loss))
            losses = torch.tensor(losses, dtype=torch.float64)
            want = (losses[:V] - losses[V:]) / (2 * h)
            assert (d[row].double() - want).abs().max() < h * h / 6 * 4 * 4 + 30 * U * (1 + losses.abs().max()) / h


@gpu
def test_module_and_definition_agree(monkeypatch):
    """The same bits, with and without a gradient, of every argument."""
    from paper_2506_01151_amd import losses
    r = Rows(9, 3001, "bf16", "share", 1.0, 18)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu("odd")
    x.requires_grad_()
    t, zeros, ids, v, half = beside(x)
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b, w = (torch.rand(9, generator=g, device="cuda") for _ in range(3))
    calls = [lambda: zf.distill_loss(x, ids.int(), v.bfloat16(), m, temperature=0.7, rest=True, weight=w), lambda: zf.distill_loss(x, ids, v, temperature=2),
             lambda: zf.policy_loss(x, t, a - 8, b, m, ref_logprobs=w - 8, temperature=1.3, clip=(0.1, 0.4), kl_weight=0.3, entropy_weight=0.2, weight=w), lambda: zf.policy_loss(x, t.int(), a - 8, b, clip=[0, 1]),
             lambda: zf.preference_loss(x, t, half.int(), a - 8, m, beta=0.3, label_smoothing=0.1, average=True, temperature=0.9, weight=w[:1]), lambda: zf.preference_loss(x, t, half)]

    def results():
        out = []
        for call in calls:
            got = call()
            with torch.no_grad():
                alone = call()
            assert type(got) is type(alone) and [y is None for y in got] == [y is None for y in alone]
            assert got.loss.requires_grad and not any(y.requires_grad for y in got[1:] if y is not None) and not alone.loss.requires_grad
            out += [y.detach() for y in (*got, *alone) if y is not None] + list(torch.autograd.grad(got.loss, x, torch.tensor(0.7, device="cuda")))
        return out

    mine = results()

    class Nothing:
        distill_loss = policy_loss = preference_loss = staticmethod(lambda *args: None)

    monkeypatch.setattr(losses, "_native_losses", Nothing)
    theirs = results()
    assert len(mine) == len(theirs) and all(torch.equal(p, q) and p.dtype == q.dtype and p.stride() == q.stride() for p, q in zip(mine, theirs))


@gpu
def test_results_are_the_same_every_time():
    r = Rows(300, 20000, "bf16", "share", 1.0, 12)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu()
    x.requires_grad_()
    for make in same_twice(x, m):
        a, b = make(), make()
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        assert torch.equal(torch.autograd.grad(a.loss, x)[0], torch.autograd.grad(b.loss, x)[0])


@gpu
def test_what_was_written_since_raises(by):
    r = Rows(6, 1000, "f32", "share", 1.0, 13)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu()
    leaf = x.clone().requires_grad_()
    for i in range(4):
        y = leaf * 1.0
        got = three(y, m)[i]
        y.add_(1.0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            got.loss.backward()
        got = three(leaf, m)[i]
        m.add_(0)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            got.loss.backward()


@gpu
def test_hooks_on_saved_tensors(by):
    """What they give back may lie elsewhere, in another layout: the gradient is the same; another shape is refused."""
    r = Rows(6, 1003, "bf16", "share", 1.0, 14)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu()
    x.requires_grad_()
    for i in range(4):
        want, = torch.autograd.grad(three(x, m)[i].loss * 2.0, x)
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach().cpu(), lambda t: t.cuda()):
            got = three(x, m)[i]
        assert torch.equal(torch.autograd.grad(got.loss * 2.0, x)[0], want)
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach().clone(), lambda t: t.t().contiguous().t() if t.dim() == 2 else t):
            got = three(x, m)[i]
        assert torch.equal(torch.autograd.grad(got.loss * 2.0, x)[0], want)
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach().clone(), lambda t: t[:-1] if t.dim() else t):
            got = three(x, m)[i]
        with pytest.raises(RuntimeError):
            torch.autograd.grad(got.loss * 2.0, x)


@gpu
def test_on_another_stream_and_differentiated_once(by):
    r = Rows(6, 1000, "f32", "share", 1.0, 15)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu()
    x.requires_grad_()
    want = [torch.autograd.grad(three(x, m)[i].loss, x)[0] for i in range(4)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [torch.autograd.grad(three(x, m)[i].loss, x)[0] for i in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for i in range(4):
        d, = torch.autograd.grad(three(x, m)[i].loss, x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(d.sum(), x)


@gpu
def test_captured_into_a_graph(by):
    """Losses and gradients replayed with other logits and other factors, eager work between the replays."""
    r = Rows(40, 5000, "f32", "share", 1.0, 16)
    r.bits[:, 1:3] = True
    x, m = r.on_gpu()
    others = [torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda") for i in range(3)]
    for i in range(4):
        s = torch.cuda.Stream()
        leaf, factor, needs = x.clone().requires_grad_(), torch.ones((), device="cuda"), beside(x)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            torch.autograd.grad(three(leaf, m, needs)[i].loss, leaf, factor)      # what the losses load, once
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = three(leaf, m, needs)[i]
            grad, = torch.autograd.grad(got.loss, leaf, factor)
            kept = got.loss.detach()
        for y, f in zip(others, (1.0, 3.0, 1.0)):
            with torch.no_grad():
                leaf.copy_(y)
                factor.fill_(f)
            for _ in range(2):
                graph.replay()
                torch.cuda.synchronize()
                own = y.clone().requires_grad_()
                want = three(own, m)[i]
                assert torch.equal(kept, want.loss.detach())
                assert torch.equal(grad, torch.autograd.grad(want.loss, own, torch.tensor(f, device="cuda"))[0])


@gpu
def test_a_backward_pass_alone_in_a_graph(by):
    """Made eagerly, followed back in a capture: each replay gives the gradient by the factor of its time."""
    r = Rows(7, 3000, "f32", "none", 1.0, 17)
    x, _ = r.on_gpu()
    for i in range(4):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        leaf, factor = x.clone().requires_grad_(), torch.ones((), device="cuda")
        want = [f * torch.autograd.grad(three(leaf)[i].loss, leaf)[0] for f in (2.0, 1.0, 0.5)]
        with torch.cuda.stream(s):
            got = three(leaf)[i]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            grad, = torch.autograd.grad(got.loss, leaf, factor, retain_graph=True)
        for f, w in zip((2.0, 1.0, 0.5), want):
            factor.fill_(f)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(grad, w)


# ---- refusals ---------------------------------------------------------------------------------------
def refused(call, *words):
    with pytest.raises(zf.ZfError) as e:
        call()
    assert e.value.code == zf.ZF_ERR_INVALID_ARG and all(w in str(e.value) for w in words), e.value


def test_refusals_on_the_host():
    """Tensors that are not on the GPU, and the C boundary's own checks (before anything is read: the addresses are none)."""
    x = torch.zeros((2, 8))
    refused(lambda: zf.distill_loss(x, torch.zeros((2, 1), dtype=torch.int64), torch.zeros((2, 1))), "logits")
    refused(lambda: zf.policy_loss(x, torch.zeros(2, dtype=torch.int64), torch.zeros(2), torch.zeros(2)), "logits")
    refused(lambda: zf.preference_loss(x, torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int64)), "logits")
    from paper_2506_01151_amd.binding import DistillArgs, PolicyArgs, PreferenceArgs
    L, at = zf.load_library(), 4096
    rows = dict(logits=at, dtype=0, V=10, rows=3, row_stride=10, temperature=1.0, loss=at, losses=at)
    mine = {DistillArgs: dict(ids=at, values=at, id_bytes=4, values_dtype=0, n_listed=2), PolicyArgs: dict(tokens=at, old_logprobs=at, advantages=at, token_bytes=8, clip_low=0.2, clip_high=0.2, logprobs=at),
            PreferenceArgs: dict(tokens=at, offsets=at, token_bytes=4, offset_bytes=8, pairs=1, beta=0.1, label_smoothing=0.0, chosen=at, rejected=at, stats=at, slopes=at)}
    calls = {DistillArgs: (L.zf_distill_loss, L.zf_distill_loss_backward), PolicyArgs: (L.zf_policy_loss, L.zf_policy_loss_backward), PreferenceArgs: (L.zf_preference_loss, L.zf_preference_loss_backward)}

    def code(kind, changed, back=False, grad=at + 64, stride=10, g=at):
        a = kind()
        for n, v in {**rows, **{k: v for k, v in changed.items() if k in rows or k == "mask"}}.items():
            setattr(a.r, n, v)
        for n, v in {**mine[kind], **{k: v for k, v in changed.items() if k in mine[kind]}}.items():
            setattr(a, n, v)
        call, call_back = calls[kind]
        if kind is PreferenceArgs:
            return call_back(ctypes.byref(a), g, grad, stride, 0, None) if back else call(ctypes.byref(a), 0, None)
        return call_back(ctypes.byref(a), g, 0, grad, stride, 0, None) if back else call(ctypes.byref(a), grad, stride, 0, None)

    for kind in mine:
        common = [dict(dtype=2), dict(V=0), dict(V=(1 << 24) + 1, row_stride=1 << 25), dict(rows=-1), dict(rows=1 << 31), dict(row_stride=9), dict(temperature=0.0), dict(temperature=math.nan), dict(temperature=INF),
                  dict(temperature=1e-39), dict(temperature=1e39), dict(loss=None), dict(losses=None), dict(logits=None), dict(logits=at + 2)]
        own = {DistillArgs: [dict(n_listed=0), dict(n_listed=1025), dict(id_bytes=2), dict(values_dtype=3), dict(ids=None), dict(values=None)],
               PolicyArgs: [dict(token_bytes=1), dict(clip_low=-0.1), dict(clip_high=math.nan), dict(tokens=None), dict(old_logprobs=None), dict(advantages=None), dict(logprobs=None)],
               PreferenceArgs: [dict(token_bytes=0), dict(offset_bytes=3), dict(pairs=-1), dict(pairs=1 << 30), dict(beta=INF), dict(label_smoothing=1.1), dict(label_smoothing=math.nan), dict(tokens=None), dict(offsets=None),
                                dict(chosen=None), dict(rejected=None), dict(stats=None), dict(stats=at + 8), dict(slopes=None), dict(rows=1 << 20, V=1 << 24, row_stride=1 << 24)]}[kind]
        for changed in common + own:
            assert code(kind, changed) == zf.ZF_ERR_INVALID_ARG, (kind, changed)
            assert code(kind, changed, back=True) == zf.ZF_ERR_INVALID_ARG, (kind, changed)
        for more in (dict(grad=at), dict(grad=at + 2), dict(stride=9), dict(grad=None), dict(g=None)):
            assert code(kind, {}, back=True, **more) == zf.ZF_ERR_INVALID_ARG, (kind, more)
    assert L.zf_distill_loss(None, None, 0, 0, None) == L.zf_policy_loss(None, None, 0, 0, None) == L.zf_preference_loss(None, 0, None) == zf.ZF_ERR_INVALID_ARG


@gpu
def test_refusals(by):
    x = torch.zeros((4, 40), device="cuda", requires_grad=True)
    t, f = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    ids, v, o = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda"), torch.tensor([0, 2, 4], device="cuda")
    for bad in (x[:, ::2], x.double(), x[0], x.cpu(), torch.zeros((4, 0), device="cuda"), None):
        refused(lambda: zf.distill_loss(bad, ids, v))
        refused(lambda: zf.policy_loss(bad, t, f, f))
        refused(lambda: zf.preference_loss(bad, t, o))
    for bad in (t[:3], t.cpu(), f, t[:, None], torch.zeros(8, dtype=torch.int64, device="cuda")[::2], None):
        refused(lambda: zf.policy_loss(x, bad, f, f), "tokens")
        refused(lambda: zf.preference_loss(x, bad, o), "tokens")
    for bad in (f[:3], f.cpu(), f.double(), f[:, None], f.expand(2, 4), torch.zeros((), device="cuda").expand(4), f.clone().requires_grad_(), torch._neg_view(f)):
        refused(lambda: zf.policy_loss(x, t, bad, f), "old_logprobs")
        refused(lambda: zf.policy_loss(x, t, f, bad), "advantages")
        refused(lambda: zf.policy_loss(x, t, f, f, ref_logprobs=bad), "ref_logprobs")
        refused(lambda: zf.policy_loss(x, t, f, f, weight=bad), "weight")
        refused(lambda: zf.preference_loss(x, t, o, bad), "ref_logprobs")
        refused(lambda: zf.distill_loss(x, ids, v, weight=bad), "weight")
    refused(lambda: zf.policy_loss(x, t, None, f), "old_logprobs")
    refused(lambda: zf.policy_loss(x, t, f, f, kl_weight=0.1), "kl_weight")
    for clip in ((0.2,), (-0.1, 0.2), (0.1, math.nan), 0.2, ("a", 0.1)):
        refused(lambda: zf.policy_loss(x, t, f, f, clip=clip), "clip")
    for bad in (math.nan, INF, "1"):
        refused(lambda: zf.policy_loss(x, t, f, f, entropy_weight=bad), "entropy_weight")
        refused(lambda: zf.preference_loss(x, t, o, beta=bad), "beta")
    for bad in (0.0, -1.0, math.nan, INF, 2.0 ** -127, "1"):
        refused(lambda: zf.distill_loss(x, ids, v, temperature=bad), "temperature")
    refused(lambda: zf.preference_loss(x, t, o[:2]), "offsets")
    refused(lambda: zf.preference_loss(x, t, o.float()), "offsets")
    refused(lambda: zf.preference_loss(x, t, o, label_smoothing=1.5), "label_smoothing")
    refused(lambda: zf.preference_loss(x, t, o, weight=torch.zeros(2, device="cuda")), "weight")
    for bad in (ids[:, 0], ids.float(), ids[:3], ids.cpu(), torch.zeros((4, 0), dtype=torch.int32, device="cuda"), torch.zeros((4, 1025), dtype=torch.int32, device="cuda"), ids.t().contiguous().t()):
        refused(lambda: zf.distill_loss(x, bad, v), "teacher_ids")
    for bad in (v[:, :1], v.double(), v.clone().requires_grad_()):
        refused(lambda: zf.distill_loss(x, ids, bad), "teacher_values")
    for bad in (torch.zeros((4, 1), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda"), torch.zeros((4, 4), dtype=torch.int32, device="cuda")[:, ::2]):
        refused(lambda: zf.policy_loss(x, t, f, f, bad), "mask")
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x.detach(), torch.ones_like(x))
        refused(lambda: zf.policy_loss(dual, t, f, f), "forward-mode")
    refused(lambda: torch.func.grad(lambda y: zf.policy_loss(y, t, f, f).loss)(x.detach()))
    refused(lambda: torch.jit.trace(lambda y: zf.policy_loss(y, t, f, f).loss, (x.detach(),)), "traced")


# ---- together ---------------------------------------------------------------------------------------
@gpu
def test_a_learner_with_all_three(by):
    """Sequences decoded under a grammar; their policy's loss, distillation from a teacher that reports as a server does, and a preference between them, on one batch of logits."""
    from examples import decode_and_train as ex
    from workloads import configs
    cfg = configs.CONFIGS[2]
    engine = zf.Engine(cfg.grammar(), cfg.vocab())
    student, other = ex.Model(engine.V, 256, "cuda:0"), ex.Model(engine.V, 256, "cuda:0", seed=5)
    steps = ex.decode(engine, student, batch=4, steps=6)
    order = [s * 4 + r for r in range(4) for s in range(6)]        # rows of a sequence one behind the other
    hidden, mask, tokens = (torch.cat([s[i] for s in steps])[order].contiguous() for i in range(3))
    old = torch.cat([s[3].logprobs for s in steps])[order].contiguous()
    head = student.head.clone().requires_grad_()
    teacher_says = zf.token_logprobs(hidden @ other.head.t(), tokens, mask, top=20)
    logits = hidden @ head.t()
    weight = torch.full((24,), 1 / 24, device="cuda")
    advantages = torch.linspace(-1, 1, 24, device="cuda")
    policy = zf.policy_loss(logits, tokens, old, advantages, mask, ref_logprobs=teacher_says.logprobs, temperature=0.8, kl_weight=0.1, entropy_weight=0.01, weight=weight)
    distill = zf.distill_loss(logits, teacher_says.top_ids, teacher_says.top_logprobs, mask, rest=True, weight=weight)
    preference = zf.preference_loss(logits, tokens, torch.arange(0, 25, 6, device="cuda"), teacher_says.logprobs, mask)
    got, = torch.autograd.grad(policy.loss + distill.loss + 0.5 * preference.loss, head, retain_graph=True)
    # the same from log probabilities, whose own tests are elsewhere, and torch's arithmetic
    lp = zf.token_logprobs(logits, tokens, mask, temperature=0.8, entropy=True)
    ratio = torch.exp(lp.logprobs - old)
    drawn = tokens >= 0
    back = teacher_says.logprobs - lp.logprobs
    a = -torch.minimum(ratio * advantages, ratio.clamp(0.8, 1.2) * advantages) + 0.1 * (torch.exp(back) - back - 1) - 0.01 * lp.entropy
    a = torch.where(drawn, a, 0.0).sum() / 24
    ids = teacher_says.top_ids.long()
    full = torch.log_softmax(torch.where(((mask.unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).bool().view(24, -1)[:, :engine.V], logits.double(), -1e30), dim=1)
    there = ids >= 0
    q = torch.where(there, torch.exp(teacher_says.top_logprobs.double()), 0.0)
    p = torch.where(there, torch.exp(full.gather(1, ids.clamp(min=0))), 0.0)
    outside = torch.ones_like(full).scatter(1, torch.where(there, ids, ids[:, :1].clamp(min=0)), 0.0)
    p_rest, q_rest = (torch.exp(full) * outside).sum(dim=1), (1 - q.sum(dim=1)).clamp(min=0)
    use = there.any(dim=1) & (p_rest > 0) & (q_rest > 0)
    b = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - full.gather(1, ids.clamp(min=0))), 0.0).sum(dim=1)
    b = b + torch.where(use, q_rest * (torch.log(q_rest.clamp(min=1e-300)) - torch.log(p_rest.clamp(min=1e-300))), 0.0)
    lp1 = zf.token_logprobs(logits, tokens, mask).logprobs
    D = torch.where(drawn, lp1 - teacher_says.logprobs, 0.0).view(4, 6).sum(dim=1)
    c = -torch.nn.functional.logsigmoid(0.1 * (D[0::2] - D[1::2])).sum()
    want, = torch.autograd.grad(a + (b.sum() / 24).float() + 0.5 * c, head)
    assert abs(float(policy.loss - a)) < 1e-5 and abs(float(distill.loss - b.sum() / 24)) < 1e-5 and abs(float(preference.loss - c)) < 1e-5
    assert (got - want).norm() < 1e-5 * want.norm()
