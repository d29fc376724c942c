"""What is timed of the losses that a learner takes on logits under masks, each with the gradient of the logits.

A case is one of
  distill     distillation from a teacher's top logits: the divergence of the student's distribution from the teacher's, over the listed tokens alone or
              with all others as one more outcome
  policy      the clipped loss of a policy's probability ratios, with a penalty on the divergence from a reference and a bonus for entropy
  preference  paired log ratios of packed sequences against a reference
`grad`: a step of training, or the losses alone, as in an evaluation.  Vocabularies are those of workloads/configs.py or generic, rows are the positions of
a learner's batch.  `own` says who computes: elementary torch operations in 32 bits, or this package.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
LIKELY = 40                                        # tokens of a row that stand out from the others
CLIP = (0.2, 0.28)
KL, ENTROPY, BETA = 0.05, 0.01, 0.1


def listed():
    return [
        # latency alone: one position at the smallest vocabulary, a short list
        distill("distill_v2k_b1", 1, 2048, "f32", "none", 5, False),
        # a small batch of constrained sequences, whose teacher reported what a server reports
        distill("distill_v32k_b300_rest", 300, 32000, "f32", "share", 20, True),
        # an evaluation against a softened teacher, odd sizes
        distill("distill_v40037_b1030_eval", 1030, 40037, "bf16", "none", 64, False, 2.0, grad=False),
        # a large step
        distill("distill_v128k_b4096_rest", 4096, 128256, "bf16", "none", 64, True),
        # one short sequence, constrained
        policy("policy_v32k_b16", 16, 32000, "f32", "share", True, True),
        # odd sizes, the ratios' loss alone
        policy("policy_v40037_b1030", 1030, 40037, "bf16", "none", False, False),
        # the largest vocabulary, a grammar that leaves a few hundred tokens
        policy("policy_v152k_b1024_few", 1024, 152064, "f32", "few", True, True, 300),
        # a large step on constrained sequences
        policy("policy_v128k_b4096", 4096, 128256, "bf16", "share", True, False),
        # one pair of short answers: latency
        preference("preference_v2k_p1", 24, 2048, "f32", "none", 1),
        # a small batch under masks
        preference("preference_v32k_p8", 1000, 32000, "f32", "share", 8),
        # a large step; answers of different lengths behind prompts, their means compared
        preference("preference_v128k_p8", 4096, 128256, "bf16", "none", 8, True, 0.1),
        # an evaluation
        preference("preference_v152k_p3_eval", 501, 152064, "f32", "none", 3, grad=False),
    ]


def distill(name, rows, V, dtype, mask, K, rest, temperature=1.0, allowed=0, grad=True):
    c = {"op": "distill", "rows": rows, "V": V, "dtype": dtype, "mask": mask, "allowed": allowed, "K": K, "rest": rest, "temperature": temperature, "ignored": 0.05, "grad": grad}
    return dict(c, name=name) if name else c


def policy(name, rows, V, dtype, mask, kl, entropy, allowed=0, temperature=1.0, grad=True):
    c = {"op": "policy", "rows": rows, "V": V, "dtype": dtype, "mask": mask, "allowed": allowed, "kl": kl, "entropy": entropy, "temperature": temperature, "ignored": 0.05, "grad": grad}
    return dict(c, name=name) if name else c


def preference(name, rows, V, dtype, mask, pairs, average=False, smoothing=0.0, allowed=0, grad=True):
    c = {"op": "preference", "rows": rows, "V": V, "dtype": dtype, "mask": mask, "allowed": allowed, "pairs": pairs, "average": average, "smoothing": smoothing, "temperature": 1.0,
         "ignored": 0.25, "grad": grad}
    return dict(c, name=name) if name else c


def between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    V, dtype, mask = between(rng, 2048, 152064), rng.choice(("f32", "bf16")), rng.choice(("none", "few", "share"))
    if rng.random() < 0.5:
        V = V // 64 * 64                           # half of the vocabularies are padded to a round size, the others are what they are
    most = 2 ** 30 // (V * SIZE[dtype])
    rows, allowed, grad = min(between(rng, 1, 4096), most), between(rng, 1, 2000) if mask == "few" else 0, rng.random() < 0.8
    op = rng.choice(("distill", "policy", "preference"))
    if op == "distill":
        return distill(None, rows, V, dtype, mask, rng.choice((1, 5, 20, 64, 200)), rng.random() < 0.5, rng.choice((1.0, 1.0, 2.0)), allowed, grad)
    if op == "policy":
        return policy(None, rows, V, dtype, mask, rng.random() < 0.5, rng.random() < 0.5, allowed, rng.choice((1.0, 1.0, 0.7)), grad)
    rows = min(max(rows, 8), most)
    return preference(None, rows, V, dtype, mask, min(between(rng, 1, 64), max(1, rows // 8)), rng.random() < 0.3, rng.choice((0.0, 0.0, 0.1)), allowed, grad)


# ---- inputs --------------------------------------------------------------------------------------
def mask_of(case, gen):
    """Packed masks, bit v % 32 of word v / 32, as the mask kernels write them; one row of sixteen or more is over and allows nothing."""
    if case["mask"] == "none":
        return None
    B, V = case["rows"], case["V"]
    W = (V + 31) // 32
    share = torch.rand((B, 1), generator=gen, device="cuda") ** 3 if case["mask"] == "share" else min(1.0, case["allowed"] / V)
    bits = torch.rand((B, W * 32), generator=gen, device="cuda") < share
    bits[:, V:] = False
    bits[torch.arange(B, device="cuda"), torch.randint(V, (B,), generator=gen, device="cuda")] = True
    if B >= 16:
        bits[B // 2] = False
    words = (bits.view(B, W, 32).int() << torch.arange(32, dtype=torch.int32, device="cuda")).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def normal(gen, *shape, sigma=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, V, T = case["rows"], case["V"], case["temperature"]
    x = normal(gen, B, V, sigma=2.0)
    stripe = V // LIKELY
    likely = torch.randint(stripe, (B, LIKELY), generator=gen, device="cuda") + stripe * torch.arange(LIKELY, device="cuda")
    x.scatter_(1, likely, 8.0 + 10.0 * torch.rand((B, LIKELY), generator=gen, device="cuda"))
    x = x.to(DTYPES[case["dtype"]])
    mask = mask_of(case, gen)
    state = {"case": case, "x": x, "mask": mask}
    ignored = torch.randperm(B, generator=gen, device="cuda")[:int(B * case["ignored"])]       # where a shorter sequence is padded
    if case["op"] == "distill":
        # a teacher's report: its most probable tokens with their log probabilities, -1 behind the last one that there is
        t = 0.9 * x.float() + normal(gen, B, V, sigma=0.5)
        if mask is not None:
            t = torch.where(allowed_of(mask, V), t, -math.inf)
        best, ids = torch.topk(t, min(case["K"], V), dim=1)
        there = best > -math.inf
        there[ignored] = False
        lp = best / T - torch.logsumexp(t / T, dim=1, keepdim=True)
        state["ids"] = torch.where(there, ids, -1).to(torch.int32)
        state["values"] = torch.where(there, lp if case["rest"] else best, -math.inf)
        state["weight"] = torch.full((B,), 1.0 / B, device="cuda")
    else:
        z = x.float() / T
        if mask is not None:
            z = torch.where(allowed_of(mask, V), z, -math.inf)
        noise = torch.empty_like(z).exponential_(generator=gen)
        tokens = (torch.softmax(z, dim=1) / noise).nan_to_num_(0.0).argmax(dim=1)              # drawn under the masks
        lp = (z.gather(1, tokens[:, None]).squeeze(1) - torch.logsumexp(z, dim=1)).nan_to_num_(0.0, neginf=0.0)
        over = (z == -math.inf).all(dim=1)                                                     # a sequence that had ended
        state["ref"] = lp + normal(gen, B, sigma=0.3)
        if case["op"] == "policy":
            tokens[ignored] = -1
            tokens[over] = -1
            state["old"] = lp + normal(gen, B, sigma=0.15)
            state["advantages"] = normal(gen, B)
            state["weight"] = torch.full((B,), 1.0 / B, device="cuda")
        else:
            # sequences of different lengths, the first part of each a prompt; a few rows behind the last one belong to none
            S = 2 * case["pairs"]
            cut = torch.rand((S,), generator=gen, device="cuda", dtype=torch.float64) + 0.3
            ends = (torch.cumsum(cut, 0) / cut.sum() * (B - B // 50)).long()
            offsets = torch.cat([ends.new_zeros(1), ends])
            row = torch.arange(B, device="cuda")
            s = torch.searchsorted(ends, row, right=True).clamp(max=S - 1)
            begin, length = offsets[s], offsets[s + 1] - offsets[s]
            tokens[(row - begin) < (length * case["ignored"]).long()] = -1
            tokens[over] = -1
            state["offsets"] = offsets.to(torch.int32)
            state["weight"] = torch.full((case["pairs"],), 1.0 / case["pairs"], device="cuda")
        state["tokens"] = tokens
    if case["grad"]:
        x.requires_grad_()
    return state


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if not own:
        return PLAIN[case["op"]](state)
    import paper_2506_01151_amd as zf
    x, T = state["x"], case["temperature"]
    if case["op"] == "distill":
        got = zf.distill_loss(x, state["ids"], state["values"], state["mask"], temperature=T, rest=case["rest"], weight=state["weight"])
        out = {"losses": got.losses}
    elif case["op"] == "policy":
        got = zf.policy_loss(x, state["tokens"], state["old"], state["advantages"], state["mask"], ref_logprobs=state["ref"] if case["kl"] else None, temperature=T, clip=CLIP,
                             kl_weight=KL if case["kl"] else 0.0, entropy_weight=ENTROPY if case["entropy"] else None, weight=state["weight"])
        out = {"losses": got.losses, "logprobs": got.logprobs, "entropy": got.entropy}
    else:
        got = zf.preference_loss(x, state["tokens"], state["offsets"], state["ref"], state["mask"], beta=BETA, label_smoothing=case["smoothing"], average=case["average"], temperature=T,
                                 weight=state["weight"])
        out = {"losses": got.losses, "chosen": got.chosen, "rejected": got.rejected}
    if case["grad"]:
        out["grad"], = torch.autograd.grad(got.loss, x)
    return dict(out, loss=got.loss.detach())


def allowed_of(mask, V):
    return ((mask.unsqueeze(-1) >> torch.arange(32, dtype=torch.int32, device=mask.device)) & 1).bool().view(mask.shape[0], -1)[:, :V]


def plain_softmax(state):
    """Whether a token is allowed, log probabilities, probabilities; zeros and -inf in rows that have nothing."""
    case = state["case"]
    x = state["x"].detach().float()
    if state["mask"] is not None:
        x = torch.where(allowed_of(state["mask"], case["V"]), x, -math.inf)
    most = x.amax(dim=1, keepdim=True)
    some = most > -math.inf
    z = torch.where(some, x - most, -math.inf) / case["temperature"]
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    lp = torch.where(some, z - torch.log(total.double()).float(), -math.inf)
    p = torch.where(some, e / total, 0.0)
    return x > -math.inf, lp, p


def total(weight, losses):
    return (weight.double() * losses.double()).sum().float()


def plain_distill(state):
    case, ids, w = state["case"], state["ids"].long(), state["weight"]
    allowed, lp, p = plain_softmax(state)
    at = ids.clamp(min=0)
    use = (ids >= 0) & allowed.gather(1, at)
    lp_k = lp.gather(1, at)
    t = torch.where(use, state["values"].double(), -math.inf)      # what is left of one, and small shares of it, in 64 bits
    if case["rest"]:
        q = torch.exp(t)
        q_rest = (1.0 - q.sum(dim=1)).clamp(min=0.0)
    else:
        t = t / case["temperature"]
        most = t.amax(dim=1, keepdim=True)
        e = torch.where(most > -math.inf, torch.exp(t - most), 0.0)
        t = t - most - torch.log(e.sum(dim=1, keepdim=True))
        q = torch.where(most > -math.inf, torch.exp(t), 0.0)
    losses = torch.where(q > 0, q * (t - lp_k.double()), 0.0).sum(dim=1)
    f = -torch.where(use, q, 0.0).float()
    total_f = f.sum(dim=1, keepdim=True)
    grad = -total_f * p
    if case["rest"]:
        inside = torch.zeros(p.shape, dtype=torch.int32, device=p.device).scatter_add_(1, at, use.int()) > 0
        p_rest = torch.where(inside, 0.0, p).sum(dim=1).double()
        some = (p_rest > 0) & use.any(dim=1)
        q_rest = torch.where(some, q_rest, 0.0)
        losses = losses + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - torch.log(p_rest)), 0.0)
        f_rest = -q_rest.float()
        grad = grad - f_rest[:, None] * p
        grad = grad + torch.where(inside, 0.0, p * torch.where(some, f_rest / p_rest.float(), 0.0)[:, None])
    out = {"losses": losses.float(), "loss": total(w, losses)}
    if case["grad"]:
        grad.scatter_add_(1, at, f)
        out["grad"] = (grad * w[:, None] / case["temperature"]).to(state["x"].dtype)
    return out


def given(allowed, lp, p, tokens):
    """Of the given tokens: whether a row counts, and the log probability (0 for padding)."""
    at = tokens.clamp(min=0).unsqueeze(1)
    counts = (tokens >= 0) & allowed.gather(1, at).squeeze(1)
    return counts, torch.where(tokens >= 0, lp.gather(1, at).squeeze(1), 0.0)


def grad_of(p, tokens, f, temperature):
    grad = -p * f.unsqueeze(1)
    grad.scatter_add_(1, tokens.clamp(min=0).unsqueeze(1), f.unsqueeze(1))
    return grad / temperature


def plain_policy(state):
    case, tokens, w = state["case"], state["tokens"], state["weight"]
    allowed, lp, p = plain_softmax(state)
    counts, at = given(allowed, lp, p, tokens)
    a, now = state["advantages"].double(), torch.where(counts, at, 0.0).double()
    ratio = torch.exp(now - state["old"].double())                 # next to a border of the clipping, and differences of nearly equal numbers: 64 bits
    kept = ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1])
    losses = -torch.minimum(ratio * a, kept * a)
    f = torch.where(kept * a < ratio * a, 0.0, -ratio * a)
    if case["kl"]:
        d = state["ref"].double() - now
        losses = losses + KL * (torch.exp(d) - d - 1.0)
        f = f + KL * (1.0 - torch.exp(d))
    f = torch.where(counts, f, 0.0).float() * w
    out = {"logprobs": at, "entropy": None}
    if case["entropy"]:
        plogp = torch.where(p > 0, p * lp, 0.0)
        H = torch.where(tokens >= 0, -plogp.sum(dim=1), 0.0)
        out["entropy"] = H
        losses = losses - ENTROPY * H.double()
    losses = torch.where(counts, losses, 0.0)
    out.update(losses=losses.float(), loss=total(w, losses))
    if case["grad"]:
        grad = grad_of(p, tokens, f, case["temperature"])
        if case["entropy"]:
            e = torch.where(counts, ENTROPY * w, 0.0) / case["temperature"]
            grad = grad + e[:, None] * (plogp + p * H[:, None])
        out["grad"] = grad.to(state["x"].dtype)
    return out


def plain_preference(state):
    case, tokens, w, P = state["case"], state["tokens"], state["weight"], state["case"]["pairs"]
    allowed, lp, p = plain_softmax(state)
    counts, at = given(allowed, lp, p, tokens)
    offsets = state["offsets"].long()
    row = torch.arange(case["rows"], device=tokens.device)
    s = torch.searchsorted(offsets[1:], row, right=True)
    s = torch.where(row < offsets[0], 2 * P, s)                    # the rows of no sequence come last
    used = (tokens >= 0) & (s < 2 * P)
    ratio = torch.where(used, at.double() - state["ref"].double(), 0.0)
    sums = torch.zeros(2 * P + 1, dtype=torch.float64, device=tokens.device).index_add_(0, s, ratio)
    n = torch.zeros_like(sums).index_add_(0, s, used.double()).clamp(min=1.0)
    if case["average"]:
        sums = sums / n
    chosen, rejected = BETA * sums[0:2 * P:2], BETA * sums[1:2 * P:2]
    h = chosen - rejected
    eps = case["smoothing"]
    # softplus(y) = max(y, 0) + log1p(exp(-|y|)), -ln sigma(h) = softplus(-h)
    tail = torch.log1p(torch.exp(-h.abs()))
    losses = (1.0 - eps) * ((-h).clamp(min=0.0) + tail) + (eps * (h.clamp(min=0.0) + tail) if eps else 0.0)
    out = {"losses": losses.float(), "chosen": chosen.float(), "rejected": rejected.float(), "loss": total(w, losses)}
    if case["grad"]:
        c = BETA * w.double() * (eps / (1.0 + torch.exp(-h)) - (1.0 - eps) / (1.0 + torch.exp(h)))
        of = torch.zeros_like(sums)
        of[0:2 * P:2], of[1:2 * P:2] = c, -c
        if case["average"]:
            of = of / n
        f = torch.where(used & counts, of[s], 0.0).float()
        out["grad"] = grad_of(p, tokens, f, case["temperature"]).to(state["x"].dtype)
    return out


PLAIN = {"distill": plain_distill, "policy": plain_policy, "preference": plain_preference}


# ---- the same in 64 bits ---------------------------------------------------------------------------
def exact(case, seed):
    """From the definitions; what a loss asks of a row is written as a dense row of weights."""
    s = prepare(case, seed)
    T, V, w = case["temperature"], case["V"], s["weight"].double()
    z = s["x"].detach().double() / T
    if s["mask"] is not None:
        z.masked_fill_(~bits_of(s["mask"], V), -math.inf)
    over = (z == -math.inf).all(dim=1)
    lp = z.sub_(torch.logsumexp(z, dim=1).masked_fill(over, 0.0)[:, None])
    rows = torch.arange(case["rows"], device="cuda")
    if case["op"] == "distill":
        use = (s["ids"] >= 0) & (lp.gather(1, s["ids"].long().clamp(min=0)) > -math.inf)
        t = s["values"].double().masked_fill(~use, -math.inf)
        if not case["rest"]:
            t = t / T
            t = t - torch.logsumexp(t, dim=1).masked_fill((t == -math.inf).all(dim=1), 0.0)[:, None]
        r, k = torch.nonzero(use, as_tuple=True)                   # entry by entry
        v, ln_q = s["ids"].long()[r, k], t[r, k]
        q = ln_q.exp()
        sums = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
        losses = sums.index_add(0, r, q * (ln_q - lp[r, v]))
        all_q = sums.index_add(0, r, q)
        if case["rest"]:
            outside = lp.clone()
            outside[r, v] = -math.inf
            ln_rest = torch.logsumexp(outside, dim=1)
            q_rest = (1.0 - all_q).clamp(min=0.0).masked_fill(~use.any(dim=1) | (ln_rest == -math.inf), 0.0)
            losses = losses + (q_rest * (q_rest.clamp(min=1e-300).log() - ln_rest.masked_fill(ln_rest == -math.inf, 0.0)))
            grad = lp.exp_() * (all_q + q_rest)[:, None]
            grad -= outside.sub_(ln_rest.masked_fill(ln_rest == -math.inf, 0.0)[:, None]).exp_() * q_rest[:, None]
        else:
            grad = lp.exp_() * all_q[:, None]
        grad.index_put_((r, v), -q, accumulate=True)
        out = {"losses": losses, "loss": w @ losses}
        if case["grad"]:
            out["grad"] = grad.mul_(w[:, None] / T)
        return out
    tokens = s["tokens"]
    at = lp[rows, tokens.clamp(min=0)].masked_fill(tokens < 0, 0.0)
    counts = (tokens >= 0) & (at > -math.inf)
    entropy = None
    if case["op"] == "policy":
        ratio, a = (at - s["old"].double()).exp(), s["advantages"].double()
        clipped = ((a > 0) & (ratio > 1 + CLIP[1])) | ((a < 0) & (ratio < 1 - CLIP[0]))
        border = torch.where(a > 0, 1 + CLIP[1], 1 - CLIP[0])
        losses = -a * torch.where(clipped, border, ratio)
        slope = -a * ratio.masked_fill(clipped, 0.0)
        if case["kl"]:
            back = (s["ref"].double() - at)
            losses = losses + KL * (torch.expm1(back) - back)
            slope = slope - KL * torch.expm1(back)
        slope = (w * slope).masked_fill(~counts, 0.0)
        if case["entropy"]:
            entropy = torch.special.entr(lp.exp()).sum(dim=1).masked_fill(tokens < 0, 0.0)
            losses = losses - ENTROPY * entropy
        losses = losses.masked_fill(~counts, 0.0)
        out = {"losses": losses, "logprobs": at, "entropy": entropy, "loss": w @ losses}
    else:
        P, offsets = case["pairs"], s["offsets"].tolist()
        value, mine = torch.zeros(2 * P, dtype=torch.float64, device="cuda"), []
        for i in range(2 * P):
            own_rows = rows[offsets[i]:offsets[i + 1]]
            own_rows = own_rows[tokens[own_rows] >= 0]
            d = (at - s["ref"].double())[own_rows]
            n = max(1, len(own_rows)) if case["average"] else 1
            value[i] = d.sum() / n
            mine.append((own_rows, n))
        h = BETA * (value[0::2] - value[1::2])
        eps = case["smoothing"]
        losses = -(1 - eps) * torch.nn.functional.logsigmoid(h) - eps * torch.nn.functional.logsigmoid(-h)
        out = {"losses": losses, "chosen": BETA * value[0::2], "rejected": BETA * value[1::2], "loss": w @ losses}
        dh = w * BETA * (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h))
        slope = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
        for i, (own_rows, n) in enumerate(mine):
            slope[own_rows] = dh[i // 2] * (1 - 2 * (i % 2)) / n
        slope = slope.masked_fill(~counts, 0.0)
    if case["grad"]:
        p = lp.exp()
        grad = p * -slope[:, None]
        grad[rows, tokens.clamp(min=0)] += slope
        if entropy is not None:
            lp.masked_fill_(lp == -math.inf, 0.0)
            grad += p.mul_(lp.add_(entropy[:, None])).mul_((ENTROPY * w).masked_fill(~counts, 0.0)[:, None])
        out["grad"] = grad.div_(T)
    return out


def bits_of(mask, V):
    v = torch.arange(V, device=mask.device)
    return torch.stack([(row.long()[v // 32] >> (v % 32)) & 1 for row in mask]).bool()


def work(case):
    B, V, size = case["rows"], case["V"], SIZE[case["dtype"]]
    read = B - int(B * case["ignored"])            # rows that count; the gradient of the others is zero, and is written
    small = {"distill": lambda: 8 * case["K"] + 8, "policy": lambda: 36, "preference": lambda: 12}[case["op"]]()
    mask = read * ((V + 31) // 32) * 4 if case["mask"] != "none" else 0
    written = B * V * size if case["grad"] else 0
    return {"bytes": read * V * size + mask + written + small * B, "flops": (10 if case["grad"] else 5) * read * V}
