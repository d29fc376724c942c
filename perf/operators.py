"""What is timed of the operators at the two ends of a step's logits: the head's product that makes them, and the log probabilities that are read from them.

A case is one of
  quantize   a tensor brought to 8 bits (e4m3) with a 32-bit scale for each block: of 1 x 128 (activations), or of 128 x 128 (a weight)
  head       hidden states brought to 8 bits and multiplied with the head's weight, which is held in 8 bits with scales for 128 x 128; under a mask
             the logits of tokens that it does not allow are -inf
  logprobs   log probabilities of given tokens under a mask, the rows' entropies, the most probable tokens beside them: what a server reports
  train      the same with the gradient of the logits: a step of training on sequences that were drawn under masks
Vocabularies and batches are those of workloads/configs.py, hidden sizes are generic.  `own` says who computes: elementary torch operations
in 32 bits, or this package.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
SIGMA = {"f32": 1.0, "bf16": 2.0}
BLOCK, LARGEST = 128, 448.0                        # elements a scale stands for in each direction; e4m3's largest number
SMALLEST = 2.0 ** -126                             # no scale is below it


def listed():
    return [
        # latency alone: one query's step at the smallest vocabulary
        head("head_v2k_b1", 1, 2048, 1024, "f32"),
        # a batch in the middle of its objects, where the grammar leaves each row a few hundred tokens
        head("head_v128k_b16_few", 16, 128256, 4096, "bf16", "few", 200),
        # a full batch at the largest vocabulary; masks that allow from next to nothing to nearly all
        head("head_v152k_b64", 64, 152064, 2048, "f32", "share"),
        # sizes that are multiples of nothing
        head("head_v40037_b130", 130, 40037, 1000, "bf16"),
        # a prompt scored, or a rollout's tokens once more: bound by the product itself
        head("head_v128k_b2048", 2048, 128256, 4096, "bf16"),
        # the activations of a prompt
        {"name": "quantize_b2048", "op": "quantize", "rows": 2048, "cols": 4096, "dtype": "bf16", "square": False},
        # a head's weight, when a model is loaded
        {"name": "quantize_weight_v32k", "op": "quantize", "rows": 32000, "cols": 4096, "dtype": "f32", "square": True},
        # one query of an interactive program that shows alternatives
        logprobs("logprobs_v32k_b1", 1, 32000, "f32", "none", 5, True),
        # a full batch under masks, what a server reports at most
        logprobs("logprobs_v128k_b64", 64, 128256, "bf16", "share", 20, True, 0.7),
        # a prompt's tokens scored, an odd vocabulary
        logprobs("logprobs_v40037_b1030", 1030, 40037, "bf16", "none", 0, False),
        # a small step of training on constrained sequences
        logprobs("train_v32k_b300", 300, 32000, "f32", "share", 0, True, op="train"),
        # a large one
        logprobs("train_v128k_b4096", 4096, 128256, "bf16", "none", 0, True, op="train"),
    ]


def head(name, batch, V, K, dtype, mask="none", allowed=0):
    c = {"op": "head", "batch": batch, "V": V, "K": K, "dtype": dtype, "mask": mask, "allowed": allowed}
    return dict(c, name=name) if name else c


def logprobs(name, batch, V, dtype, mask, top, entropy, temperature=1.0, op="logprobs"):
    c = {"op": op, "batch": batch, "V": V, "dtype": dtype, "mask": mask, "allowed": 0, "top": top, "entropy": entropy, "temperature": temperature}
    return dict(c, name=name) if name else c


def between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    V, dtype, kind = between(rng, 2048, 152064), rng.choice(("f32", "bf16")), rng.random()
    if rng.random() < 0.5:
        V = V // 64 * 64                           # half of the vocabularies are padded to a round size, the others are what they are
    K = between(rng, 256, 4096)
    K = K // 128 * 128 if rng.random() < 0.7 else K
    K = 3200 if K == 3072 else K
    if kind < 0.15:
        return {"op": "quantize", "rows": between(rng, 1, 32000), "cols": K, "dtype": dtype, "square": rng.random() < 0.4}
    mask = rng.choice(("none", "few", "share"))
    if kind < 0.5:
        batch = min(between(rng, 1, 2048), 2048 * 128256 * 4096 // (V * K), 2 ** 29 // (V * SIZE[dtype]))
        return head(None, max(1, batch), V, K, dtype, mask, between(rng, 1, 2000) if mask == "few" else 0)
    op = "logprobs" if kind < 0.75 else "train"
    batch = min(between(rng, 1, 4096), 2 ** 30 // (V * SIZE[dtype]))
    c = logprobs(None, max(1, batch), V, dtype, mask, rng.choice((0, 1, 5, 20)) if op == "logprobs" else 0, op == "train" or rng.random() < 0.7,
                 rng.choice((1.0, 1.0, 0.7, 1.3)), op)
    return dict(c, allowed=between(rng, 1, 2000) if mask == "few" else 0)


# ---- inputs --------------------------------------------------------------------------------------
def mask_of(case, gen):
    """Packed masks, bit v % 32 of word v / 32, as the mask kernels write them; one row of sixteen or more is over and allows nothing."""
    if case["mask"] == "none":
        return None
    B, V = case["batch"], case["V"]
    W = (V + 31) // 32
    share = torch.rand((B, 1), generator=gen, device="cuda") ** 3 if case["mask"] == "share" else min(1.0, case["allowed"] / V)
    bits = torch.rand((B, W * 32), generator=gen, device="cuda") < share
    bits[:, V:] = False
    bits[torch.arange(B, device="cuda"), torch.randint(V, (B,), generator=gen, device="cuda")] = True
    if B >= 16:
        bits[B // 2] = False
    words = (bits.view(B, W, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def weight_of(V, K, gen):
    """A weight in 8 bits and its scales: columns padded with zeros to whole blocks, as a checkpoint holds them."""
    rows, cols = -(-V // BLOCK) * BLOCK, -(-K // BLOCK) * BLOCK
    w = torch.zeros((rows, cols), device="cuda")
    w[:V, :K].normal_(0.0, 2.0 / math.sqrt(K), generator=gen)
    tiles = w.view(rows // BLOCK, BLOCK, cols // BLOCK, BLOCK)
    scale = tiles.abs().amax(dim=(1, 3)).div_(LARGEST).clamp_(min=SMALLEST)
    tiles.div_(scale[:, None, :, None]).clamp_(-LARGEST, LARGEST)
    return w[:V].to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "quantize":
        x = torch.empty((case["rows"], case["cols"]), device="cuda").normal_(0.0, 1.0, generator=gen)
        x[:, torch.randint(case["cols"], (8,), generator=gen, device="cuda")] *= 10.0   # a few columns stand out
        return {"case": case, "x": x.to(DTYPES[case["dtype"]])}
    B, V = case["batch"], case["V"]
    if case["op"] == "head":
        x = torch.empty((B, case["K"]), device="cuda").normal_(0.0, 1.0, generator=gen)
        x[:, torch.randint(case["K"], (8,), generator=gen, device="cuda")] *= 10.0
        weight, scale = weight_of(V, case["K"], gen)
        return {"case": case, "x": x.to(torch.bfloat16), "weight": weight, "scale": scale, "mask": mask_of(case, gen)}
    x = torch.empty((B, V), dtype=DTYPES[case["dtype"]], device="cuda").normal_(0.0, SIGMA[case["dtype"]], generator=gen)
    mask = mask_of(case, gen)
    if mask is None:
        tokens = torch.randint(V, (B,), generator=gen, device="cuda")
    else:                                          # the tokens were drawn under their masks
        score = torch.where(allowed_of(mask, V), torch.rand((B, V), generator=gen, device="cuda"), -1.0)
        tokens = score.argmax(dim=1)
    state = {"case": case, "x": x, "tokens": tokens, "mask": mask}
    if case["op"] == "train":
        x.requires_grad_()
        tokens[torch.rand((B,), generator=gen, device="cuda") < 0.05] = -1      # where a shorter sequence is padded
        state["g"] = torch.empty((B,), device="cuda").normal_(0.0, 1.0, generator=gen)
        state["gh"] = torch.empty((B,), device="cuda").normal_(0.0, 0.01, generator=gen)
    return state


# ---- one pass ------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if not own:
        return PLAIN[case["op"]](state)
    import paper_2506_01151_amd as zf
    if case["op"] == "quantize":
        q, scale = zf.quantize_blocks(state["x"], block_rows=BLOCK if case["square"] else 1)
        return {"q": q, "scale": scale}
    if case["op"] == "head":
        q, scale = zf.quantize_blocks(state["x"])
        return zf.head_logits(q, scale, state["weight"], state["scale"], mask=state["mask"], dtype=DTYPES[case["dtype"]])
    got = zf.token_logprobs(state["x"], state["tokens"], state["mask"], temperature=case["temperature"], entropy=case["entropy"], top=case["top"])
    if case["op"] == "train":
        grad, = torch.autograd.grad((got.logprobs, got.entropy), state["x"], (state["g"], state["gh"]))
        return {"logprobs": got.logprobs.detach(), "entropy": got.entropy.detach(), "grad": grad}
    return {"logprobs": got.logprobs, "entropy": got.entropy, "top_ids": got.top_ids, "top_logprobs": got.top_logprobs}


def allowed_of(mask, V):
    return ((mask.unsqueeze(-1) >> torch.arange(32, dtype=torch.int32, device=mask.device)) & 1).bool().view(mask.shape[0], -1)[:, :V]


def plain_blocks(x, block_rows):
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % block_rows))
    tiles = x.view(x.shape[0] // block_rows, block_rows, x.shape[1] // BLOCK, BLOCK)
    most = tiles.abs().amax(dim=(1, 3))
    scale = (most / torch.full_like(most, LARGEST)).clamp(min=SMALLEST)      # by a tensor: by a number, torch multiplies with its reciprocal
    q = (tiles / scale[:, None, :, None]).clamp(-LARGEST, LARGEST).view(x.shape)[:rows]
    return q.to(torch.float8_e4m3fn), scale


def plain_quantize(state):
    q, scale = plain_blocks(state["x"], BLOCK if state["case"]["square"] else 1)
    return {"q": q, "scale": scale}


def plain_head(state):
    V = state["case"]["V"]
    q, scale = plain_blocks(state["x"], 1)
    x = q.float() * scale.repeat_interleave(BLOCK, dim=1)
    w = state["weight"].float() * state["scale"].repeat_interleave(BLOCK, dim=0)[:V].repeat_interleave(BLOCK, dim=1)
    y = x @ w.t()
    if state["mask"] is not None:
        y = torch.where(allowed_of(state["mask"], V), y, -math.inf)
    return y.to(DTYPES[state["case"]["dtype"]])


def plain_softmax(state):
    """What both directions start from: whether a row has anything, z = x / temperature less its maximum, e ** z, the sum, the log probabilities."""
    case = state["case"]
    x = state["x"].detach().float()
    if state["mask"] is not None:
        x = torch.where(allowed_of(state["mask"], case["V"]), x, -math.inf)
    most = x.amax(dim=1, keepdim=True)
    some = most > -math.inf
    z = torch.where(some, x - most, -math.inf) / case["temperature"]
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    lp = torch.where(some, z - torch.log(total), -math.inf)
    p = torch.where(some, e / total, 0.0)
    return x, lp, p


def given(lp, tokens):
    return torch.where(tokens >= 0, lp.gather(1, tokens.clamp(min=0).unsqueeze(1)).squeeze(1), 0.0)


def entropy_of(lp, p):
    return -torch.where(p > 0, p * lp, 0.0).sum(dim=1)


def plain_logprobs(state):
    x, lp, p = plain_softmax(state)
    out = {"logprobs": given(lp, state["tokens"]), "entropy": None, "top_ids": None, "top_logprobs": None}
    if state["case"]["entropy"]:
        out["entropy"] = entropy_of(lp, p)
    if state["case"]["top"]:
        best, ids = (t[:, :state["case"]["top"]] for t in torch.sort(x, dim=1, descending=True, stable=True))
        out["top_ids"] = torch.where(best > -math.inf, ids, -1).to(torch.int32)
        out["top_logprobs"] = lp.gather(1, ids)
    return out


def plain_train(state):
    _, lp, p = plain_softmax(state)
    tokens, entropy = state["tokens"], entropy_of(lp, p)
    at = given(lp, tokens)
    g = torch.where((tokens >= 0) & (at > -math.inf), state["g"], 0.0)
    grad = -p * g.unsqueeze(1) - torch.where(p > 0, p * (lp + entropy.unsqueeze(1)), 0.0) * state["gh"].unsqueeze(1)
    grad.scatter_add_(1, tokens.clamp(min=0).unsqueeze(1), g.unsqueeze(1))
    return {"logprobs": at, "entropy": entropy, "grad": (grad / state["case"]["temperature"]).to(state["x"].dtype)}


PLAIN = {"quantize": plain_quantize, "head": plain_head, "logprobs": plain_logprobs, "train": plain_train}


# ---- the same in 64 bits ---------------------------------------------------------------------------
def exact(case, seed):
    """From the definitions: 8-bit numbers by their definition from the 32-bit quotient, everything behind them in 64 bits."""
    s = prepare(case, seed)
    if case["op"] in ("quantize", "head"):
        square = case.get("square", False)
        x = s["x"].double()
        rows, cols = x.shape
        tall = BLOCK if square else 1
        of_row = torch.arange(rows, device="cuda") // tall
        of_col = torch.arange(cols, device="cuda") // BLOCK
        by_col = torch.zeros((rows, -(-cols // BLOCK)), dtype=torch.float64, device="cuda")
        by_col.scatter_reduce_(1, of_col.expand(rows, cols), x.abs(), "amax")
        by_block = torch.zeros((-(-rows // tall), by_col.shape[1]), dtype=torch.float64, device="cuda")
        by_block.scatter_reduce_(0, of_row[:, None].expand_as(by_col), by_col, "amax")
        scale = torch.maximum(by_block / LARGEST, torch.full_like(by_block, SMALLEST)).float()
        quotient = s["x"].float() / scale[of_row][:, of_col]
        q = torch.zeros((rows, by_col.shape[1] * BLOCK), dtype=torch.float64, device="cuda")
        q[:, :cols] = quotient.clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn).double()
        if case["op"] == "quantize":
            return {"q": q, "scale": scale.double()}
        k = torch.arange(q.shape[1], device="cuda") // BLOCK
        w = s["weight"].double()
        for r in range(0, w.shape[0], 16384):
            n = torch.arange(r, min(r + 16384, w.shape[0]), device="cuda") // BLOCK
            w[r:r + 16384] *= s["scale"].double()[n][:, k]
        y = (q * scale.double()[:, k]) @ w.t()
        if s["mask"] is not None:
            y.masked_fill_(~bits_of(s["mask"], case["V"]), -math.inf)
        return y
    x = s["x"].detach().double()
    if s["mask"] is not None:
        x.masked_fill_(~bits_of(s["mask"], case["V"]), -math.inf)
    over = (x == -math.inf).all(dim=1)
    z = x / case["temperature"]
    lp = z - torch.logsumexp(z, dim=1).masked_fill(over, 0.0)[:, None]
    rows, tokens = torch.arange(x.shape[0], device="cuda"), s["tokens"]
    at = lp[rows, tokens.clamp(min=0)].masked_fill(tokens < 0, 0.0)
    p = lp.exp()
    entropy = -(p * lp.masked_fill(lp == -math.inf, 0.0)).sum(dim=1)
    if case["op"] == "train":
        gold = s["g"].double().masked_fill((tokens < 0) | (at == -math.inf), 0.0)
        grad = p * (-gold[:, None] - s["gh"].double()[:, None] * (lp.masked_fill(lp == -math.inf, 0.0) + entropy[:, None]))
        grad[rows, tokens.clamp(min=0)] += gold
        return {"logprobs": at, "entropy": entropy, "grad": grad / case["temperature"]}
    out = {"logprobs": at, "entropy": entropy if case["entropy"] else None, "top_ids": None, "top_logprobs": None}
    if case["top"]:
        out["top_logprobs"] = torch.topk(lp, case["top"], dim=1).values
    return out


def bits_of(mask, V):
    v = torch.arange(V, device=mask.device)
    return torch.stack([(row.long()[v // 32] >> (v % 32)) & 1 for row in mask]).bool()


def work(case):
    if case["op"] == "quantize":
        n, blocks = case["rows"] * case["cols"], -(-case["rows"] // (BLOCK if case["square"] else 1)) * -(-case["cols"] // BLOCK)
        return {"bytes": n * (SIZE[case["dtype"]] + 1) + 4 * blocks, "flops": 2 * n}
    B, V, words = case["batch"], case["V"], (case["V"] + 31) // 32
    mask = B * words * 4 if case["mask"] != "none" else 0
    if case["op"] == "head":
        K, of_row, needed = case["K"], V, V
        if case["mask"] == "few":                  # the tokens that a row allows, and those that some row does
            of_row = min(V, case["allowed"])
            needed = V * (1.0 - (1.0 - of_row / V) ** B)
        return {"bytes": needed * K + 4 * (needed / BLOCK) * (K / BLOCK) + 2 * B * K + B * V * SIZE[case["dtype"]] + mask, "flops": 2 * B * of_row * K}
    passes = 2 if case["op"] == "train" else 1     # the logits read; their gradient written
    return {"bytes": passes * B * V * SIZE[case["dtype"]] + mask + 24 * B, "flops": (5 if passes == 1 else 10) * B * V}
