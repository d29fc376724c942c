"""Sequences drawn under a grammar, with their log probabilities, and a step of training on them.

    python examples/decode_and_train.py [--config 1..5] [--steps N] [--hidden K]

What a server does at each step: the masks of the rows' parser states, the hidden states brought to 8 bits, their product with the head under
the masks, a token drawn for each row, the log probability, entropy and alternatives that it reports, and the states' advance.  Then what a learner does with
such sequences: the same positions' logits from a product in bf16, log probabilities under the masks the tokens were drawn under, and the
gradient of a policy's loss for the model's parameters.  The model is a stand-in: a table of embeddings, a mixing matrix and a head, random and seeded.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2506_01151_amd as zf  # noqa: E402
from workloads import configs  # noqa: E402


class Model:
    """hidden' = tanh(hidden mix + embedding[token]), logits = hidden head^T."""

    def __init__(self, V, K, device, seed=1):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, sigma):
            return torch.randn(shape, generator=g, device=device) * sigma

        self.embedding = normal(V, K, sigma=1.0)
        self.mix = normal(K, K, sigma=K ** -0.5)
        self.head = normal(V, K, sigma=2 * K ** -0.5)
        self.head_q, self.head_scale = zf.quantize_blocks(self.head, block_rows=128)      # once, when the model is loaded

    def step(self, hidden, tokens):
        return torch.tanh(hidden @ self.mix + self.embedding[tokens.clamp(min=0)])


def draw(logits, temperature, generator):
    """A token of each row from softmax(logits / temperature): the largest of the logits with Gumbel noise.  -1 where all are -inf."""
    noise = torch.rand(logits.shape, generator=generator, device=logits.device).clamp_(min=1e-20).log_().neg_().log_().neg_()
    best, tokens = (logits.float() / temperature + noise).max(dim=1)
    return torch.where(best > float("-inf"), tokens, -1).to(torch.int32)


def decode(engine, model, batch, steps, temperature=0.8, top=5, seed=2):
    """`steps` tokens for each of `batch` rows: a list of steps, each (hidden, masks, tokens, reported).  A row that is at the end of its sentence (its
    mask leaves nothing) begins another; its token of that step is -1."""
    device = model.head.device
    generator = torch.Generator(device=device)
    generator.manual_seed(seed)
    states = zf.StateBatch([engine.new_state() for _ in range(batch)])
    hidden = torch.zeros((batch, model.head.shape[1]), device=device)
    out = []
    for _ in range(steps):
        mask = torch.empty((batch, engine.W), dtype=torch.int32, device=device)
        zf.compute_mask_async(engine, states, mask)
        q, scale = zf.quantize_blocks(hidden)
        logits = zf.head_logits(q, scale, model.head_q, model.head_scale, mask, dtype=torch.bfloat16)
        tokens = draw(logits, temperature, generator)
        reported = zf.token_logprobs(logits, tokens, mask, temperature=temperature, entropy=True, top=top)
        out.append((hidden, mask, tokens, reported))
        hidden = model.step(hidden, tokens)
        zf.mask_wait(engine)
        states.advance(tokens.tolist())                    # (a negative token resets its row)
    return out


def train_step(model, steps, advantage, temperature=0.8, entropy_weight=0.01):
    """Loss, its gradients for (hidden, head) and the tokens' log probabilities: -advantage x log probability - entropy_weight x entropy, a mean over the
    tokens that were drawn.  The masks are those of the drawing, so a token's probability is again its share of what the grammar allowed."""
    hidden = torch.cat([s[0] for s in steps]).to(torch.bfloat16).requires_grad_()
    head = model.head.to(torch.bfloat16).requires_grad_()
    mask = torch.cat([s[1] for s in steps])
    tokens = torch.cat([s[2] for s in steps])
    logits = hidden @ head.t()
    got = zf.token_logprobs(logits, tokens, mask, temperature=temperature, entropy=True)
    drawn = tokens >= 0
    entropy = torch.where(drawn, got.entropy, 0.0)
    loss = -(advantage * got.logprobs + entropy_weight * entropy).sum() / drawn.sum()
    loss.backward()
    return loss.detach(), hidden.grad, head.grad, got.logprobs.detach()


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", type=int, default=2, choices=sorted(configs.CONFIGS))
    p.add_argument("--batch", type=int, default=4)
    p.add_argument("--steps", type=int, default=24)
    p.add_argument("--hidden", type=int, default=1024)
    a = p.parse_args()
    cfg = configs.CONFIGS[a.config]
    vocab = cfg.vocab()
    engine = zf.Engine(cfg.grammar(), vocab)
    model = Model(engine.V, a.hidden, "cuda:0")
    steps = decode(engine, model, a.batch, a.steps)
    for t, (_, mask, tokens, reported) in enumerate(steps[:8]):
        token = int(tokens[0])
        others = ", ".join(f"{vocab[i]!r} {p:.2f}" for i, p in zip(reported.top_ids[0].tolist(), reported.top_logprobs[0].tolist()) if i >= 0)
        print(f"step {t}: {vocab[token] if token >= 0 else None!r}  log probability {float(reported.logprobs[0]):.3f}, entropy {float(reported.entropy[0]):.3f}; most probable: {others}")
    for r in range(a.batch):
        ids = [int(s[2][r]) for s in steps]
        print(f"row {r}: {b''.join(vocab[i] if i >= 0 else b' | ' for i in ids)!r}")
    served = torch.cat([s[3].logprobs for s in steps])
    advantage = torch.ones_like(served)
    loss, g_hidden, g_head, learnt = train_step(model, steps, advantage)
    print(f"loss {float(loss):.4f}; |gradient| of hidden states {float(g_hidden.float().norm()):.4f}, of the head {float(g_head.float().norm()):.4f}")
    print(f"log probabilities from 8-bit and from bf16 products differ by {float((served - learnt).abs().mean()):.4f} on the mean")


if __name__ == "__main__":
    main()
