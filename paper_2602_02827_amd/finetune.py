"""Fine-tunes a small late-interaction encoder on the score that the library computes.

    python -m paper_2602_02827_amd.finetune [--steps 60] [--docs 256] [--seed 0]
        [--positions bias|rotary] [--window N] [--optimiser descent|orthogonal]

One block of attention over packed token sequences, and a projection to the embedding width.  Positions
are a learned bias by buckets of distance, or a rotation of normalised queries and keys; with --window a
row sees so many tokens to either side, and the first of its sequence.  Queries are noisy excerpts of their documents in words of their
own, which the encoder has to learn to place where the documents' words are.  A step encodes a
batch of documents and their queries, takes the contrastive MaxSim loss over all pairs of the batch,
clips the gradients to a global norm and updates the weights: by plain descent, or those of the linear
layers by orthogonalised momenta.  The token table, norms with rotation, attention, loss, clipping and
orthogonalising are the library's (`training`), the linear layers torch's.  At the end the whole corpus is encoded and
searched with `colbandit_full_maxsim`; the share of queries that find their document is printed.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding, training

WORDS, WIDTH, HEADS, EMBED, QUERY_TOKENS, BUCKETS, MAX_DISTANCE = 400, 256, 4, 128, 24, 32, 128
PUNCTUATION = 20                                     # words below are masked as keys
LONGEST = 150                                        # tokens of a document


class Encoder(torch.nn.Module):
    """Token numbers of packed sequences -> unit embeddings [total, EMBED] in bfloat16."""

    def __init__(self, positions="bias", window=None):
        super().__init__()
        if positions not in ("bias", "rotary"):
            raise ValueError("positions are bias or rotary")
        self.window = window
        self.tokens = torch.nn.Parameter(torch.randn(2 * WORDS, WIDTH) * 0.5)
        self.norm = torch.nn.LayerNorm(WIDTH)
        self.qkv = torch.nn.Linear(WIDTH, 3 * WIDTH, bias=False)
        self.out = torch.nn.Linear(WIDTH, WIDTH, bias=False)
        self.project = torch.nn.Linear(WIDTH, EMBED, bias=False)
        self.rotary = positions == "rotary"
        if self.rotary:
            self.q_weight = torch.nn.Parameter(torch.ones(WIDTH // HEADS))
            self.k_weight = torch.nn.Parameter(torch.ones(WIDTH // HEADS))
            self.register_buffer("turns", training.colbandit_rotary_table(LONGEST, WIDTH // HEADS, device="cpu"))
        else:
            self.bias = torch.nn.Parameter(torch.zeros(BUCKETS, HEADS))

    def forward(self, tokens, offsets):
        x = training.embedding(self.tokens, tokens)
        q, k, v = self.qkv(self.norm(x)).bfloat16().view(-1, 3, HEADS, WIDTH // HEADS).unbind(1)
        how = {} if self.window is None else dict(window=(self.window, self.window), sinks=1)
        if self.rotary:
            rows = torch.arange(tokens.shape[0], device=tokens.device)
            positions = rows - offsets[torch.searchsorted(offsets, rows, right=True) - 1]
            q, k = training.norm_rotate(q, k, positions=positions, table=self.turns, q_weight=self.q_weight, k_weight=self.k_weight)
        else:
            how.update(bias=self.bias.bfloat16(), max_distance=MAX_DISTANCE)
        a = training.attention(q, k, v, offsets, keep=tokens >= PUNCTUATION, **how)
        x = x + self.out(a.float().flatten(1))
        return torch.nn.functional.normalize(self.project(x), dim=-1).bfloat16()


def corpus(n_docs, seed, device):
    """Packed documents of 20 to 150 tokens, and a query of QUERY_TOKENS for each: tokens of the document, a
    fifth of them replaced, in the queries' words (word w of a document is WORDS + other[w])."""
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(20, LONGEST + 1, (n_docs,), generator=g)
    offsets = torch.zeros(n_docs + 1, dtype=torch.int64)
    offsets[1:] = torch.cumsum(lengths, 0)
    tokens = torch.randint(0, WORDS, (int(offsets[-1]),), generator=g)
    other = WORDS + torch.randperm(WORDS, generator=g)
    at = torch.stack([torch.randint(int(a), int(b), (QUERY_TOKENS,), generator=g) for a, b in zip(offsets[:-1], offsets[1:])])
    queries = other[torch.where(torch.rand(at.shape, generator=g) < 0.2, torch.randint(0, WORDS, at.shape, generator=g), tokens[at])]
    return tokens.to(device), offsets.to(device), queries.to(device)


def batch_of(docs, tokens, offsets):
    """The given documents' tokens, packed, and their offsets."""
    lengths = (offsets[1:] - offsets[:-1])[docs]
    off = torch.cat([lengths.new_zeros(1), torch.cumsum(lengths, 0)])
    rows = torch.arange(int(off[-1]), device=docs.device) + torch.repeat_interleave(offsets[docs] - off[:-1], lengths)
    return tokens[rows], off


def encode_queries(encoder, queries):
    off = torch.arange(queries.shape[0] + 1, device=queries.device) * QUERY_TOKENS
    return encoder(queries.reshape(-1), off).view(queries.shape[0], QUERY_TOKENS, EMBED)


def accuracy(encoder, tokens, offsets, queries):
    """Share of the queries whose best document, by the scoring library, is their own."""
    with torch.no_grad():
        docs = encoder(tokens, offsets)
        Q = encode_queries(encoder, queries).contiguous()
    top = binding.colbandit_full_maxsim(Q, docs, offsets, K=1, want_scores=False)["topk_ids"][:, 0]
    return float((top == torch.arange(len(top), device=top.device)).float().mean())


def train(steps=60, n_docs=256, batch=32, temperature=1.0, max_norm=1.0, rate=2.0, seed=0, report=None, positions="bias", window=None,
          optimiser="descent"):
    """`rate`: of descent; orthogonalised updates, whose size does not go by the gradient's, take a hundredth of it.  Returns dict(losses, norms, before, after): the loss and gradient norm of every step, and the
    accuracy over the whole corpus before and after."""
    if optimiser not in ("descent", "orthogonal"):
        raise ValueError("an optimiser is descent or orthogonal")
    device = torch.device("cuda", torch.cuda.current_device())
    torch.manual_seed(seed)
    encoder = Encoder(positions, window).to(device)
    tokens, offsets, queries = corpus(n_docs, seed, device)
    g = torch.Generator().manual_seed(seed + 1)
    before = accuracy(encoder, tokens, offsets, queries)
    losses, norms = [], []
    parameters = list(encoder.parameters())
    layers = [m.weight for m in encoder.modules() if isinstance(m, torch.nn.Linear)] if optimiser == "orthogonal" else []
    others = [p for p in parameters if all(p is not x for x in layers)]
    momenta = {}
    batch = min(batch, n_docs)
    targets = torch.arange(batch, device=device)
    for step in range(steps):
        ids = torch.randperm(n_docs, generator=g)[:batch].to(device)
        docs, off = batch_of(ids, tokens, offsets)
        loss = training.contrastive_maxsim(encode_queries(encoder, queries[ids]), encoder(docs, off), off, targets, temperature)
        for p in parameters:
            p.grad = None
        loss.backward()
        norms.append(training.clip_gradients_(parameters, max_norm))
        now = rate / math.sqrt(1 + step / 20)
        training.orthogonal_step_(layers, momenta, rate=0.01 * now)
        with torch.no_grad():
            for p in others:
                p.sub_(p.grad, alpha=now)
        losses.append(loss.detach())
        if report and (step + 1) % 10 == 0:
            report(f"step {step + 1}: loss {float(losses[-1]):.3f}, gradient norm {float(norms[-1]):.3f}")
    return {"losses": [float(x) for x in losses], "norms": [float(x) for x in norms], "before": before,
            "after": accuracy(encoder, tokens, offsets, queries)}


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--docs", type=int, default=256)
    p.add_argument("--seed", type=int, default=0)
    p.add_argument("--positions", choices=("bias", "rotary"), default="bias")
    p.add_argument("--window", type=int)
    p.add_argument("--optimiser", choices=("descent", "orthogonal"), default="descent")
    a = p.parse_args()
    r = train(a.steps, a.docs, seed=a.seed, report=lambda line: print(line, flush=True), positions=a.positions, window=a.window,
              optimiser=a.optimiser)
    print(f"queries that find their document: {r['before']:.3f} before, {r['after']:.3f} after")


if __name__ == "__main__":
    main()
