"""A small language model trained and sampled with the token operators.

The corpus is a made-up one: a word is followed by one of four others, picked by
a fixed table, so a model that has learned it reaches a loss near log 4.  The
model reads the last CONTEXT words, and its output matrix is its embedding
table (tied), whose gradient therefore has two parts: the dense one of the
output product, and the one of the words that were looked up, which
``embed_grad`` adds to it.

With ``normed`` the output is added to the last word's embedding and normed before
the output product (``add_norm``, its backward pass ``norm_grad``).  ``answer`` writes
with the table in 8 bits: the rows in 8 bits (``add_norm_int8`` or ``quantise_rows``), the
output product of whole numbers (``project_int8``), the rules, and a word by top-k, top-p
and a uniform number (``sample_logits``).

    python examples/language_model.py [--full]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1505_03851_amd as lda  # noqa: E402

VOCABULARY, SPECIAL, SUCCESSORS = 1000, 10, 4  # words below SPECIAL are never written
CONTEXT, WIDTH, HIDDEN = 4, 64, 256
P_DROP, SEED, EPS = 0.1, 20150513, 1e-6


class Dropout(torch.autograd.Function):
    """The operator is linear and its mask is made again: it is its own backward."""

    @staticmethod
    def forward(ctx, x, p, seed, step):
        ctx.args = p, seed, step
        return lda.dropout(x.contiguous(), p, seed, step)

    @staticmethod
    def backward(ctx, grad):
        return lda.dropout(grad.contiguous(), *ctx.args), None, None, None


class Norm(torch.autograd.Function):
    """(y, h): h = x + residual, normed and weighted."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        ctx.set_materialize_grads(False)
        y, h = lda.add_norm(x.contiguous(), weight, eps, residual=residual.contiguous())
        ctx.save_for_backward(h, weight)
        ctx.eps = eps
        return y, h

    @staticmethod
    def backward(ctx, grad, grad_h):
        h, weight = ctx.saved_tensors
        if grad is None:  # only h is used
            return grad_h, grad_h, None, None
        dx, dw = lda.norm_grad(grad.contiguous(), h, weight, ctx.eps,
                               residual_grad=None if grad_h is None else grad_h.contiguous())
        return dx, dx, dw, None


def corpus(sequences: int, length: int, g: torch.Generator):
    """(successors [V][4], words int32 [sequences][length])."""
    after = torch.randint(SPECIAL, VOCABULARY, (VOCABULARY, SUCCESSORS), device="cuda", generator=g)
    words = torch.empty((sequences, length), dtype=torch.int64, device="cuda")
    words[:, 0] = torch.randint(SPECIAL, VOCABULARY, (sequences,), device="cuda", generator=g)
    for t in range(1, length):
        pick = torch.randint(0, SUCCESSORS, (sequences,), device="cuda", generator=g)
        words[:, t] = after[words[:, t - 1], pick]
    return after, words.int()


class Model:
    def __init__(self, g: torch.Generator, normed: bool = False):
        def weight(*shape):
            w = torch.randn(shape, device="cuda", generator=g) * shape[0] ** -0.5
            return w.requires_grad_()
        self.table = weight(VOCABULARY, WIDTH)
        self.inner = weight(CONTEXT * WIDTH, HIDDEN)
        self.outer = weight(HIDDEN, WIDTH)
        self.gain = torch.ones(WIDTH, device="cuda").requires_grad_() if normed else None

    def parameters(self):
        return [self.table, self.inner, self.outer] + ([] if self.gain is None else [self.gain])

    def output(self, rows, dropout=None):
        """(output [B][WIDTH], last word's embedding) of rows [B * CONTEXT][WIDTH], the
        context's embeddings."""
        h = torch.relu(rows.view(-1, CONTEXT * WIDTH) @ self.inner)
        if dropout is not None:
            h = Dropout.apply(h, *dropout)
        return h @ self.outer, rows.view(-1, CONTEXT, WIDTH)[:, -1]

    def logits(self, rows, dropout=None):
        """rows [B * CONTEXT][WIDTH], the context's embeddings -> [B][V]."""
        out, last = self.output(rows, dropout)
        if self.gain is not None:
            out, _ = Norm.apply(out, last, self.gain, EPS)
        return out @ self.table.t()


def train(model: Model, words, steps: int, batch: int, g: torch.Generator) -> list[float]:
    optimiser = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    scale = WIDTH ** 0.5
    for step in range(steps):
        row = torch.randint(0, words.shape[0], (batch,), device="cuda", generator=g)
        at = torch.randint(CONTEXT, words.shape[1], (batch, 1), device="cuda", generator=g)
        ids = words[row[:, None], at + torch.arange(-CONTEXT, 0, device="cuda")].reshape(-1)
        target = words[row, at[:, 0]].long()
        drop = P_DROP, SEED, step
        rows = lda.embed(model.table.detach(), ids, scale, *drop).requires_grad_()
        loss = torch.nn.functional.cross_entropy(model.logits(rows, (P_DROP, SEED + 1, step)), target)
        optimiser.zero_grad()
        loss.backward()
        # the output product's part is in table.grad; the lookup's is added to it
        lda.embed_grad(rows.grad, ids, VOCABULARY, scale, *drop, out=model.table.grad,
                       accumulate=True)
        optimiser.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def generate(model: Model, prompts, length: int, temperature: float = 0.8):
    """``length`` more words for each row of prompts (int32 [B][>= CONTEXT]):
    the words int32 [B][prompt + length], and each new one's probability."""
    B, start = prompts.shape
    history = torch.zeros((B, start + length), dtype=torch.int32, device="cuda")
    history[:, :start] = prompts
    lengths = torch.full((B,), start, dtype=torch.int32, device="cuda")
    prompt = lengths.clone()
    allowed = torch.ones((VOCABULARY + 31) // 32 * 32, dtype=torch.int64, device="cuda")
    allowed[:SPECIAL] = 0  # the grammar: no special words
    bits = (allowed.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
    mask = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()

    def each(value, dtype=torch.float32):
        return torch.full((B,), value, dtype=dtype, device="cuda")
    rules = dict(history=history, lengths=lengths, prompt=prompt, repetition=each(1.05),
                 presence=each(0.1), mask=mask)
    seed = torch.arange(B, device="cuda") + SEED
    chances = []
    for t in range(start, start + length):
        rows = lda.embed(model.table, history[:, t - CONTEXT:t].reshape(-1), WIDTH ** 0.5)
        z, prob = lda.draw_logits(model.logits(rows), seed, lengths, temperature=each(temperature),
                                  min_p=each(0.05), **rules)
        history[:, t] = z
        lengths += 1
        chances.append(prob)
    return history, torch.stack(chances, 1)


@torch.no_grad()
def answer(model: Model, prompts, length: int, g: torch.Generator, temperature: float = 0.8):
    """As ``generate``, with the table in 8 bits and words by uniform numbers from ``g``."""
    B, start = prompts.shape
    history = torch.zeros((B, start + length), dtype=torch.int32, device="cuda")
    history[:, :start] = prompts
    lengths = torch.full((B,), start, dtype=torch.int32, device="cuda")
    special = torch.zeros(VOCABULARY, device="cuda")
    special[:SPECIAL] = -torch.inf

    def each(value, dtype=torch.float32):
        return torch.full((B,), value, dtype=dtype, device="cuda")
    rules = dict(history=history, lengths=lengths, prompt=lengths.clone(), repetition=each(1.05),
                 bias=special)
    table, scale = lda.quantise_rows(model.table)
    chances = []
    for t in range(start, start + length):
        rows = lda.embed(model.table, history[:, t - CONTEXT:t].reshape(-1), WIDTH ** 0.5)
        out, last = model.output(rows)
        if model.gain is None:
            q, s = lda.quantise_rows(out)
        else:
            q, s, _ = lda.add_norm_int8(out, model.gain, EPS, residual=last)
        logits = lda.project_int8(q, s, table, scale, dtype=torch.float32)
        lda.penalise_logits(logits, **rules, out=logits)
        z, prob = lda.sample_logits(logits, torch.rand(B, device="cuda", generator=g),
                                    temperature=each(temperature), top_k=each(20, torch.int32),
                                    top_p=each(0.95), min_p=each(0.02))
        history[:, t] = z
        lengths += 1
        chances.append(prob)
    return history, torch.stack(chances, 1)


def main(steps: int = 400, batch: int = 512, sequences: int = 64, length: int = 24,
         normed: bool = False, eight_bits: bool = False) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(SEED)
    after, words = corpus(2000, 64, g)
    model = Model(g, normed)
    losses = train(model, words, steps, batch, g)
    prompts = words[:sequences, :CONTEXT].contiguous()
    if eight_bits:
        history, chances = answer(model, prompts, length, g)
    else:
        history, chances = generate(model, prompts, length)
    follows = (after[history[:, CONTEXT - 1:-1].long()] == history[:, CONTEXT:, None]).any(2)
    return dict(first=losses[0], last=sum(losses[-20:]) / 20, words=history,
                follows=float(follows.float().mean()), chance=float(chances.mean()))


if __name__ == "__main__":
    full = "--full" in sys.argv[1:]  # normed, and answering in 8 bits
    r = main(normed=full, eight_bits=full)
    print(f"loss {r['first']:.2f} -> {r['last']:.2f} (log {SUCCESSORS} is 1.39)")
    print(f"{100 * r['follows']:.1f}% of the generated words follow the word before them in the "
          f"corpus; mean probability of a draw {r['chance']:.2f}")
    print("one sequence:", r["words"][0].tolist())
