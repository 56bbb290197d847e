"""Scores tokens with a quantized output layer: `python -m paper_1901_09504_amd.score`.

What a language model is judged by is its perplexity, exp of the mean of -log p over the tokens that came.  Drawn from a
seed: an output layer with heavy-tailed channels, hidden states with outliers, and the tokens that the layer itself gives
(so that the 32-bit layer's perplexity is what its entropy says).  Printed: the perplexity of the 32-bit layer, and of the layer with a
grid per token and per output channel at each weight width, without and with outlier channel splitting, its change, and how
often the most likely token is the 32-bit layer's.
"""
import argparse

import torch

from .layer import TokenLayer, token_logprobs


def synthetic(tokens, hidden, vocab, seed=190109504, device="cuda"):
    """Weights fp32 [vocab, hidden], hidden states fp32 [tokens, hidden], token ids int32 [tokens] drawn from softmax(X W^T)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    W = torch.randn((vocab, hidden), device=device, generator=gen) * (2.0 / hidden ** 0.5)
    W *= 1 + 3 * (torch.rand((1, hidden), device=device, generator=gen) < 0.01)
    X = torch.randn((tokens, hidden), device=device, generator=gen)
    X = torch.where(torch.rand((tokens, hidden), device=device, generator=gen) < 0.005, X * 5, X)
    logits = X @ W.t()
    noise = torch.rand((tokens, vocab), device=device, generator=gen).clamp_min_(1e-20).log_().neg_().log_()
    return W, X, (logits - noise).argmax(1).to(torch.int32)


def perplexity(logits, tokens):
    """(exp of the mean of -log p over the positions that have a token, NaN where none has; the most likely token of every position)"""
    out = token_logprobs(logits, tokens, 1)
    has = (tokens >= 0) & (tokens < logits.shape[1])
    return float(torch.exp(-out["logprob"][has].mean())), out["top_ids"][:, 0]


def run(tokens=700, hidden=1500, vocab=10000, widths=(8, 6, 5, 4), ratios=(0.0, 0.05), seed=190109504):
    """[(bits, r, perplexity, share of positions whose most likely token is the 32-bit layer's)], the 32-bit layer first (bits 32)."""
    W, X, ids = synthetic(tokens, hidden, vocab, seed)
    exact, best = perplexity(X @ W.t(), ids)
    rows = [(32, 0.0, exact, 1.0)]
    for bits in widths:
        for r in ratios:
            head = TokenLayer(vocab, hidden, r, bits_w=bits, max_rows=tokens)
            head.prepare_weights(W)
            p, top = perplexity(head.forward(X), ids)
            rows.append((bits, r, p, float((top == best).float().mean())))
    return rows


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=700)
    ap.add_argument("--hidden", type=int, default=1500)
    ap.add_argument("--vocab", type=int, default=10000)
    a = ap.parse_args()
    rows = run(a.tokens, a.hidden, a.vocab)
    print(f"32-bit weights: perplexity {rows[0][2]:.3f}")
    for bits, r, p, same in rows[1:]:
        print(f"{bits}-bit weights, r = {r:.2f}: perplexity {p:.3f} ({100 * (p / rows[0][2] - 1):+.2f} %), same first choice {100 * same:.1f} %")


if __name__ == "__main__":
    main()
