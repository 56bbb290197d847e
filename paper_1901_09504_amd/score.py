"""Scores tokens with a quantized output layer: `python -m paper_1901_09504_amd.score`.

What a language model is judged by is its perplexity, exp of the mean of -log p over the tokens that came.  Drawn from a
seed: an output layer with heavy-tailed channels, hidden states with outliers, and the tokens that the layer itself gives
(so that the 32-bit layer's perplexity is what its entropy says).  Printed: the perplexity of the 32-bit layer, and of the layer with a
grid per token and per output channel at each weight width, without and with outlier channel splitting, its change, and how
often the most likely token is the 32-bit layer's; the same for the layer on microscaled 4-bit grids, and behind an attention layer whose
keys and values are quantized in a cache, without and with outlier channels halved.
"""
import argparse

import torch

from .layer import MxLayer, TokenCache, TokenLayer, outlier_depths, token_logprobs


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


def run_mx(tokens=700, hidden=1500, vocab=10000, ratios=(0.0, 0.05), seed=190109504):
    """As run(), with the output layer and its inputs on microscaled 4-bit grids: [(4, r, perplexity, share of same first choices)]."""
    W, X, ids = synthetic(tokens, hidden, vocab, seed)
    _, best = perplexity(X @ W.t(), ids)
    rows = []
    for r in ratios:
        head = MxLayer(vocab, hidden, r, max_rows=tokens)
        head.prepare_weights(W)
        p, top = perplexity(head.forward(X), ids)
        rows.append((4, r, p, float((top == best).float().mean())))
    return rows


def synthetic_attention(sequences, length, heads, query_heads, D, vocab, seed=190109504, device="cuda"):
    """Queries, keys (some channels far larger) and values fp32 [sequences * length, .., D], and an output layer's weights."""
    gen = torch.Generator(device=device).manual_seed(seed)
    T = sequences * length
    K = torch.randn((T, heads, D), device=device, generator=gen)
    K *= torch.where(torch.rand((1, heads, D), device=device, generator=gen) < 0.05, 8.0, 1.0)
    V = torch.randn((T, heads, D), device=device, generator=gen)
    Q = torch.randn((T, query_heads, D), device=device, generator=gen)
    W = torch.randn((vocab, query_heads * D), device=device, generator=gen) * (4.0 / (query_heads * D) ** 0.5)
    return Q, K, V, W


def causal(Q, K, V, sequences):
    """Attention of every token over its sequence up to itself, in 32 bits."""
    T, heads, D = K.shape
    L, G = T // sequences, Q.shape[1] // heads
    q = Q.view(sequences, L, heads, G, D).permute(0, 2, 3, 1, 4).reshape(sequences * heads, G * L, D)
    k = K.view(sequences, L, heads, D).permute(0, 2, 3, 1).reshape(sequences * heads, D, L)
    v = V.view(sequences, L, heads, D).transpose(1, 2).reshape(sequences * heads, L, D)
    s = ((q @ k) * D ** -0.5).view(-1, G, L, L)
    s = s.masked_fill(torch.ones((L, L), dtype=torch.bool, device=Q.device).triu(1), -torch.inf).softmax(-1).view(-1, G * L, L)
    return (s @ v).view(sequences, heads, G, L, D).permute(0, 3, 1, 2, 4).reshape(T, -1)


def run_cache(sequences=4, length=200, heads=4, query_heads=8, D=64, vocab=10000, ratios=(0.0, 0.1), seed=190109504):
    """[(bits of the cache, r, perplexity, share of same first choices)], 32 bits first: prompts of all but the last 8 tokens, then one by one."""
    Q, K, V, W = synthetic_attention(sequences, length, heads, query_heads, D, vocab, seed)
    logits = causal(Q, K, V, sequences) @ W.t()
    gen = torch.Generator(device=Q.device).manual_seed(seed + 1)
    noise = torch.rand(logits.shape, device=Q.device, generator=gen).clamp_min_(1e-20).log_().neg_().log_()
    ids = (logits - noise).argmax(1).to(torch.int32)
    exact, best = perplexity(logits, ids)
    rows, prompt = [(32, 0.0, exact, 1.0)], max(length - 8, 0)
    of = [x.view(sequences, length, -1, D) for x in (Q, K, V)]
    for bits in (8, 4):
        for r in ratios:
            cache = TokenCache(sequences, sequences * -(-length // 32), heads, D, page_rows=32, bits=bits, key_depth=outlier_depths(K, r))
            y = torch.empty_like(of[0])
            for begin, end in ([(0, prompt)] if prompt else []) + [(i, i + 1) for i in range(prompt, length)]:
                q, k, v = (x[:, begin:end].flatten(0, 1) for x in of)
                counts = [end - begin] * sequences
                cache.append(k, v, counts)
                y[:, begin:end] = cache.attend(q, counts).view(sequences, end - begin, query_heads, D)
            p, top = perplexity(y.view(sequences * length, -1) @ W.t(), ids)
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
    for bits, r, p, same in run_mx(a.tokens, a.hidden, a.vocab):
        print(f"{bits}-bit microscaled layer, r = {r:.2f}: perplexity {p:.3f} ({100 * (p / rows[0][2] - 1):+.2f} %), same first choice {100 * same:.1f} %")
    rows = run_cache(vocab=a.vocab)
    print(f"behind attention, 32-bit keys and values: perplexity {rows[0][2]:.3f}")
    for bits, r, p, same in rows[1:]:
        print(f"{bits}-bit cache, r = {r:.2f}: perplexity {p:.3f} ({100 * (p / rows[0][2] - 1):+.2f} %), same first choice {100 * same:.1f} %")


if __name__ == "__main__":
    main()
