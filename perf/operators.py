"""Layers with a grid per token and the scoring of tokens, as measurable cases.

  quantize  ocs_split_quantize_rows: channels split and every row put on a grid of its own
  product   ocs_qgemm_rows: int8 product with a scale per token and per output channel
  forward   ocs_forward_rows: the two as one call, what a layer runs per batch
  logprobs  ocs_token_logprobs: log probabilities of given tokens, entropy, top alternatives
  score     a language model's output layer on hidden states: ocs_forward_rows, then ocs_token_logprobs

Sizes: the package's small fully connected layer and the LSTM language model (hidden 1500, gates 3000 -> 6000,
batch 20, windows of 35), and generic ones for models of today: thousands of channels, vocabularies of tens of
thousands.  Where `own` is false the same outputs come from elementary torch operations.
"""
import math

import torch

own = False

# ---- the cases -------------------------------------------------------------------------------


def _quantize(name, M, C, r, dtype, bits=8, halved=False, g=1):
    return dict(name=name, kind="quantize", M=M, C=C, g=g, r=r, bits=bits, dtype=dtype, halved=halved)


def _layer(name, kind, M, C, N, r, dtype, bias, bits_w=8):
    return dict(name=name, kind=kind, M=M, C=C, N=N, r=r, bits_w=bits_w, dtype=dtype, bias=bias)


def _logprobs(name, M, V, k, dtype, masked=0.0):
    return dict(name=name, kind="logprobs", M=M, V=V, k=k, dtype=dtype, masked=masked)


def _score(name, M, C, V, k, dtype):
    return dict(name=name, kind="score", M=M, C=C, N=V, r=0.05, bits_w=8, k=k, dtype=dtype)


def listed():
    return [
        # the smallest workload's activations: a batch of 64 rows of 256
        _quantize("quantize_64x256", 64, 256, 0.05, "float32"),
        # hidden states of a long prompt in a wide model
        _quantize("quantize_4096x4096_bf16", 4096, 4096, 0.02, "bfloat16"),
        # one token through the LSTM's gates: generation at batch 1
        _layer("product_1x3000_6000", "product", 1, 3000, 6000, 0.05, "float32", True, bits_w=5),
        # the gates over a window of 20 x 35 positions
        _layer("product_700x3000_6000", "product", 700, 3000, 6000, 0.05, "float32", True, bits_w=5),
        # a square layer of a wide model over a batch of prompts: the most arithmetic
        _layer("product_8192x4096_4096_bf16", "product", 8192, 4096, 4096, 0.02, "bfloat16", False),
        # one step of the LSTM at batch 20, from its inputs
        _layer("forward_20x3000_6000", "forward", 20, 3000, 6000, 0.05, "float32", True, bits_w=5),
        # odd everything: a batch that fills no tile, rows of 1001 halves, 2049 outputs
        _layer("forward_333x1001_2049_f16", "forward", 333, 1001, 2049, 0.05, "float16", True),
        # one generated token with its twenty alternatives
        _logprobs("logprobs_1x33001", 1, 33001, 20, "float32"),
        # perplexity over a window of 20 x 35 positions, some tokens banned
        _logprobs("logprobs_700x33001", 700, 33001, 5, "float32", masked=0.01),
        # scoring a long prompt against a large vocabulary, rows of odd length
        _logprobs("logprobs_4096x100003_bf16", 4096, 100003, 8, "bfloat16"),
        # one step of generation at batch 20: hidden states to scored tokens
        _score("score_20x1500_33001", 20, 1500, 33001, 5, "bfloat16"),
        # the whole window of 20 x 35 positions
        _score("score_700x1500_33001", 700, 1500, 33001, 5, "bfloat16"),
    ]


# the largest listed case's work, which no drawn case exceeds
MOST_BYTES, MOST_FLOPS = 8.2e8, 2.8e11


def draw(rng):
    """One more case: sizes spread over the ranges by their logarithm, odd ones among them."""
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n + 1 if n == 3 * 1024 else n

    while True:
        kind = rng.choice(["quantize"] + ["product", "forward", "logprobs"] * 2 + ["score"])
        dtype = rng.choice(["float32", "bfloat16", "float16"])
        r = rng.choice([0.0, 0.01, 0.02, 0.05, 0.1])
        bits_w = rng.choice([4, 5, 6, 8, 8])
        if kind == "quantize":
            g = rng.choice([1, 1, 1, 9])
            case = _quantize(None, size(1, 8192), size(32, 6000 if g == 1 else 512), r, dtype, rng.choice([4, 6, 8, 8]),
                             rng.random() < 0.3, g)
        elif kind == "logprobs":
            case = _logprobs(None, size(1, 4096), size(300, 130000), rng.choice([1, 2, 5, 8, 20, 32]), dtype,
                             rng.choice([0.0, 0.01, 0.5]))
        elif kind == "score":
            case = _score(None, size(1, 1500), size(64, 4096), size(1000, 60000), rng.choice([1, 5, 20]), dtype)
        else:
            case = _layer(None, kind, rng.choice([size(1, 64), size(1, 8192)]), size(64, 6000), size(16, 12000), r, dtype,
                          rng.random() < 0.5, bits_w)
        del case["name"]
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


def _splits(case):
    return math.ceil(case["r"] * case["C"]) if case["r"] > 0 else 0


def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    M = case["M"]
    if case["kind"] == "quantize":
        K, Ke = case["C"] * case["g"], (case["C"] + _splits(case)) * case["g"]
        # the codes come back as the values they stand for, as 32-bit numbers
        return {"bytes": M * (K * size + 4 + 4 * Ke), "flops": 6 * M * Ke}
    if case["kind"] == "logprobs":
        return {"bytes": M * (case["V"] * size + 12 + 8 * case["k"]), "flops": 6 * M * case["V"]}
    N, Ke = case["N"], case["C"] + _splits(case)
    out = 4 if case["kind"] == "score" else size
    total = M * N * out + N * Ke + 4 * N
    total += M * (Ke + 4) if case["kind"] == "product" else M * case["C"] * size
    flops = 2 * M * N * Ke
    if case["kind"] == "score":
        total += M * (12 + 8 * case["k"])
        flops += 6 * M * N
    elif case["bias"]:
        total += 4 * N
    return {"bytes": total, "flops": flops}


# ---- inputs ----------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(190109504 + 104729 * int(seed))


def _hidden(M, K, gen, dtype):
    """Activations: N(0, 1), one value in a hundred and one channel in two hundred far larger."""
    x = torch.randn((M, K), device="cuda", generator=gen)
    x = torch.where(torch.rand((M, K), device="cuda", generator=gen) < 0.01, x * 6, x)
    x *= torch.where(torch.rand((1, K), device="cuda", generator=gen) < 0.005, 12.0, 1.0)
    return x.to(getattr(torch, dtype))


def _lists(maxima, C, s):
    """The channels of the s largest maxima, each split once: sources and halvings of the C + s expanded channels."""
    pick = maxima.topk(s).indices.sort().values if s else torch.zeros(0, dtype=torch.int64, device="cuda")
    src = torch.cat([torch.arange(C, device="cuda"), pick])
    depth = torch.zeros(C + s, dtype=torch.int32, device="cuda")
    depth[pick] = 1
    depth[C:] = 1
    return src.to(torch.int32), depth


def _on_row_grids(x, bits):
    """Codes and steps of the rows of x: T = max|x|, inv = fl(qmax / T), round half to even, step = fl(T / qmax)."""
    T = x.abs().amax(1, keepdim=True)
    qmax = torch.full_like(T, 2 ** (bits - 1) - 1)          # tensor by tensor: one division, rounded once
    inv = torch.where(T > 0, (qmax / T).clamp_max(torch.finfo(torch.float32).max), torch.zeros_like(T))
    return torch.minimum(torch.maximum(x * inv, -qmax), qmax).round_(), (T / qmax).squeeze(1)


def _pitch(cols):
    return -(-cols // 128) * 128


def _held(codes, pitch):
    """Codes as a layer keeps them: int8 rows of `pitch` bytes, zeros behind the codes."""
    q = torch.zeros((codes.shape[0], pitch), dtype=torch.int8, device="cuda")
    q[:, :codes.shape[1]] = codes
    return q


def _given(case, seed):
    """The inputs of a case, made from the seed alone."""
    gen = _gen(seed)
    M, kind = case["M"], case["kind"]
    if kind == "quantize":
        C, g, s = case["C"], case["g"], _splits(case)
        x = _hidden(M, C * g, gen, case["dtype"])
        src, depth = _lists(x.float().abs().amax(0).view(C, g).amax(1), C, s)
        return dict(x=x, src=src, depth=depth if case["halved"] else None)
    if kind == "logprobs":
        V, k = case["V"], case["k"]
        # frequent tokens ahead of rare ones, and in most rows one that the model is sure of
        x = 2.5 * torch.randn((M, V), device="cuda", generator=gen)
        x -= 0.7 * torch.log1p(torch.randperm(V, device="cuda", generator=gen).float())
        tokens = torch.randint(V, (M,), device="cuda", generator=gen, dtype=torch.int32)
        sure = torch.rand((M,), device="cuda", generator=gen) < 0.7
        x[torch.arange(M, device="cuda"), tokens.long()] += torch.where(sure, 10.0, 0.0)
        if case["masked"] > 0:
            x[:, torch.rand((V,), device="cuda", generator=gen) < case["masked"]] = -math.inf
            if M > 2:
                x[1] = -math.inf                    # a row whose mask leaves nothing
                x[2, 1:] = -math.inf                # and one that it leaves a single token
        if M > 4:
            tokens[3] = -1                          # padding: a position without a token
        return dict(x=x.to(getattr(torch, case["dtype"])), tokens=tokens, k=k)
    C, N, s = case["C"], case["N"], _splits(case)
    w = torch.randn((N, C), device="cuda", generator=gen) * (1.0 / math.sqrt(C))
    w = torch.where(torch.rand((N, C), device="cuda", generator=gen) < 0.001, w * 10, w)
    w *= torch.rand((N, 1), device="cuda", generator=gen) + 0.5             # output channels of different ranges
    src, depth = _lists(w.abs().amax(0), C, s)
    w = w[:, src.long()] * torch.exp2(-depth.float())
    wq, wstep = _on_row_grids(w, case["bits_w"])
    Ke = C + s
    pitch = _pitch(Ke)
    got = dict(src=src, wq=_held(wq, pitch), wstep=wstep, Ke=Ke, pitch=pitch)
    del w, wq
    if kind == "product":
        xq, got["xstep"] = _on_row_grids(_hidden(M, C, gen, "float32")[:, src.long()], 8)
        got["xq"] = _held(xq, pitch)
    else:
        got["x"] = _hidden(M, C, gen, case["dtype"])
    if case.get("bias"):
        got["bias"] = torch.randn((N,), device="cuda", generator=gen)
    if kind == "score":
        got["tokens"] = torch.randint(N, (M,), device="cuda", generator=gen, dtype=torch.int32)
    return got


def prepare(case, seed):
    state = dict(case, **_given(case, seed))
    M, kind = case["M"], case["kind"]
    # what a program keeps beside its inputs: the buffers that its calls write to
    if kind in ("quantize", "forward", "score"):
        cols = (case["C"] + _splits(case)) * case.get("g", 1)
        state["codes"] = torch.empty((M, _pitch(cols)), dtype=torch.int8, device="cuda")
        state["steps"] = torch.empty(M, device="cuda")
    if kind in ("product", "forward", "score"):
        out = torch.float32 if kind == "score" else getattr(torch, case["dtype"])
        state["y"] = torch.empty((M, case["N"]), dtype=out, device="cuda")
    if kind in ("logprobs", "score"):
        state["logprob"] = torch.empty(M, device="cuda")
        state["entropy"] = torch.empty(M, device="cuda")
        state["top_ids"] = torch.empty((M, case["k"]), dtype=torch.int32, device="cuda")
        state["top_logprobs"] = torch.empty((M, case["k"]), device="cuda")
        state["workspace"] = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    return state


# ---- the plain forms -------------------------------------------------------------------------


def _plain_codes(x, src, depth, g, bits):
    x = x.float()
    M = x.shape[0]
    cols = (src.long()[:, None] * g + torch.arange(g, device=x.device)).reshape(-1)
    x = x[:, cols]
    if depth is not None:
        x = x * torch.exp2(-depth.float()).repeat_interleave(g)
    return _on_row_grids(x, bits)


def _plain_product(codes, steps, st, out):
    y = (codes @ st["wq"][:, :st["Ke"]].float().t()) * (steps[:, None] * st["wstep"])
    if "bias" in st:
        y = y + st["bias"]
    return y.to(out)


def _plain_logprobs(x, tokens, k):
    x = x.float() + 0.0
    V = x.shape[1]
    top = x.amax(1, keepdim=True)
    none = torch.isneginf(top)
    d = torch.where(torch.isneginf(x), -math.inf, x - torch.where(none, 0.0, top))
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_total = torch.where(none, 0.0, torch.log(total))
    mean = torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
    entropy = torch.where(none, 0.0, log_total - mean).squeeze(1)
    has = (tokens >= 0) & (tokens < V)
    at = torch.where(has, tokens, 0).long()[:, None]
    logprob = torch.where(has, (d.gather(1, at) - log_total).squeeze(1), 0.0)
    # the k largest by value, then by lowest index, as one whole number per entry
    bits = x.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    ids = V - 1 - (order * (1 << 20) + torch.arange(V - 1, -1, -1, device=x.device)).topk(k, dim=1).values.remainder(1 << 20)
    return dict(logprob=logprob, entropy=entropy, top_ids=ids.to(torch.int32), top_logprobs=d.gather(1, ids) - log_total)


def _plain(st):
    kind = st["kind"]
    if kind == "quantize":
        codes, steps = _plain_codes(st["x"], st["src"], st["depth"], st["g"], st["bits"])
        return dict(values=codes * steps[:, None], steps=steps)
    if kind == "logprobs":
        return _plain_logprobs(st["x"], st["tokens"], st["k"])
    if kind == "product":
        return _plain_product(st["xq"][:, :st["Ke"]].float(), st["xstep"], st, getattr(torch, st["dtype"]))
    codes, steps = _plain_codes(st["x"], st["src"], None, 1, 8)
    if kind == "forward":
        return _plain_product(codes, steps, st, getattr(torch, st["dtype"]))
    logits = _plain_product(codes, steps, st, torch.float32)
    return dict(_plain_logprobs(logits, st["tokens"], st["k"]), logits=logits)


# ---- one pass --------------------------------------------------------------------------------


def run(st):
    if not own:
        return _plain(st)
    from paper_1901_09504_amd import binding as B

    kind, M = st["kind"], st["M"]
    if kind == "quantize":
        g = st["g"]
        B.ocs_split_quantize_rows(st["x"], M, st["C"], g, st["x"].stride(0), st["src"], st["depth"],
                                  st["src"].shape[0] - st["C"], st["bits"], 1.0, st["codes"], st["codes"].stride(0), st["steps"])
        cols = st["src"].shape[0] * g
        return dict(values=st["codes"][:, :cols] * st["steps"][:, None], steps=st["steps"])
    if kind == "product":
        B.ocs_qgemm_rows(st["xq"], st["pitch"], st["wq"], st["pitch"], M, st["N"], st["Ke"], 8, st["bits_w"], st["xstep"],
                         st["wstep"], st.get("bias"), st["y"], st["N"])
        return st["y"]
    if kind in ("forward", "score"):
        B.ocs_forward_rows(st["x"], M, st["C"], 1, st["x"].stride(0), st["src"], st["Ke"] - st["C"], 8, 1.0, st["codes"],
                           st["pitch"], st["steps"], st["wq"], st["pitch"], st["N"], st["bits_w"], st["wstep"],
                           st.get("bias"), st["y"], st["N"])
        if kind == "forward":
            return st["y"]
    x = st["y"] if kind == "score" else st["x"]
    B.ocs_token_logprobs(x, M, x.shape[1], x.stride(0), st["tokens"], st["k"], st["logprob"], st["entropy"],
                         st["top_ids"], st["top_logprobs"], st["workspace"])
    out = {n: st[n] for n in ("logprob", "entropy", "top_ids", "top_logprobs")}
    return dict(out, logits=x) if kind == "score" else out


# ---- the definitions in 64 bits --------------------------------------------------------------


def _exact_codes(x, src, depth, g, bits):
    """Eq. 1 row by row.  The grid's two numbers and the scaled value are 32-bit numbers by definition."""
    def fl(t):
        return t.to(torch.float32).to(torch.float64)

    C, M = x.shape[1] // g, x.shape[0]
    v = x.to(torch.float64).view(M, C, g).index_select(1, src.to(torch.int64))
    if depth is not None:
        v = v / (2.0 ** depth.to(torch.float64))[None, :, None]
    v = v.reshape(M, -1)
    qmax = 2 ** (bits - 1) - 1
    T = v.abs().max(1).values
    factor = fl(torch.full_like(T, qmax) / T)
    factor[T == 0] = 0
    return torch.round(fl(v * factor[:, None])).clamp(-qmax, qmax), fl(T / qmax)


def _exact_logprobs(x, tokens, k):
    out = dict(logprob=[], entropy=[], top_logprobs=[])
    for row, t in zip(x.split(64), tokens.split(64)):       # 64 rows at a time: 64-bit copies of a large vocabulary
        row = row.to(torch.float64)
        lse = torch.logsumexp(row, 1)
        alive = torch.isfinite(lse)
        lp = torch.where(alive[:, None], row - lse[:, None], torch.full_like(row, -math.inf))
        p = lp.exp()
        out["entropy"].append(-torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1))
        n = torch.arange(row.shape[0], device=row.device)
        good = (t >= 0) & (t < row.shape[1])
        picked = lp[n, torch.where(good, t, torch.zeros_like(t)).to(torch.int64)]
        out["logprob"].append(torch.where(good, picked, torch.zeros_like(picked)))
        out["top_logprobs"].append(lp.sort(1, descending=True).values[:, :k])
    return {n: torch.cat(v) for n, v in out.items()}


def exact(case, seed):
    st = _given(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        codes, steps = _exact_codes(st["x"], st["src"], st["depth"], case["g"], case["bits"])
        return dict(values=codes * steps[:, None], steps=steps)
    if kind == "logprobs":
        return dict(_exact_logprobs(st["x"], st["tokens"], case["k"]), top_ids=None)
    if kind == "product":
        codes, steps = st["xq"][:, :st["Ke"]].to(torch.float64), st["xstep"].to(torch.float64)
    else:
        codes, steps = _exact_codes(st["x"], st["src"], None, 1, 8)
    y = torch.matmul(codes, st["wq"][:, :st["Ke"]].to(torch.float64).t())
    y *= steps[:, None]
    y *= st["wstep"].to(torch.float64)[None, :]
    if "bias" in st:
        y += st["bias"].to(torch.float64)
    if kind != "score":
        return y
    return dict(_exact_logprobs(y, st["tokens"], case["k"]), top_ids=None, logits=y)
