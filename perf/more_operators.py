"""Microscaled 4-bit layers, and a quantized key/value cache with the attention that reads it, as measurable cases.

  quantize  ocs_split_quantize_mx, then ocs_dequantize_mx: channels split, blocks of 32 put on 4-bit grids, the values they stand for
  product   ocs_qgemm_mx: product of two microscaled operands
  forward   ocs_forward_mx: a layer per batch, from its inputs
  cache     ocs_cache_write, then ocs_cache_read: new tokens' keys and values quantized into pages, and rows read back
  attend    ocs_cache_attention: queries of the newest tokens over the pages

Sizes: the package's small fully connected layer and the LSTM language model (gates 3000 -> 6000), and generic ones
for models of today: thousands of channels, heads of 32 to 256, caches of tens of thousands of positions.  Where `own` is
false the same outputs come from elementary torch operations.
"""
import math

import torch

own = False

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]        # magnitudes of the 4-bit codes 0 .. 7; bit 3 is the sign

# ---- the cases -------------------------------------------------------------------------------


def _quantize(name, M, C, r, dtype, halved=False, g=1):
    return dict(name=name, kind="quantize", M=M, C=C, g=g, r=r, dtype=dtype, halved=halved)


def _layer(name, kind, M, C, N, r, dtype, bias):
    return dict(name=name, kind=kind, M=M, C=C, N=N, r=r, dtype=dtype, bias=bias)


def _cache(name, B, n, held, H, D, P, fmt, dtype, halved, back):
    """B sequences with up to `held` positions, the newest up to `n` of each written; back: those, or all rows, read."""
    return dict(name=name, kind="cache", B=B, n=n, held=held, H=H, D=D, P=P, fmt=fmt, dtype=dtype, halved=halved, back=back)


def _attend(name, B, n, held, G, H, D, P, fmt, dtype, halved=False, window=0):
    """The newest up to `n` tokens of B sequences of up to `held` positions; H heads in the cache, G query heads for each."""
    return dict(name=name, kind="attend", B=B, n=n, held=held, G=G, H=H, D=D, P=P, fmt=fmt, dtype=dtype, halved=halved,
                window=window)


def listed():
    return [
        # the smallest workload's activations: a batch of 64 rows of 256
        _quantize("quantize_64x256", 64, 256, 0.05, "float32"),
        # hidden states of a long prompt in a wide model
        _quantize("quantize_4096x4096_bf16", 4096, 4096, 0.02, "bfloat16"),
        # one token through the LSTM's gates: generation at batch 1
        _layer("forward_1x3000_6000", "forward", 1, 3000, 6000, 0.05, "float32", True),
        # odd everything: a batch that fills no tile, rows of 1001 halves, 2049 outputs
        _layer("forward_333x1001_2049_f16", "forward", 333, 1001, 2049, 0.05, "float16", True),
        # a square layer of a wide model over a batch of prompts: the most arithmetic
        _layer("product_8192x4096_4096_bf16", "product", 8192, 4096, 4096, 0.02, "bfloat16", False),
        # one step of generation at batch 64: a token's keys and values of each sequence
        _cache("cache_64_tokens", 64, 1, 2000, 8, 128, 64, "int8", "bfloat16", True, "new"),
        # prompts of odd lengths on their way into the cache, 4 bits, odd head size
        _cache("cache_prompts_mx4_f16", 5, 1777, 2100, 6, 96, 16, "mx4", "float16", True, "new"),
        # a few new tokens, then whole sequences handed on as numbers
        _cache("cache_back_mx4", 16, 3, 4097, 8, 128, 128, "mx4", "bfloat16", False, "all"),
        # the smallest: one sequence of the LSTM's window of 35 positions
        _attend("attend_1x35", 1, 1, 35, 1, 4, 64, 16, "int8", "float32"),
        # one step of generation at batch 64, sequences of all lengths to 8192
        _attend("attend_64x8192_bf16", 64, 1, 8192, 4, 8, 128, 64, "int8", "bfloat16", True),
        # one long sequence at batch 1, 4 bits
        _attend("attend_1x100003_mx4_bf16", 1, 1, 100003, 8, 8, 128, 256, "mx4", "bfloat16"),
        # prompts in chunks behind what the cache holds: the most attention arithmetic
        _attend("attend_prompts_bf16", 4, 2048, 6001, 4, 8, 128, 64, "int8", "bfloat16"),
    ]


# the largest listed cases' work, which no drawn case exceeds
MOST_BYTES, MOST_FLOPS = 5.6e8, 2.8e11


def draw(rng):
    """One more case: sizes spread over the ranges by their logarithm, odd ones among them."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["quantize", "product", "forward", "forward", "cache", "cache", "attend", "attend", "attend"])
        dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
        if kind in ("cache", "attend"):
            fmt, P = rng.choice(["int8", "mx4"]), rng.choice([16, 32, 64, 128, 256])
            D = rng.choice([32, 64, 96, 128, 128, 128, 192, 256])
            one = rng.random() < 0.5
            B, n, held = size(1, 200), 1 if one else size(2, 2500), size(1, 100000)
            n = min(n, held)
            if kind == "cache":
                case = _cache(None, B, n, held, size(1, 16), D, P, fmt, dtype, rng.random() < 0.5, rng.choice(["new", "all"]))
            else:
                case = _attend(None, B, n, held, rng.choice([1, 1, 2, 3, 4, 5, 8, 8, 16]), size(1, 16), D, P, fmt, dtype,
                               rng.random() < 0.3, rng.choice([0, 0, 0, size(1, 5000)]))
            # what the plain form lays out: padded rows and scores
            padded = B * held * case["H"] * D
            scores = B * n * held * case["H"] * case.get("G", 1)
            if padded > 6e8 or scores > 2e9:
                continue
        elif kind == "quantize":
            g = rng.choice([1, 1, 1, 9])
            r = rng.choice([0.0, 0.01, 0.02, 0.05, 0.1])
            case = _quantize(None, size(1, 8192), size(32, 6000 if g == 1 else 512), r, dtype, rng.random() < 0.3, g)
        else:
            r = rng.choice([0.0, 0.01, 0.02, 0.05, 0.1])
            case = _layer(None, kind, rng.choice([size(1, 64), size(1, 8192)]), size(64, 6000), size(16, 12000), r, dtype,
                          rng.random() < 0.5)
        del case["name"]
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


def _splits(case):
    return math.ceil(case["r"] * case["C"]) if case["r"] > 0 else 0


def _lengths(case):
    """Positions of every sequence, spread evenly up to the longest, and how many of them are new."""
    B = case["B"]
    held = [-(-case["held"] * (b + 1) // B) for b in range(B)]
    return held, [min(held[b], -(-case["n"] * (B - b) // B)) for b in range(B)]


def _row_bytes(case):
    return case["D"] + 4 if case["fmt"] == "int8" else case["D"] // 2 + case["D"] // 32


def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    kind = case["kind"]
    if kind == "quantize":
        K, Ke = case["C"] * case["g"], (case["C"] + _splits(case)) * case["g"]
        # the codes come back as the values they stand for
        return {"bytes": case["M"] * (K * size + Ke * (4 if size == 4 else 2)), "flops": 4 * case["M"] * Ke}
    if kind in ("product", "forward"):
        M, N, Ke = case["M"], case["N"], case["C"] + _splits(case)
        held = -(-Ke * 17 // 32)
        total = N * held + M * N * size + (4 * N if case["bias"] else 0)
        return {"bytes": total + M * (held if kind == "product" else case["C"] * size), "flops": 2 * M * N * Ke}
    held, new = _lengths(case)
    H, D = case["H"], case["D"]
    if kind == "cache":
        back = sum(new if case["back"] == "new" else held)
        total = 2 * H * (sum(new) * D * size + back * D * size)
        # rows that come back but were held before are read; the new ones' codes are written
        total += 2 * H * (sum(new) + (back - sum(new))) * _row_bytes(case)
        return {"bytes": total, "flops": 6 * 2 * H * D * back}
    window = case["window"] if case["window"] else max(held)
    rows = sum(min(L, window + n - 1) for L, n in zip(held, new))
    # the newest n positions p = L - n .. L - 1 see min(p + 1, window) positions each
    def seen(L, n):
        full = max(0, min(n, L - window))                   # of them, those that see a whole window
        part = n - full
        return full * window + part * (L - n + 1) + part * (part - 1) // 2
    pairs = sum(seen(L, n) for L, n in zip(held, new))
    q = case["G"] * H
    return {"bytes": 2 * rows * H * _row_bytes(case) + sum(new) * q * (2 * D * size + 4), "flops": 4 * D * q * pairs}


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


def _nearest(v):
    """The 4-bit codes of scaled values: nearest of GRID, halves to the even code, at most 6; the sign in bit 3."""
    a = v.abs().clamp_max(6.0)
    fine = torch.round(a * 2)                               # 0 .. 4: codes 0 .. 4
    code = torch.where(a < 2, fine, torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    return code.to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)


def _blocks(x):
    """Codes [.., K] and scale bytes [.., ceil(K / 32)] of fp32 rows: 2^e with e = floor(log2(max|x|)) - 2 for every 32 columns."""
    K = x.shape[-1]
    x = torch.nn.functional.pad(x, (0, -K % 32))
    x = x.view(*x.shape[:-1], -1, 32)
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(-127, 125)
    codes = _nearest(torch.ldexp(x, -e[..., None]))
    return codes.flatten(-2)[..., :K], (e + 127).to(torch.uint8)


def _packed(codes, pitch):
    """Two codes a byte, the even column in the low half, rows of `pitch` bytes with zeros behind the codes."""
    q = torch.zeros((codes.shape[0], 2 * pitch), dtype=torch.uint8, device="cuda")
    q[:, :codes.shape[1]] = codes
    return q[:, 0::2] | (q[:, 1::2] << 4)


def _scales_held(scales, pitch):
    s = torch.zeros((scales.shape[0], pitch), dtype=torch.uint8, device="cuda")
    s[:, :scales.shape[1]] = scales
    return s


def _values(codes, scales):
    """What codes [.., K] on scales [.., ceil(K / 32)] stand for."""
    v = torch.tensor(GRID + [-t for t in GRID], device=codes.device)[codes.long()]
    return v * torch.exp2(scales.float() - 127.0).repeat_interleave(32, -1)[..., :codes.shape[-1]]


def _on_row_grids(x):
    """8-bit codes and steps of the rows of x: T = max|x|, inv = fl(127 / T), round half to even, step = fl(T / 127)."""
    T = x.abs().amax(-1, keepdim=True)
    qmax = torch.full_like(T, 127.0)                        # tensor by tensor: one division, rounded once
    inv = torch.where(T > 0, (qmax / T).clamp_max(torch.finfo(torch.float32).max), torch.zeros_like(T))
    return torch.minimum(torch.maximum(x * inv, -qmax), qmax).round_(), (T / qmax).squeeze(-1)


def _pitch(cols):
    """Bytes of a row of 4-bit codes, and of its scales."""
    return -(-cols // 256) * 128, -(-cols // 512) * 16


def _held_rows(rows, fmt):
    """Cache rows [.., D] as the pages keep them: codes and scales."""
    if fmt == "int8":
        codes, steps = _on_row_grids(rows)
        return codes.to(torch.int8), steps
    codes, scales = _blocks(rows)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales


def _given_layer(case, gen):
    M, kind, C, N, s = case["M"], case["kind"], case["C"], case["N"], _splits(case)
    w = torch.randn((N, C), device="cuda", generator=gen) * (1.0 / math.sqrt(C))
    w = torch.where(torch.rand((N, C), device="cuda", generator=gen) < 0.001, w * 10, w)
    w *= torch.rand((N, 1), device="cuda", generator=gen) + 0.5             # output channels of different ranges
    src, depth = _lists(w.abs().amax(0), C, s)
    w = w[:, src.long()] * torch.exp2(-depth.float())
    codes, scales = _blocks(w)
    Ke = C + s
    pitch, spitch = _pitch(Ke)
    got = dict(src=src, wq=_packed(codes, pitch), ws=_scales_held(scales, spitch), Ke=Ke, pitch=pitch, spitch=spitch)
    if kind == "product":
        codes, scales = _blocks(_hidden(M, C, gen, "float32")[:, src.long()])
        got["xq"], got["xs"] = _packed(codes, pitch), _scales_held(scales, spitch)
    else:
        got["x"] = _hidden(M, C, gen, case["dtype"])
    got["bias"] = torch.randn((N,), device="cuda", generator=gen) if case["bias"] else None
    return got


def _given_cache(case, gen, seed):
    B, H, D, P = case["B"], case["H"], case["D"], case["P"]
    held, new = _lengths(case)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed))).tolist()
    held, new = [held[b] for b in order], [new[b] for b in order]
    cols = -(-max(held) // P) + 1                           # one column more than the longest needs
    need = [-(-L // P) for L in held]
    pages = sum(need) + 2
    table = torch.full((B, cols), -1, dtype=torch.int32)
    loose = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed) + 1)).to(torch.int32)
    used = torch.arange(cols)[None, :] < torch.tensor(need)[:, None]
    table[used] = loose[:sum(need)]
    # keys: one channel in thirty far larger than the others, as they are found; values: rows of different sizes
    big = torch.where(torch.rand((2, H, D), device="cuda", generator=gen) < torch.tensor([0.03, 0.0], device="cuda")[:, None, None],
                      9.0, 1.0)
    depth = torch.where(big > 1, 3, 0).to(torch.int32) if case["halved"] else None

    def rows(which, lead):
        x = torch.randn(lead + (H, D), device="cuda", generator=gen) * big[which]
        return x * (torch.rand(lead + (H, 1), device="cuda", generator=gen) + 0.5)

    got = dict(table=table.cuda(), cu=torch.tensor([0] + new).cumsum(0).to(torch.int32).cuda(), pages=pages, T=sum(new),
               starts=torch.tensor([L - n for L, n in zip(held, new)], dtype=torch.int32).cuda(), most=max(held), most_new=max(new))
    if depth is not None:
        got["kdepth"], got["vdepth"] = depth[0].contiguous(), depth[1].contiguous()
    else:
        got["kdepth"] = got["vdepth"] = None

    def into_pages(which, d):
        x = rows(which, (pages * P,))
        if d is not None:
            x *= torch.exp2(-d.float())
        codes, scales = _held_rows(x.view(pages, P, H, D).transpose(1, 2).contiguous(), case["fmt"])
        return codes, scales

    got["keys"], got["kscales"] = into_pages(0, got["kdepth"])
    got["values"], got["vscales"] = into_pages(1, got["vdepth"])
    dtype = getattr(torch, case["dtype"])
    if case["kind"] == "cache":
        got["newk"], got["newv"] = rows(0, (got["T"],)).to(dtype), rows(1, (got["T"],)).to(dtype)
        if case["back"] == "all":
            got["back_cu"] = torch.tensor([0] + held).cumsum(0).to(torch.int32).cuda()
            got["back_starts"], got["back"] = torch.zeros_like(got["starts"]), sum(held)
        else:
            got["back_cu"], got["back_starts"], got["back"] = got["cu"], got["starts"], got["T"]
    else:
        q = torch.randn((got["T"], H * case["G"], D), device="cuda", generator=gen)
        q *= torch.exp2(4 * torch.rand((got["T"], H * case["G"], 1), device="cuda", generator=gen) - 2)   # flat rows and sharp ones
        got["q"] = q.to(dtype)
    return got


def _given(case, seed):
    """The inputs of a case, made from the seed alone."""
    gen = _gen(seed)
    if case["kind"] == "quantize":
        M, C, g, s = case["M"], case["C"], case["g"], _splits(case)
        x = _hidden(M, C * g, gen, case["dtype"])
        src, depth = _lists(x.float().abs().amax(0).view(C, g).amax(1), C, s)
        return dict(x=x, src=src, depth=depth if case["halved"] else None, Ke=(C + s) * g)
    if case["kind"] in ("product", "forward"):
        return _given_layer(case, gen)
    return _given_cache(case, gen, seed)


def prepare(case, seed):
    state = dict(case, **_given(case, seed))
    kind, dtype = case["kind"], getattr(torch, case["dtype"])
    # what a program keeps beside its inputs: the buffers that its calls write to
    if kind in ("quantize", "forward"):
        pitch, spitch = _pitch(state["Ke"])
        state["codes"] = torch.empty((case["M"], pitch), dtype=torch.uint8, device="cuda")
        state["scales"] = torch.empty((case["M"], spitch), dtype=torch.uint8, device="cuda")
    if kind == "quantize":
        out = torch.float32 if case["dtype"] == "float32" else torch.bfloat16
        state["y"] = torch.empty((case["M"], state["Ke"]), dtype=out, device="cuda")
    if kind in ("product", "forward"):
        state["y"] = torch.empty((case["M"], case["N"]), dtype=dtype, device="cuda")
    if kind == "cache":
        state["backk"] = torch.empty((state["back"], case["H"], case["D"]), dtype=dtype, device="cuda")
        state["backv"] = torch.empty_like(state["backk"])
    if kind == "attend":
        state["y"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty(state["q"].shape[:2], device="cuda")
        state["workspace"] = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    return state


# ---- the plain forms -------------------------------------------------------------------------


def _plain_expanded(x, src, depth, g):
    cols = (src.long()[:, None] * g + torch.arange(g, device=x.device)).reshape(-1)
    x = x.float()[:, cols]
    return x if depth is None else x * torch.exp2(-depth.float()).repeat_interleave(g)


def _unpacked(q, cols):
    return torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :cols]


def _plain_product(x, st):
    w = _values(_unpacked(st["wq"], st["Ke"]), st["ws"][:, :-(-st["Ke"] // 32)])
    y = x @ w.t()
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(getattr(torch, st["dtype"]))


def _plain_rows(codes, scales, depth, fmt):
    """Cache rows [.., H, D] as numbers."""
    v = codes.float() * scales[..., None] if fmt == "int8" else _values(_unpacked(codes, 2 * codes.shape[-1]), scales)
    return v if depth is None else v * torch.exp2(depth.float())


def _plain_cache(st):
    dtype, P, fmt = getattr(torch, st["dtype"]), st["P"], st["fmt"]
    seq = torch.repeat_interleave(torch.arange(st["B"], device="cuda"), st["back_cu"].diff().long(), output_size=st["back"])
    pos = torch.arange(st["back"], device="cuda") - st["back_cu"].long()[seq] + st["back_starts"].long()[seq]
    page = st["table"].long()[seq, pos // P]
    # row of the new tokens, where it is one
    at = pos - st["starts"].long()[seq] + st["cu"].long()[seq]
    new = pos >= st["starts"].long()[seq]
    at = torch.where(new, at, 0)

    def back(fresh, codes, scales, depth):
        x = fresh.float() if depth is None else fresh.float() * torch.exp2(-depth.float())
        x = _plain_rows(*_held_rows(x, fmt), depth, fmt)
        if st["back"] == st["T"]:
            return x.to(dtype)
        old = _plain_rows(codes[page, :, pos % P], scales[page, :, pos % P], depth, fmt)
        return torch.where(new[:, None, None], x[at], old).to(dtype)

    return dict(keys=back(st["newk"], st["keys"], st["kscales"], st["kdepth"]),
                values=back(st["newv"], st["values"], st["vscales"], st["vdepth"]))


def _plain_attend(st):
    B, G, H, D, P, L, n = st["B"], st["G"], st["H"], st["D"], st["P"], st["most"], st["most_new"]
    dev = st["q"].device
    j = torch.arange(L, device=dev)
    page = st["table"].long()[:, j // P]                    # [B, L]
    there = page >= 0
    page = torch.where(there, page, 0)
    row = (j % P)[None, :].expand(B, L)
    k = _plain_rows(st["keys"][page, :, row], st["kscales"][page, :, row], st["kdepth"], st["fmt"]).transpose(1, 2)
    v = _plain_rows(st["values"][page, :, row], st["vscales"][page, :, row], st["vdepth"], st["fmt"]).transpose(1, 2)
    new = st["cu"].diff().long()
    i = torch.arange(n, device=dev)
    real = i[None, :] < new[:, None]                        # [B, n]
    token = torch.where(real, st["cu"].long()[:B, None] + i, 0)
    q = st["q"].float()[token].view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    s = (q * (1.0 / math.sqrt(D))) @ k.transpose(2, 3).contiguous()
    pos = st["starts"].long()[:, None] + i                  # [B, n]
    sees = there[:, None, :] & (j <= pos[:, :, None])
    if st["window"]:
        sees = sees & (j > pos[:, :, None] - st["window"])
    sees = sees[:, None, :, None, :].expand(B, 1, n, G, L).reshape(B, 1, n * G, L)
    s = s.masked_fill_(~sees, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isneginf(top), 0.0, top)
    s = s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    y = (s @ v) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)

    def in_order(t):                                        # [B, H, n * G, ..] to the tokens' rows
        t = t.view(B, H, n, G, -1).permute(0, 2, 1, 3, 4).reshape(B, n, H * G, -1)
        return t[real]

    return dict(y=in_order(y).to(st["q"].dtype), lse=in_order(lse).squeeze(-1))


def _plain(st):
    kind = st["kind"]
    if kind == "quantize":
        out = _values(*_blocks(_plain_expanded(st["x"], st["src"], st["depth"], st["g"])))
        return out if st["dtype"] == "float32" else out.to(torch.bfloat16)
    if kind == "product":
        return _plain_product(_values(_unpacked(st["xq"], st["Ke"]), st["xs"][:, :-(-st["Ke"] // 32)]), st)
    if kind == "forward":
        return _plain_product(_values(*_blocks(_plain_expanded(st["x"], st["src"], None, 1))), st)
    return _plain_cache(st) if kind == "cache" else _plain_attend(st)


# ---- one pass --------------------------------------------------------------------------------


def run(st):
    if not own:
        return _plain(st)
    from paper_1901_09504_amd import binding as B

    kind = st["kind"]
    if kind == "quantize":
        M, g, x, Ke = st["M"], st["g"], st["x"], st["Ke"]
        B.ocs_split_quantize_mx(x, M, st["C"], g, x.stride(0), st["src"], st["depth"], Ke // g - st["C"], st["codes"],
                                st["codes"].stride(0), st["scales"], st["scales"].stride(0))
        B.ocs_dequantize_mx(st["codes"], st["codes"].stride(0), st["scales"], st["scales"].stride(0), M, Ke, st["y"], Ke)
        return st["y"]
    if kind == "product":
        B.ocs_qgemm_mx(st["xq"], st["pitch"], st["xs"], st["spitch"], st["wq"], st["pitch"], st["ws"], st["spitch"], st["M"], st["N"],
                       st["Ke"], st["bias"], st["y"], st["N"])
        return st["y"]
    if kind == "forward":
        B.ocs_forward_mx(st["x"], st["M"], st["C"], 1, st["x"].stride(0), st["src"], st["Ke"] - st["C"], st["codes"], st["pitch"],
                         st["scales"], st["spitch"], st["wq"], st["pitch"], st["ws"], st["spitch"], st["N"], st["bias"],
                         st["y"], st["N"])
        return st["y"]
    table, fmt = st["table"], B.CACHE_INT8 if st["fmt"] == "int8" else B.CACHE_MX4
    cache = (table, table.shape[1], table.stride(0), fmt, st["keys"], st["kscales"], st["values"], st["vscales"], st["pages"], st["P"],
             st["H"], st["D"], st["kdepth"], st["vdepth"])
    if kind == "cache":
        k, v, bk, bv = st["newk"], st["newv"], st["backk"], st["backv"]
        B.ocs_cache_write(k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1), st["T"], st["cu"], st["starts"], st["B"], *cache)
        B.ocs_cache_read(bk, bk.stride(0), bk.stride(1), bv, bv.stride(0), bv.stride(1), st["back"], st["back_cu"],
                         st["back_starts"], st["B"], *cache)
        return dict(keys=bk, values=bv)
    q, y = st["q"], st["y"]
    B.ocs_cache_attention(q, q.stride(0), q.stride(1), q.shape[1], st["T"], st["cu"], st["starts"], st["B"], st["most"], *cache,
                          1.0 / math.sqrt(st["D"]), st["window"], y, y.stride(0), y.stride(1), st["lse"], st["workspace"])
    return dict(y=y, lse=st["lse"])


# ---- the definitions in 64 bits --------------------------------------------------------------


def _exact_blocks(x):
    """Values of 64-bit rows on their blocks' grids: the nearest number of the grid times the block's power of two."""
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    K = x.shape[-1]
    wide = torch.zeros(x.shape[:-1] + (-(-K // 32) * 32,), dtype=torch.float64, device=x.device)
    wide[..., :K] = x
    wide = wide.unflatten(-1, (-1, 32))
    most = wide.abs().max(-1, keepdim=True).values
    scale = torch.ones_like(most)
    scale[most > 0] = 2.0 ** (torch.floor(torch.log2(most[most > 0])) - 2)
    # log2 of a number just below a power of two may round up to it
    scale = torch.where(most / scale < 4, scale / 2, scale)
    scale[most == 0] = 1
    a = (wide / scale).abs()
    above = torch.bucketize(a, (grid[1:] + grid[:-1]) / 2, right=False)      # a tie falls to the lower code ...
    tie = (a == ((grid[1:] + grid[:-1]) / 2)[above.clamp_max(6)]) & (above < 7) & (above % 2 == 1)
    return (torch.sign(wide) * grid[above + tie.to(above.dtype)] * scale).flatten(-2)[..., :K]    # ... unless that is odd


def _exact_held(codes, scales, cols):
    """64-bit values of packed codes on their scales."""
    low, high = codes.remainder(16).to(torch.int64), codes.div(16, rounding_mode="floor").to(torch.int64)
    both = torch.stack((low, high), dim=-1).reshape(*codes.shape[:-1], -1)[..., :cols]
    size = torch.tensor(GRID, dtype=torch.float64, device=codes.device)[both.remainder(8)]
    block = torch.arange(cols, device=codes.device).div(32, rounding_mode="floor")
    return torch.where(both >= 8, -size, size) * 2.0 ** (scales.to(torch.float64) - 127)[..., block]


def _exact_grid(x):
    """Eq. 1 over the last dimension: the grid's two numbers and the scaled value are 32-bit numbers by definition."""
    def fl(t):
        return t.to(torch.float32).to(torch.float64)

    T = x.abs().max(-1, keepdim=True).values
    factor = fl(torch.full_like(T, 127) / T)
    factor[T == 0] = 0
    return torch.round(fl(x * factor)).clamp(-127, 127) * fl(T / 127)


def _exact_page_rows(st, which, page, row):
    codes, scales = st[which + "s" if which == "key" else "values"][page, :, row], st[which[0] + "scales"][page, :, row]
    if st["fmt"] == "int8":
        x = codes.to(torch.float64) * scales.to(torch.float64)[..., None]
    else:
        x = _exact_held(codes, scales, st["D"])
    d = st[which[0] + "depth"]
    return x if d is None else x * 2.0 ** d.to(torch.float64)


def exact(case, seed):
    st = dict(case, **_given(case, seed))
    kind = case["kind"]
    if kind == "quantize":
        v = st["x"].to(torch.float64).unflatten(1, (case["C"], case["g"]))[:, st["src"].to(torch.int64)]
        if st["depth"] is not None:
            v = v / (2.0 ** st["depth"].to(torch.float64))[None, :, None]
        return _exact_blocks(v.flatten(1))
    if kind in ("product", "forward"):
        w = _exact_held(st["wq"], st["ws"], st["Ke"])
        if kind == "product":
            x = _exact_held(st["xq"], st["xs"], st["Ke"])
        else:
            x = _exact_blocks(st["x"].to(torch.float64)[:, st["src"].to(torch.int64)])
        y = torch.matmul(x, w.t())
        if st["bias"] is not None:
            y += st["bias"].to(torch.float64)
        return y
    cu, starts, table = st["cu"].tolist(), st["starts"].tolist(), st["table"].to(torch.int64)
    P = case["P"]
    if kind == "cache":
        def fresh(rows, d):
            x = rows.to(torch.float64)
            x = x if d is None else x / 2.0 ** d.to(torch.float64)
            x = _exact_grid(x) if case["fmt"] == "int8" else _exact_blocks(x)
            return x if d is None else x * 2.0 ** d.to(torch.float64)

        out = dict(keys=fresh(st["newk"], st["kdepth"]), values=fresh(st["newv"], st["vdepth"]))
        if case["back"] == "new":
            return out
        whole = dict(keys=[], values=[])
        for b in range(case["B"]):
            old = torch.arange(starts[b], device="cuda")
            for name, which in (("keys", "key"), ("values", "value")):
                whole[name].append(_exact_page_rows(st, which, table[b, old // P], old % P))
                whole[name].append(out[name][cu[b]:cu[b + 1]])
        return {name: torch.cat(v) for name, v in whole.items()}
    if work(case)["flops"] > 4e11:
        return None
    ys, lses = [], []
    for b in range(case["B"]):
        n, at = cu[b + 1] - cu[b], starts[b]
        seen = torch.arange(at + n, device="cuda")
        k = _exact_page_rows(st, "key", table[b, seen // P], seen % P)       # [L, H, D]
        v = _exact_page_rows(st, "value", table[b, seen // P], seen % P)
        y = torch.empty((n, case["H"] * case["G"], case["D"]), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, case["H"] * case["G"]), dtype=torch.float64, device="cuda")
        hidden = seen[None, :] > (at + torch.arange(n, device="cuda"))[:, None]
        if case["window"]:
            hidden |= seen[None, :] + case["window"] <= (at + torch.arange(n, device="cuda"))[:, None]
        for h in range(case["H"] * case["G"]):
            w = torch.mv if n == 1 else torch.mm
            kh, vh, qh = k[:, h // case["G"]], v[:, h // case["G"]], st["q"][cu[b]:cu[b + 1], h].to(torch.float64)
            s = (w(kh, qh[0])[None] if n == 1 else torch.mm(qh, kh.t())) / math.sqrt(case["D"])
            s[hidden] = -math.inf
            lse[:, h] = torch.logsumexp(s, 1)
            y[:, h] = torch.mm(torch.exp(s - lse[:, h:h + 1]), vh)
        ys.append(y)
        lses.append(lse)
    return dict(y=torch.cat(ys), lse=torch.cat(lses))
