"""Microscaled 4-bit grids on the GPU: codes and scale bytes bit for bit against 64-bit definitions, products exactly where sums are whole
numbers of 24 bits and within the roundings of a 32-bit sum elsewhere; edges, strides, alignments, NaN, streams and graphs."""
import math

import numpy as np
import pytest
import torch

from paper_1901_09504_amd import binding as B
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NUMBERS = np.concatenate([MAGNITUDES, -MAGNITUDES])


@pytest.fixture(autouse=True)
def _gpu():
    G.require_gpu()


def lists(rng, C, s):
    """Sources and halvings as a selection leaves them: some channels split again and again."""
    src, depth = list(range(C)), [0] * C
    for _ in range(s):
        j = int(rng.integers(0, len(src))) if rng.random() < 0.7 else len(src) - 1
        depth[j] += 1
        src.append(src[j])
        depth.append(depth[j])
    return np.array(src, dtype=np.int32), np.array(depth, dtype=np.int32)


def on_grids(x):
    """fp32 rows [M, K] -> codes [M, K], scale bytes [M, blocks]: the definition in 64 bits, one block after the other."""
    M, K = x.shape
    codes, scales = np.zeros((M, K), np.uint8), np.zeros((M, -(-K // 32)), np.uint8)
    for b in range(scales.shape[1]):
        v = x[:, 32 * b:32 * b + 32].astype(np.float64)
        finite = np.isfinite(v).all(1)
        a = np.abs(np.where(np.isfinite(v), v, 0.0)).max(1)
        e = np.where(a > 0, np.frexp(np.where(a > 0, a, 1.0))[1] - 3, -127).clip(-127, None)
        scaled = np.where(finite[:, None], v, 0.0) * np.ldexp(1.0, -e)[:, None]
        far = np.abs(np.abs(scaled)[:, :, None] - MAGNITUDES)
        near = far.min(2, keepdims=True) == far                              # two of them at a tie: the even one
        code = np.where(near[:, :, 0::2].any(2), near[:, :, 0::2].argmax(2) * 2, near[:, :, 1::2].argmax(2) * 2 + 1)
        code = np.where(np.abs(scaled) >= 6, 7, code)
        codes[:, 32 * b:32 * b + 32] = np.where(finite[:, None], code | (np.signbit(v) * 8), 0)
        scales[:, b] = np.where(finite, e + 127, 255)
    return codes, scales


def packed(codes, pitch):
    q = np.zeros((codes.shape[0], 2 * pitch), np.uint8)
    q[:, :codes.shape[1]] = codes
    return q[:, 0::2] | (q[:, 1::2] << 4)


def numbers(codes, scales):
    """64-bit numbers of codes [.., K] on scale bytes [.., blocks]."""
    size = np.ldexp(1.0, scales.astype(np.int64) - 127)
    size = np.where(scales == 255, np.nan, size)
    return NUMBERS[codes] * np.repeat(size, 32, -1)[..., :codes.shape[-1]]


def expanded(x, C, g, src, depth):
    v = x[:, :C * g].float().cpu().numpy().reshape(x.shape[0], C, g)[:, src, :]
    if depth is not None:
        v = (v * np.ldexp(np.float32(1), -depth.astype(np.int64)).astype(np.float32)[None, :, None]).astype(np.float32)
    return np.ascontiguousarray(v.reshape(x.shape[0], -1), dtype=np.float32)


def quantized(x, C, g, src, depth, s, more=0):
    """The call's codes and scales, pads included, into buffers that hold rubbish; more: 16s of bytes behind the needed pitches."""
    M, cols = x.shape[0], (C + s) * g
    ldq, lds = -(-cols // 32) * 16 + 16 * more, B.ocs_mx_scale_pitch(cols) + 16 * more
    q = torch.full((M, ldq), 0x77, dtype=torch.uint8, device="cuda")
    sc = torch.full((M, lds), 0x55, dtype=torch.uint8, device="cuda")
    B.ocs_split_quantize_mx(x, M, C, g, x.stride(0), None if src is None else G.dev(src), None if depth is None else G.dev(depth), s, q,
                            ldq, sc, lds)
    return q, sc


def check_quantized(x, C, g, src, depth, s, more=0):
    q, sc = quantized(x, C, g, src, depth, s, more)
    codes, scales = on_grids(expanded(x, C, g, np.arange(C) if src is None else src, depth))
    want = np.zeros(tuple(sc.shape), np.uint8)
    want[:, :scales.shape[1]] = scales
    assert np.array_equal(G.host(sc), want)
    assert np.array_equal(G.host(q), packed(codes, q.shape[1]))
    return q, sc, codes, scales


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,C,g,s", [(1, 1, 1, 0), (3, 1, 1, 2), (5, 31, 1, 1), (7, 32, 1, 3), (64, 256, 1, 13), (9, 255, 1, 11),
                                     (4, 3, 49, 1), (3, 511, 1, 0), (5, 513, 1, 30), (2, 1001, 1, 51), (3, 64, 9, 4), (2, 3000, 1, 150),
                                     (1, 7900, 1, 100), (300, 70, 1, 5)])
@pytest.mark.parametrize("halved", [False, True])
def test_codes_and_scales_are_those_of_the_definition(dtype, M, C, g, s, halved):
    rng = np.random.default_rng(M * 7919 + C * 31 + g + s)
    x = rng.standard_normal((M, C * g)).astype(np.float32) * np.exp2(rng.integers(-12, 5, (M, C * g))).astype(np.float32)
    src, depth = lists(rng, C, s)
    check_quantized(torch.from_numpy(x).to(dtype).cuda(), C, g, src, depth if halved else None, s, more=C % 3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_ties_borders_and_zeros(dtype):
    """Every half step between two numbers and its neighbours, on scales from the smallest to the largest that the type has."""
    steps = np.arange(0, 65) * 0.125
    exps = {F32: range(-149, 126, 5), BF16: range(-130, 126, 5), F16: range(-24, 13)}[dtype]
    rows = []
    for e in exps:
        for part in (steps[:31], steps[31:62], -steps[34:]):
            rows.append(np.concatenate([[4.0], part, np.zeros(31 - len(part))]) * 2.0 ** e)
    rows += [np.zeros(32), np.full(32, -0.0), np.full(32, 7.9375), np.full(32, 2.0 ** -14)]
    x = torch.from_numpy(np.array(rows)).to(dtype).cuda()                    # (what the type cannot hold is rounded before the call)
    check_quantized(x, 32, 1, None, None, 0)
    if dtype == F32:
        up = torch.nextafter(x, torch.full_like(x, torch.inf))
        check_quantized(up, 32, 1, None, None, 0)
        check_quantized(torch.nextafter(x, torch.full_like(x, -torch.inf)), 32, 1, None, None, 0)
        check_quantized(torch.full((2, 40), torch.finfo(F32).max, device="cuda"), 40, 1, None, None, 0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("bad", [torch.nan, torch.inf, -torch.inf])
def test_a_block_with_nan_or_infinity_says_so_and_leaves_the_others(dtype, bad):
    x = torch.randn((5, 100), generator=torch.Generator().manual_seed(3)).to(dtype)
    x[1, 40], x[3, 99], x[4, 0] = bad, bad, bad
    q, sc, codes, scales = check_quantized(x.cuda(), 100, 1, None, None, 0)
    assert (scales == 255).sum() == 3
    y = torch.empty((5, 100), device="cuda")
    B.ocs_dequantize_mx(q, q.shape[1], sc, sc.shape[1], 5, 100, y, 100)
    assert np.array_equal(G.host(y), numbers(codes, scales).astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_any_pitch_and_alignment_of_rows(dtype):
    for off, ld, C in ((1, 77, 70), (3, 131, 131), (2, 64, 33)):
        buf = torch.randn(20 * ld + 8, device="cuda").to(dtype)
        x = buf[off:off + 20 * ld].view(20, ld)
        check_quantized(x, C, 1, None, None, 0)


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("M,cols", [(1, 1), (7, 31), (3, 32), (5, 100), (2, 4099), (130, 257)])
def test_numbers_of_codes(out, M, cols):
    rng = np.random.default_rng(M + cols)
    codes = rng.integers(0, 16, (M, cols)).astype(np.uint8)
    scales = rng.integers(0, 255, (M, -(-cols // 32))).astype(np.uint8)
    ldq, lds = B.ocs_mx_code_pitch(cols), B.ocs_mx_scale_pitch(cols)
    sc = np.zeros((M, lds), np.uint8)
    sc[:, :scales.shape[1]] = scales
    y = torch.full((M, cols + 3), 9.0, dtype=out, device="cuda")
    B.ocs_dequantize_mx(G.dev(packed(codes, ldq)), ldq, G.dev(sc), lds, M, cols, y, cols + 3)
    want = torch.from_numpy(numbers(codes, scales)).to(out)                  # one rounding; exact in bf16 and fp32
    assert torch.equal(y[:, :cols].cpu(), want) and bool((y[:, cols:] == 9).all())


# ---- the product -----------------------------------------------------------------------------

def operands(rng, M, N, K, spread, pitch=0):
    """Codes and scales of both operands on the device, and the 64-bit numbers they stand for."""
    got = []
    for rows in (M, N):
        codes = rng.integers(0, 16, (rows, K)).astype(np.uint8)
        scales = rng.integers(127 - spread, 128 + spread, (rows, -(-K // 32))).astype(np.uint8)
        ldq, lds = max(B.ocs_mx_code_pitch(K) + 16 * pitch, -(-K // 32) * 16), B.ocs_mx_scale_pitch(K)
        sc = np.zeros((rows, lds), np.uint8)
        sc[:, :scales.shape[1]] = scales
        got += [G.dev(packed(codes, ldq)), G.dev(sc), numbers(codes, scales)]
    return got


def product(xq, xs, wq, ws, K, bias, out, ldy=None, off=0, stream=None):
    M, N = xq.shape[0], wq.shape[0]
    ldy = N if ldy is None else ldy
    buf = torch.full((M * ldy + off + 8,), 7.0, dtype=out, device="cuda")
    y = buf[off:off + M * ldy].view(M, ldy)
    B.ocs_qgemm_mx(xq, xq.shape[1], xs, xs.shape[1], wq, wq.shape[1], ws, ws.shape[1], M, N, K, bias, y, ldy, stream)
    assert bool((buf[:off] == 7).all()) and bool((y[:, N:] == 7).all()) and bool((buf[off + M * ldy:] == 7).all())
    return y[:, :N]


SHAPES = [(1, 1, 1), (1, 16, 32), (3, 17, 33), (16, 100, 256), (17, 33, 500), (32, 16, 1000), (1, 6000, 3150), (20, 500, 3150), (33, 70, 257),
          (64, 64, 2000), (65, 129, 512), (100, 2049, 1052), (128, 128, 64), (333, 2049, 1052), (300, 1000, 777), (513, 1030, 513),
          (2050, 1500, 300), (1030, 4100, 260)]


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products_are_exact_where_32_bits_hold_the_sums(out, M, N, K):
    """On one scale every product is a multiple of 1/4 and at most 36, so sums of K < 2^24 / 144 of them are exact in fp32."""
    rng = np.random.default_rng(M * 131 + N * 17 + K)
    xq, xs, x, wq, ws, w = operands(rng, M, N, K, 0, pitch=K % 2)
    y = product(xq, xs, wq, ws, K, None, out, ldy=N + M % 3, off=M % 2)
    want = torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().t()
    assert torch.equal(y, want.to(F32).to(out))


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products_on_scales_of_their_own_with_a_bias(M, N, K):
    """K + 1 additions in 32 bits, each off by a step of what has been added up (2^-23, whichever way it rounds)."""
    rng = np.random.default_rng(M + N + K)
    xq, xs, x, wq, ws, w = operands(rng, M, N, K, 6)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(N)).cuda()
    x, w = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    want, size = x @ w.t() + bias.double(), x.abs() @ w.abs().t() + bias.double().abs()
    for out in (F32, BF16, F16):
        y = product(xq, xs, wq, ws, K, bias, out).double()
        tol = (K + 1) * 2.0 ** -23 * size + HALF_STEP[out] * want.abs() + (2.0 ** -25 if out == F16 else 0)
        big = want.abs() > 65504 if out == F16 else torch.zeros_like(want, dtype=torch.bool)
        assert bool((((y - want).abs() <= tol * (1 + HALF_STEP[out])) | big).all())


def test_scales_at_the_ends_and_nan():
    rng = np.random.default_rng(5)
    for M, N in ((5, 40), (200, 300)):
        xq, xs, _, wq, ws, _ = operands(rng, M, N, 700, 0)
        xs.fill_(7)                                                          # 2^-120 times 2^120
        ws.fill_(247)
        y = product(xq, xs, wq, ws, 700, None, F32)
        xs.fill_(127)
        ws.fill_(127)
        assert torch.equal(y, product(xq, xs, wq, ws, 700, None, F32))
        xs[3, 21], ws[N - 1, 0] = 255, 255
        z = product(xq, xs, wq, ws, 700, None, F32)
        assert bool(z[3].isnan().all()) and bool(z[:, N - 1].isnan().all())
        z[3], z[:, N - 1], y[3], y[:, N - 1] = 0, 0, 0, 0
        assert torch.equal(z, y)


# ---- the layer per batch ---------------------------------------------------------------------

def forward(x, C, g, src, s, wq, ws, N, bias, out, more=0, stream=None):
    M, cols = x.shape[0], (C + s) * g
    ldq, lds = B.ocs_mx_code_pitch(cols) + 16 * more, B.ocs_mx_scale_pitch(cols) + 16 * more
    q = torch.full((M, ldq), 0x77, dtype=torch.uint8, device="cuda")
    sc = torch.full((M, lds), 0x55, dtype=torch.uint8, device="cuda")
    y = torch.full((M, N), 7.0, dtype=out, device="cuda")
    B.ocs_forward_mx(x, M, C, g, x.stride(0), src, s, q, ldq, sc, lds, wq, wq.shape[1], ws, ws.shape[1], N, bias, y, N, stream)
    return q, sc, y


@pytest.mark.parametrize("dtype,out", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("M,C,g,s,N", [(1, 1, 1, 0, 1), (1, 3000, 1, 150, 6000), (2, 33, 1, 2, 50), (16, 257, 1, 13, 100), (5, 30, 9, 2, 33),
                                       (17, 1001, 1, 51, 500), (40, 1001, 1, 51, 2049), (300, 500, 1, 25, 700), (16, 31, 1, 0, 5000)])
def test_a_layer_is_its_codes_and_their_product(dtype, out, M, C, g, s, N):
    rng = np.random.default_rng(M + C + N)
    src, _ = lists(rng, C, s)
    x = torch.from_numpy(rng.standard_normal((M, C * g + 3)).astype(np.float32)).to(dtype).cuda()
    K = (C + s) * g
    _, _, _, wq, ws, w = operands(rng, 1, N, K, 2)
    bias = torch.randn(N, device="cuda")
    q, sc, y = forward(x, C, g, G.dev(src) if s else None, s, wq, ws, N, bias, out, more=M % 2)
    codes, scales = on_grids(expanded(x, C, g, src, None))
    assert np.array_equal(G.host(q), packed(codes, q.shape[1]))
    assert np.array_equal(G.host(sc)[:, :scales.shape[1]], scales) and not G.host(sc)[:, scales.shape[1]:].any()
    v, w = torch.from_numpy(numbers(codes, scales)).cuda(), torch.from_numpy(w).cuda()
    want, size = v @ w.t() + bias.double(), v.abs() @ w.abs().t() + bias.double().abs()
    assert bool(((y.double() - want).abs() <= (K + 1) * 2.0 ** -23 * size + HALF_STEP[out] * want.abs()).all())


def test_a_layer_in_place_reads_its_rows_before_it_writes():
    C = N = 64
    rng = np.random.default_rng(1)
    _, _, _, wq, ws, _ = operands(rng, 1, N, C, 2)
    x = torch.randn((4, C), device="cuda")
    q = torch.empty((4, 128), dtype=torch.uint8, device="cuda")
    sc = torch.empty((4, 16), dtype=torch.uint8, device="cuda")
    _, _, want = forward(x, C, 1, None, 0, wq, ws, N, None, F32)
    B.ocs_forward_mx(x, 4, C, 1, C, None, 0, q, 128, sc, 16, wq, wq.shape[1], ws, ws.shape[1], N, None, x, N)
    assert torch.equal(x, want)


def test_bad_sources_do_not_fault():
    x = torch.randn((3, 40), device="cuda")
    src = torch.arange(43, dtype=torch.int32, device="cuda")
    src[40:] = torch.tensor([-5, 1 << 30, 7], dtype=torch.int32)
    q, sc = quantized(x, 40, 1, None, None, 0)
    rng = np.random.default_rng(2)
    _, _, _, wq, ws, _ = operands(rng, 1, 10, 43, 2)
    _, _, y = forward(x, 40, 1, src, 3, wq, ws, 10, None, F32)
    src[40:] = torch.tensor([0, 39, 7], dtype=torch.int32)
    assert torch.equal(y, forward(x, 40, 1, src, 3, wq, ws, 10, None, F32)[2])


@pytest.mark.parametrize("M", [3, 100])
def test_streams_and_graphs(M):
    """A captured layer replayed on new inputs, with eager calls of other sizes between the replays."""
    C, N = 300, 400
    rng = np.random.default_rng(M)
    _, _, _, wq, ws, _ = operands(rng, 1, N, C, 2)
    x = torch.randn((M, C), device="cuda")
    side = torch.cuda.Stream()
    q = torch.empty((M, B.ocs_mx_code_pitch(C)), dtype=torch.uint8, device="cuda")
    sc = torch.empty((M, B.ocs_mx_scale_pitch(C)), dtype=torch.uint8, device="cuda")
    y = torch.empty((M, N), device="cuda")
    side.wait_stream(torch.cuda.current_stream())

    def call():
        B.ocs_forward_mx(x, M, C, 1, C, None, 0, q, q.shape[1], sc, sc.shape[1], wq, wq.shape[1], ws, ws.shape[1], N, None, y, N)

    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        x.copy_(torch.randn((M, C), generator=torch.Generator().manual_seed(seed)))
        y.fill_(5.0)
        graph.replay()
        got = y.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, forward(x, C, 1, None, 0, wq, ws, N, None, F32)[2])


# ---- the layer that keeps its buffers --------------------------------------------------------

@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("N,C,r,g", [(50, 64, 0.05, 1), (300, 500, 0.1, 1), (33, 40, 0.0, 9), (700, 1001, 0.02, 1), (1, 1, 0.0, 1)])
def test_layers_from_their_weights(out, N, C, r, g):
    """prepare_weights: channels chosen on the tensor, halved, put on their grids; forward: codes of the batch, product and bias."""
    from oracle import ref
    from paper_1901_09504_amd.layer import MxLayer

    rng = np.random.default_rng(N + C)
    W = rng.standard_normal((N, C * g)).astype(np.float32)
    W[:, :g] *= 7
    bias = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda()
    layer = MxLayer(N, C, r, g, out_dtype=out)
    layer.prepare_weights(torch.from_numpy(W).cuda(), bias)
    s, K = layer.s, layer.Ke
    if s:
        sel = ref.split_weights(W, C, g, s)
        src, depth = sel["chan_src"], sel["chan_depth"]
        assert np.array_equal(G.host(layer.chan_src), src) and np.array_equal(G.host(layer.chan_depth), depth)
    else:
        src, depth = np.arange(C, dtype=np.int32), None
    codes, scales = on_grids(expanded(torch.from_numpy(W), C, g, src, depth))
    assert np.array_equal(G.host(layer.Wq), packed(codes, layer.ldq)) and np.array_equal(G.host(layer.step_w)[:, :scales.shape[1]], scales)
    w = torch.from_numpy(numbers(codes, scales)).cuda()
    for M in (1, 5, 40, 3, 0):
        x = torch.from_numpy(rng.standard_normal((M, C * g)).astype(np.float32)).cuda()
        y = layer.forward(x)
        assert y.shape == (M, N) and y.dtype == out
        if M:
            codes, scales = on_grids(expanded(x, C, g, src, None))
            v = torch.from_numpy(numbers(codes, scales)).cuda()
            want, size = v @ w.t() + bias.double(), v.abs() @ w.abs().t() + bias.double().abs()
            assert bool(((y.double() - want).abs() <= (K + 1) * 2.0 ** -23 * size + HALF_STEP[out] * want.abs()).all())


def test_a_layer_on_streams_and_in_a_graph():
    from paper_1901_09504_amd.layer import MxLayer

    W = torch.randn((200, 300), device="cuda")
    layer = MxLayer(200, 300, 0.05, max_rows=4)
    layer.prepare_weights(W)
    x = torch.randn((4, 300), device="cuda")
    want = layer.forward(x).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = layer.forward(x, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.forward(x)
    big = torch.randn((50, 300), device="cuda")
    for seed in range(3):
        x.copy_(torch.randn((4, 300), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        got = y.clone()
        layer.forward(big)                                                   # outgrows the buffers that the graph was captured with
        torch.cuda.synchronize()
        assert torch.equal(got, layer.forward(x))


def test_scores_of_microscaled_layers():
    from paper_1901_09504_amd import score

    rows = score.run_mx(tokens=200, hidden=256, vocab=1000)
    assert [(b, r) for b, r, _, _ in rows] == [(4, 0.0), (4, 0.05)]
    assert all(math.isfinite(p) and p >= 1 and 0 <= same <= 1 for _, _, p, same in rows)
