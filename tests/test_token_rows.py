"""Layers with a grid per row and the scoring of tokens on the GPU: codes and steps bit for bit against the oracle's Eq. 1 row by
row, products against exact integers and 64-bit factors, log probabilities against 64 bits; edges, strides, alignments, masks,
streams and graphs."""
import numpy as np
import pytest
import torch

from oracle import ref
from paper_1901_09504_amd import binding as B
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24                                            # half a step of fp32, relative
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}


@pytest.fixture(autouse=True)
def _gpu():
    G.require_gpu()


def _strided(t, ld, off=0, fill=None):
    """A device copy of the matrix t with row pitch ld whose first element lies `off` elements into its allocation."""
    rows, cols = t.shape
    buf = torch.empty(rows * ld + off + 16, dtype=t.dtype, device="cuda")
    if fill is not None:
        buf.fill_(fill)
    v = buf[off:off + rows * ld].view(rows, ld)
    v[:, :cols] = t.cuda()
    return v


def _lists(rng, C, s):
    """Sources and halvings as a selection leaves them: some channels split again and again."""
    src, depth = list(range(C)), [0] * C
    for _ in range(s):
        j = int(rng.integers(0, len(src))) if rng.random() < 0.7 else len(src) - 1
        depth[j] += 1
        src.append(src[j])
        depth.append(depth[j])
    return np.array(src, dtype=np.int32), np.array(depth, dtype=np.int32)


# ---- a grid per row --------------------------------------------------------------------------

def _codes(x, C, g, src, depth, s, bits, clip=1.0, ldq=None, stream=None):
    M = x.shape[0]
    ldq = B.ocs_padded_cols((C + s) * g) if ldq is None else ldq
    q = torch.full((M, ldq), 77, dtype=torch.int8, device="cuda")
    step = torch.full((M,), -1.0, device="cuda")
    B.ocs_split_quantize_rows(x, M, C, g, x.stride(0), None if src is None else G.dev(src), None if depth is None else G.dev(depth),
                              s, bits, clip, q, ldq, step, stream)
    return G.host(q), G.host(step)


def _expanded(x, C, g, src, depth):
    M = x.shape[0]
    v = x[:, :C * g].float().cpu().numpy().reshape(M, C, g)
    v = v[:, src, :]
    if depth is not None:
        v = (v * np.ldexp(np.float32(1), -depth.astype(np.int64)).astype(np.float32)[None, :, None]).astype(np.float32)
    return np.ascontiguousarray(v.reshape(M, -1), dtype=np.float32)


def _check_codes(x, C, g, src, depth, s, bits, clip=1.0, ldq=None):
    q, step = _codes(x, C, g, src, depth, s, bits, clip, ldq)
    e = _expanded(x, C, g, np.arange(C) if src is None else src, depth)
    for m in range(e.shape[0]):
        want, scale = ref.quantize(e[m:m + 1], bits, clip_ratio=clip, ldq=q.shape[1])
        assert np.array_equal(q[m], want[0]), (m, np.flatnonzero(q[m] != want[0])[:5])
        assert step[m].view(np.uint32) == scale.view(np.uint32)[1], m


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,C,g,s", [(1, 1, 1, 0), (3, 1, 1, 2), (5, 3, 1, 1), (7, 7, 1, 3), (64, 256, 1, 13), (9, 255, 1, 11),
                                     (6, 257, 1, 12), (4, 3, 49, 1), (3, 511, 1, 0), (5, 513, 1, 30), (2, 1001, 1, 51),
                                     (3, 1024, 1, 20), (2, 1025, 1, 7), (3, 64, 9, 4), (2, 3000, 1, 150), (2, 4096, 1, 82),
                                     (1, 7900, 1, 100), (2, 1000, 9, 10), (1, 2000, 9, 3)])
@pytest.mark.parametrize("halved", [False, True])
def test_codes_and_steps_are_those_of_each_row_alone(dtype, M, C, g, s, halved):
    rng = np.random.default_rng(M * 7919 + C * 31 + g + s)
    x = torch.from_numpy(rng.standard_normal((M, C * g)).astype(np.float32) * rng.choice([1e-3, 1.0, 50.0], (M, 1)).astype(np.float32))
    x[:, 0] *= 8
    src, depth = _lists(rng, C, s)
    _check_codes(x.to(dtype).cuda(), C, g, src, depth if halved else None, s, 8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [256, 300, 1030])
@pytest.mark.parametrize("C", [1030, 2051, 2500, 4102, 7003])
def test_codes_of_many_long_rows(dtype, M, C):
    """Lanes per row change with the count of rows; s copies and a last partial piece behind them."""
    rng = np.random.default_rng(M + C)
    src, depth = _lists(rng, C, 40)
    x = torch.randn((M, C), generator=torch.Generator().manual_seed(C)).to(dtype).cuda() * torch.rand((M, 1), device="cuda").to(dtype)
    for halved in (None, depth):
        q, step = _codes(x, C, 1, src, halved, 40, 8)
        for m in (0, 1, 255, M - 1):
            want, scale = ref.quantize(_expanded(x[m:m + 1], C, 1, src, halved), 8, ldq=q.shape[1])
            assert np.array_equal(q[m], want[0]) and step[m].view(np.uint32) == scale.view(np.uint32)[1], m
        if halved is None:                                  # every row: the grid's definition on the device, row by row
            v = x.float()[:, torch.from_numpy(src).long().cuda()]
            t = v.abs().amax(1, keepdim=True)
            code = (v * (torch.full_like(t, 127) / t)).clamp(-127, 127).round()
            assert np.array_equal(q[:, :C + 40], G.host(code.to(torch.int8))) and not q[:, C + 40:].any()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [40, 333, 1200])
def test_codes_of_any_pitch_and_alignment(dtype, C):
    rng = np.random.default_rng(C)
    src, depth = _lists(rng, C, 5)
    t = torch.from_numpy(rng.standard_normal((6, C)).astype(np.float32)).to(dtype)
    for ld, off in ((C, 1), (C + 1, 0), (C + 3, 3), (C + 8, 5)):
        _check_codes(_strided(t, ld, off, float("inf")), C, 1, src, None, 5, 8, ldq=(C + 5 + 15) // 16 * 16 + 4096)
        _check_codes(_strided(t, ld, off, float("nan")), C, 1, src, depth, 5, 6, clip=0.8)


@pytest.mark.parametrize("bits", range(2, 9))
def test_codes_of_every_width_with_ties_and_clips(bits):
    rng = np.random.default_rng(bits)
    qmax = 2 ** (bits - 1) - 1
    x = torch.from_numpy(rng.integers(-4 * qmax, 4 * qmax + 1, (40, 200)).astype(np.float32) * 0.25)
    x[:, 3] = qmax                                          # inv = 1 or less: quarters and exact halves on the grid
    for dtype in (F32, BF16):
        for clip in (1.0, 0.9, 0.5, 3.0):
            _check_codes(x.to(dtype).cuda(), 200, 1, None, None, 0, bits, clip)


def test_rows_of_zeros_of_tiny_and_of_huge_values():
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.standard_normal((8, 100)).astype(np.float32))
    x[0] = 0
    x[1] *= 1e-38                                           # qmax / T beyond fp32
    x[2] *= 1e-42                                           # subnormal
    x[3] *= 1e37
    x[4, 1:] = 0
    x[5] = -0.0
    _check_codes(x.cuda(), 100, 1, None, None, 0, 8)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("C", [100, 600, 5000])
def test_infinities_and_nan_stay_in_their_row(dtype, C):
    rng = np.random.default_rng(C)
    x = torch.from_numpy(rng.standard_normal((7, C)).astype(np.float32)).to(dtype)
    src, _ = _lists(rng, C, 6)
    x[1, C // 2] = float("inf")
    x[3, C - 1] = float("nan")
    x[5, 0] = float("-inf")
    q, step = _codes(x.cuda(), C, 1, src, None, 6, 8)
    assert not np.isfinite(step[[1, 3, 5]]).any()
    e = _expanded(x, C, 1, src, None)
    for m in (0, 2, 4, 6):
        want, scale = ref.quantize(e[m:m + 1], 8, ldq=q.shape[1])
        assert np.array_equal(q[m], want[0]) and step[m].view(np.uint32) == scale.view(np.uint32)[1]


def test_sources_outside_the_channels_are_clamped():
    x = torch.randn((3, 50), generator=torch.Generator().manual_seed(1))
    src = np.arange(54, dtype=np.int32)
    src[50:] = [-5, 1 << 30, 49, 0]
    q, _ = _codes(x.cuda(), 50, 1, src, None, 4, 8)
    assert np.array_equal(q[:, 50], q[:, 0]) and np.array_equal(q[:, 51], q[:, 49])
    assert np.array_equal(q[:, 52], q[:, 49]) and np.array_equal(q[:, 53], q[:, 0])


# ---- the product -----------------------------------------------------------------------------

def _random_codes(rng, rows, cols, ld, bits=8):
    qmax = 2 ** (bits - 1) - 1
    q = np.zeros((rows, ld), dtype=np.int8)
    q[:, :cols] = rng.integers(-qmax, qmax + 1, (rows, cols))
    return q


def _check_y(y, acc, sx, sw, bias, dtype, M, N):
    """acc is exact; its conversion, the factor, the product and the sum round once each, then the output type does."""
    f = sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None, :]
    want = acc.astype(np.float64) * f
    tol = 3.001 * U * np.abs(want)
    if bias is not None:
        want = want + bias.astype(np.float64)[None, :]
        tol = tol + 1.001 * U * np.abs(want)
    if dtype != F32:
        tol = tol + 1.001 * HALF_STEP[dtype] * np.abs(want) + (2.0 ** -25 if dtype == F16 else 0.0)
    got = y.float().cpu().numpy()[:M, :N].astype(np.float64)
    bad = np.abs(got - want) > tol + 1e-40
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist())


def _check_product(rng, M, N, K, dtype, with_bias, ldx=None, ldw=None, ld_extra=0, off=0, extreme=False):
    pad = B.ocs_padded_cols(K)
    ldx, ldw = ldx or pad, ldw or pad
    xq, wq = _random_codes(rng, M, K, ldx), _random_codes(rng, N, K, ldw)
    if extreme:
        xq[:, :K] = 127
        wq[:, :K] = np.where(np.arange(N)[:, None] % 2, -127, 127)
    sx = (rng.random(M) * 0.02 + 1e-4).astype(np.float32)
    sw = (rng.random(N) * 0.02 + 1e-4).astype(np.float32)
    bias = rng.standard_normal(N).astype(np.float32) if with_bias else None
    y = _strided(torch.full((M, N), 7.0, dtype=dtype), N + ld_extra, off, 7.0)
    B.ocs_qgemm_rows(G.dev(xq), ldx, G.dev(wq), ldw, M, N, K, 8, 8, G.dev(sx), G.dev(sw), None if bias is None else G.dev(bias), y,
                     y.stride(0))
    torch.cuda.synchronize()
    # products below 2^14 and sums below 2^31: exact in 64-bit floating point
    acc = xq[:, :K].astype(np.float64) @ wq[:, :K].astype(np.float64).T
    _check_y(y, acc, sx, sw, bias, dtype, M, N)
    if ld_extra:
        assert bool((y[:, N:] == 7.0).all())                # nothing is written between the rows


SHAPES = [(1, 1, 1), (1, 7, 64), (2, 16, 65), (3, 33, 128), (4, 100, 129), (5, 24, 300), (8, 48, 256), (9, 31, 1000), (15, 65, 320),
          (16, 256, 269), (17, 130, 321), (20, 600, 3150), (31, 64, 640), (32, 96, 1575), (33, 129, 500), (48, 17, 96), (63, 200, 1000),
          (64, 256, 269), (65, 127, 400), (100, 300, 2000), (127, 129, 257), (128, 128, 128), (129, 255, 384), (200, 512, 1052),
          (255, 257, 700), (256, 256, 1024), (257, 511, 520), (333, 2049, 1052), (500, 1000, 270), (700, 640, 3150), (1000, 72, 4302)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_product_of_every_shape(M, N, K, dtype):
    rng = np.random.default_rng(M * 131 + N * 17 + K)
    _check_product(rng, M, N, K, dtype, with_bias=(M + N) % 2 == 0)


@pytest.mark.parametrize("M", [1, 6, 20, 40, 100, 300, 520])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_product_into_any_pitch_and_alignment(M, dtype):
    rng = np.random.default_rng(M)
    for N, extra, off in ((64, 0, 1), (65, 0, 0), (66, 5, 3), (128, 4, 2), (250, 3, 0)):
        _check_product(rng, M, N, 200, dtype, True, ld_extra=extra, off=off)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("M,N,K", [(333, 2049, 1052), (1500, 2049, 1000), (1000, 4099, 600), (2000, 4001, 1000), (2000, 8001, 500),
                                   (300, 20001, 900)])
def test_product_into_rows_that_begin_between_two_words(dtype, M, N, K):
    """Tiles of every size: every second row of an odd pitch, and every row of an even one from an odd base; with a last column of
    tiles that is not whole."""
    rng = np.random.default_rng(M + N)
    _check_product(rng, M, N, K, dtype, True)
    _check_product(rng, M, N - 1, K, dtype, False, ld_extra=3, off=1)
    if M == 333:
        for off in (0, 1):
            _check_product(rng, M, 2048, K, dtype, True, ld_extra=off * 2, off=1)


@pytest.mark.parametrize("M,N", [(1, 40), (7, 50), (20, 70), (64, 33), (130, 140), (300, 260)])
def test_product_of_pitches_that_end_inside_a_step(M, N):
    rng = np.random.default_rng(N)
    for K, ldx, ldw in ((68, 80, 80), (68, 128, 80), (269, 272, 288), (320, 320, 320), (330, 384, 448), (330, 512, 384), (1, 16, 16),
                        (400, 448, 1024)):
        _check_product(rng, M, N, K, F32, True, ldx=ldx, ldw=ldw)


@pytest.mark.parametrize("M", [1, 16, 64, 260])
def test_product_of_extreme_codes(M):
    """The largest sums an accumulator may hold: 127 x 127 over the longest K that is accepted."""
    rng = np.random.default_rng(M)
    K = 2 ** 31 // (127 * 127)                              # 133,144
    while K * 127 * 127 >= 2 ** 31:
        K -= 1
    _check_product(rng, M, 36, K, F32, False, extreme=True)


@pytest.mark.parametrize("M,N,ldx,ldw", [(3, 5, 1 << 24, 128), (70, 3, 128, (1 << 24) + 64), (20, 40, (1 << 25) + 64, 192)])
def test_product_of_pitches_whose_offsets_in_a_tile_pass_32_bits(M, N, ldx, ldw):
    """A tile of 256 rows at a pitch of 2^24 bytes spans 2^32: 64-bit offsets."""
    rng = np.random.default_rng(M)
    K = 100
    xq, wq = _random_codes(rng, M, K, 128), _random_codes(rng, N, K, 128)
    big_x, big_w = torch.empty(M * ldx, dtype=torch.int8, device="cuda"), torch.empty(N * ldw, dtype=torch.int8, device="cuda")
    x, w = big_x.view(M, ldx), big_w.view(N, ldw)
    x[:, :128], w[:, :128] = G.dev(xq), G.dev(wq)
    sx, sw = np.full(M, 0.01, np.float32), np.full(N, 0.02, np.float32)
    y = torch.full((M, N), 7.0, device="cuda")
    B.ocs_qgemm_rows(x, ldx, w, ldw, M, N, K, 8, 8, G.dev(sx), G.dev(sw), None, y, N)
    torch.cuda.synchronize()
    _check_y(y, xq.astype(np.float64) @ wq.astype(np.float64).T, sx, sw, None, F32, M, N)


# ---- the layer -------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,C,g,s,N", [(1, 3000, 1, 150, 600), (1, 40, 1, 2, 8), (2, 1500, 1, 75, 1000), (3, 333, 1, 0, 100),
                                       (4, 256, 1, 13, 256), (8, 900, 1, 45, 333), (16, 512, 1, 26, 70), (20, 3000, 1, 150, 600),
                                       (33, 100, 9, 5, 64), (64, 256, 1, 13, 256), (300, 1001, 1, 51, 300), (2, 7000, 1, 70, 50),
                                       (5, 5000, 1, 50, 31)])
def test_layer_call_is_its_two_steps(dtype, M, C, g, s, N):
    rng = np.random.default_rng(M + C + N)
    src, depth = _lists(rng, C, s)
    x = torch.from_numpy(rng.standard_normal((M, C * g)).astype(np.float32)).to(dtype)
    x[:, 1] *= 20
    x = _strided(x, C * g + 3, 1, float("nan"))
    w = torch.from_numpy((rng.standard_normal((N, C * g)) * rng.random((N, 1))).astype(np.float32)).cuda()
    Ke = (C + s) * g
    ld = B.ocs_padded_cols(Ke)
    wq, sw = torch.empty((N, ld), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    B.ocs_split_quantize_rows(w, N, C, g, C * g, G.dev(src), G.dev(depth), s, 8, 1.0, wq, ld, sw)
    bias = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda()
    out = []
    for one in (False, True):
        xq, sx = torch.full((M, ld), 77, dtype=torch.int8, device="cuda"), torch.full((M,), -1.0, device="cuda")
        y = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
        if one:
            B.ocs_forward_rows(x, M, C, g, x.stride(0), G.dev(src), s, 8, 0.95, xq, ld, sx, wq, ld, N, 8, sw, bias, y, N)
        else:
            B.ocs_split_quantize_rows(x, M, C, g, x.stride(0), G.dev(src), None, s, 8, 0.95, xq, ld, sx)
            B.ocs_qgemm_rows(xq, ld, wq, ld, M, N, Ke, 8, 8, sx, sw, bias, y, N)
        torch.cuda.synchronize()
        out.append((xq, sx, y))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # and near the unquantized product: each value off by at most half a step of its row, on either side
    xe = _expanded(x, C, g, src, None).astype(np.float64)
    we = _expanded(w, C, g, src, depth).astype(np.float64)
    sxn, swn = out[0][1].cpu().numpy().astype(np.float64), sw.cpu().numpy().astype(np.float64)
    lo = np.float64(np.float32(0.95))
    clipped = np.clip(xe, -lo * np.abs(xe).max(1, keepdims=True), lo * np.abs(xe).max(1, keepdims=True))
    want = clipped @ we.T + bias.cpu().numpy().astype(np.float64)
    bound = (0.5001 * sxn[:, None] * np.abs(we).sum(1)[None, :] + 0.5001 * swn[None, :] * np.abs(clipped).sum(1)[:, None] +
             0.2501 * Ke * sxn[:, None] * swn[None, :])
    got = out[0][2].float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= bound + (HALF_STEP[dtype] + 8 * U) * np.abs(got) + 1e-6)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,C,g,s,N", [(1, 1, 1, 0, 1), (1, 5, 1, 2, 17), (3, 100, 1, 0, 33), (24, 60, 1, 6, 40), (20, 256, 1, 13, 256),
                                       (17, 255, 1, 3, 4097), (9, 130, 1, 7, 4100), (8, 511, 1, 20, 8200), (2, 40, 9, 3, 100),
                                       (5, 900, 1, 45, 9000), (1, 6000, 1, 300, 300), (1, 1000, 1, 50, 25000), (7, 64, 1, 4, 25001),
                                       (1, 1029, 1, 0, 8193), (12, 300, 1, 400, 70)])
def test_layer_of_few_tokens_is_its_two_steps(dtype, M, C, g, s, N):
    """The layer as one launch: one share of outputs a workgroup or several, waves without a step of K, rows with a last partial
    piece, more copies than channels, a pitch beyond the steps; from a graph as well."""
    rng = np.random.default_rng(M * 31 + C + N)
    src, depth = _lists(rng, C, s)
    Ke = (C + s) * g
    x = _strided(torch.from_numpy(rng.standard_normal((M, C * g)).astype(np.float32)).to(dtype), C * g + 1, 3, float("inf"))
    ldq, ldw = B.ocs_padded_cols(Ke) + 128 * (M % 2), max(B.ocs_padded_cols(Ke), 64)
    wq = G.dev(_random_codes(rng, N, Ke, ldw))
    sw = G.dev((rng.random(N) * 0.02 + 1e-4).astype(np.float32))
    bias = G.dev(rng.standard_normal(N).astype(np.float32)) if N % 2 else None
    srcd = G.dev(src)

    def outputs():
        return (torch.full((M, ldq), 77, dtype=torch.int8, device="cuda"), torch.full((M,), -1.0, device="cuda"),
                _strided(torch.full((M, N), 7.0, dtype=dtype), N + 3, 1, 7.0))

    def layer(o):
        B.ocs_forward_rows(x, M, C, g, x.stride(0), srcd, s, 8, 0.9, o[0], ldq, o[1], wq, ldw, N, 6, sw, bias, o[2], o[2].stride(0))

    two, one, captured = outputs(), outputs(), outputs()
    B.ocs_split_quantize_rows(x, M, C, g, x.stride(0), srcd, None, s, 8, 0.9, two[0], ldq, two[1])
    B.ocs_qgemm_rows(two[0], ldq, wq, ldw, M, N, Ke, 8, 6, two[1], sw, bias, two[2], two[2].stride(0))
    layer(one)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(two, one))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(captured)
    for _ in range(3):
        for a in captured:
            a.fill_(5)
        captured[2][:, N:] = 7.0
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(two, captured))


def test_bad_rows_of_few_tokens_stay_alone():
    rng = np.random.default_rng(3)
    M, C, N = 6, 300, 50
    x = torch.from_numpy(rng.standard_normal((M, C)).astype(np.float32))
    x[1, 7], x[3, 299], x[5] = float("nan"), float("inf"), 0.0
    src, _ = _lists(rng, C, 9)
    src[C:C + 2] = [-7, 1 << 20]                             # clamped
    wq = G.dev(_random_codes(rng, N, C + 9, 384))
    sw = torch.ones(N, device="cuda")
    xq, sx = torch.empty((M, 384), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    y = torch.empty((M, N), device="cuda")
    B.ocs_forward_rows(x.cuda(), M, C, 1, C, G.dev(src), 9, 8, 1.0, xq, 384, sx, wq, 384, N, 8, sw, None, y, N)
    y, q = G.host(y), G.host(xq).astype(np.float64)
    assert not np.isfinite(y[[1, 3]]).any() and (y[5] == 0).all()
    for m in (0, 2, 4):
        want = (G.host(wq)[:, :C + 9].astype(np.float64) @ q[m, :C + 9]) * float(G.host(sx)[m])
        assert np.all(np.abs(y[m] - want) <= 4 * U * np.abs(want))
        assert q[m, C] == q[m, 0] and q[m, C + 1] == q[m, C - 1]


# ---- scoring ---------------------------------------------------------------------------------

def _score(x, tokens, k, want_entropy=True, stream=None):
    M, V = x.shape
    lp = torch.full((M,), 7.0, device="cuda") if tokens is not None else None
    ent = torch.full((M,), 7.0, device="cuda") if want_entropy else None
    ids = torch.full((M, k), -7, dtype=torch.int32, device="cuda") if k else None
    top = torch.full((M, k), 7.0, device="cuda") if k else None
    wb = B.ocs_token_logprobs_workspace_bytes(M, V, k)
    ws = torch.full((wb,), 255, dtype=torch.uint8, device="cuda") if wb else None
    B.ocs_token_logprobs(x, M, V, x.stride(0), tokens, k, lp, ent, ids, top, ws, stream)
    torch.cuda.synchronize()
    return tuple(None if t is None else t.cpu().numpy() for t in (lp, ent, ids, top))


def _check_scores(x, tokens, k):
    """Against 64 bits.  An exponential's relative error: its argument x - m and the product with log2 e round, |d| U each, and the
    exponential itself 2 U more.  A sum's: as many U as a lane adds values (at least 256 lanes a row; 64 more for raising the maximum and
    joining the lanes).  The logarithm and the subtractions round on top, relative to their results."""
    M, V = x.shape
    lp, ent, ids, top = _score(x, None if tokens is None else tokens.cuda(), k)
    d = x.detach().cpu().double().numpy()
    m = d.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        none = np.isneginf(m)[:, 0]
        z = np.where(none[:, None], -np.inf, d - np.where(none[:, None], 0, m))
        e = np.exp(z)
        s = e.sum(1, keepdims=True)
        logs = np.where(none[:, None], 0.0, np.log(s))
        mean = np.where(e > 0, e * z, 0).sum(1, keepdims=True) / np.where(s > 0, s, 1)
        second = np.where(e > 0, e * z * z, 0).sum(1, keepdims=True) / np.where(s > 0, s, 1)
    n = V / 256 + 72
    ds = U * (n + 2.1 * np.abs(mean))                        # relative error of s, in 64 rows' worst case
    dlog = ds + 2 * U * np.abs(logs) + 1e-12
    if tokens is not None:
        t = tokens.numpy()
        has = (t >= 0) & (t < V)
        want = np.where(has, z[np.arange(M), np.where(has, t, 0)] - logs[:, 0], 0.0)
        fin = np.isfinite(want)
        assert np.array_equal(np.isneginf(lp), np.isneginf(want))
        err = np.abs(lp[fin] - want[fin])
        tol = dlog[fin, 0] + U * (np.abs(want[fin]) + np.abs(want[fin] + logs[fin, 0]))
        assert np.all(err <= tol), (err.max(), tol[err.argmax()])
        assert np.all(lp[~has] == 0)
    hw = np.where(none, 0.0, (logs - mean)[:, 0])
    dw = U * (n * np.abs(mean) + 2.1 * second + 3 * np.abs(mean))
    tol = (dlog + dw + ds * np.abs(mean) + 2 * U * (np.abs(hw)[:, None] + np.abs(mean)))[:, 0]
    err = np.abs(ent - hw)
    assert np.all(err <= tol), (err.max(), tol[err.argmax()])
    if k:
        order = np.argsort(-(d + 0.0), axis=1, kind="stable")[:, :k]
        assert np.array_equal(ids, order), np.argwhere(ids != order)[:5].tolist()
        want = np.take_along_axis(z, order, 1) - logs
        fin = np.isfinite(want)
        assert np.array_equal(np.isneginf(top), np.isneginf(want))
        tol = np.where(fin, dlog + U * (np.abs(want) + np.abs(want + logs)), 0)
        assert np.all(np.abs(np.where(fin, top - np.where(fin, want, 0), 0)) <= tol)


def _logits(M, V, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = 3 * torch.randn((M, V), generator=g)
    t = torch.randint(V, (M,), generator=g, dtype=torch.int32)
    x[torch.arange(M), t.long()] += 8
    return x.to(dtype), t


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,V,k", [(1, 1, 1), (1, 2, 2), (3, 5, 5), (2, 33, 32), (5, 100, 20), (4, 255, 3), (2, 256, 32), (3, 1000, 1),
                                   (1, 1023, 8), (2, 4096, 0), (1, 4099, 32), (3, 33001, 5), (1, 50021, 20), (2, 131073, 10),
                                   (1, 300007, 32), (70, 777, 6), (300, 1501, 5), (600, 301, 7), (1030, 64, 4)])
def test_scores(dtype, M, V, k):
    x, t = _logits(M, V, dtype, M + V + k)
    _check_scores(x.cuda(), t, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,V,k", [(1, 65537, 32), (5, 70001, 1), (64, 98305, 5), (250, 66001, 8), (2, 2200000, 20), (1, 5000001, 3)])
def test_scores_of_few_long_rows(dtype, M, V, k):
    """Rows in parts: one logit more than a workgroup holds, as many rows as take part in it, more parts asked for than there may be."""
    x, t = _logits(M, V, dtype, V)
    _check_scores(x.cuda(), t, k)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,V", [(3, 999), (2, 40000), (700, 130)])
def test_scores_of_any_pitch_and_alignment(dtype, M, V):
    x, t = _logits(M, V, dtype, V)
    for ld, off in ((V, 1), (V + 1, 0), (V + 3, 3), (V + 7, 5)):
        _check_scores(_strided(x, ld, off, float("nan"))[:, :V], t, 5)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,V", [(6, 500), (6, 33001), (520, 300), (6, 70001)])
def test_masks(dtype, M, V):
    """-inf, the type's lowest value, a row with nothing left, rows with fewer tokens left than alternatives asked for."""
    x, t = _logits(M, V, dtype, V + 1)
    g = torch.Generator().manual_seed(V)
    x[:, torch.rand(V, generator=g) < 0.5] = float("-inf")
    x[0] = float("-inf")
    x[1, 1:] = float("-inf")
    x[2, :] = float("-inf")
    x[2, [V - 1, 17, 250]] = torch.tensor([1.0, 2.0, 2.0], dtype=dtype)
    x[3, ::2] = torch.finfo(dtype).min
    x[4] = torch.finfo(dtype).min
    t[5] = V
    _check_scores(x.cuda(), t, 8)
    t[5] = -1
    t[2] = 17
    _check_scores(x.cuda(), t, 32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,V", [(4, 400), (4, 33001), (520, 600), (2, 100000)])
def test_ties_go_to_the_lowest_index(dtype, M, V):
    x = torch.zeros((M, V))
    x[0] = -3.0
    x[0, V // 2:] = 1.0                                      # more equal values than any list holds
    x[1] = torch.arange(V) % 7
    x[1, ::3] = -0.0
    if M > 2:
        x[2] = torch.arange(V, 0, -1) / V
        x[3] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    _check_scores(x.to(dtype).cuda(), torch.zeros(M, dtype=torch.int32), 32)


@pytest.mark.parametrize("V", [50, 3000, 100000])
def test_large_logits_lose_nothing(V):
    x, t = _logits(3, V, F32, V)
    x[0] = x[0] * 1e3 + 5e4
    x[1] *= 1e37
    x[2] -= 3e4
    x[1, 0], x[1, 1] = 3.0e38, -3.0e38
    _check_scores(x.cuda(), t, 5)


@pytest.mark.parametrize("V", [60, 5000, 100000])
def test_nan_and_infinity_spoil_their_row_alone(V):
    x, t = _logits(5, V, F32, V)
    clean = _score(x.cuda(), t.cuda(), 4)
    x[1, V // 3] = float("nan")
    x[3, V - 2] = float("inf")
    x[3, 1] = float("nan")
    t[3] = -1
    lp, ent, ids, top = _score(x.cuda(), t.cuda(), 4)
    for m in (0, 2, 4):
        assert lp[m] == clean[0][m] and ent[m] == clean[1][m]
        assert np.array_equal(ids[m], clean[2][m]) and np.array_equal(top[m], clean[3][m])
    assert np.isnan(lp[1]) and lp[3] == 0 and np.isnan(ent[[1, 3]]).all() and np.isnan(top[[1, 3]]).all()
    assert ids[1, 0] == V // 3 and list(ids[3, :2]) == [1, V - 2]


def test_outputs_that_are_not_asked_for():
    x, t = _logits(5, 999, F32, 3)
    lp, ent, ids, top = _score(x.cuda(), t.cuda(), 6)
    assert np.array_equal(_score(x.cuda(), None, 0)[1], ent)
    a = _score(x.cuda(), None, 6, want_entropy=False)
    assert np.array_equal(a[2], ids) and np.array_equal(a[3], top)
    assert np.array_equal(_score(x.cuda(), t.cuda(), 0, want_entropy=False)[0], lp)


def test_the_same_bits_every_time():
    for M, V in ((2, 90001), (700, 2001)):
        x, t = _logits(M, V, BF16, 9)
        first = _score(x.cuda(), t.cuda(), 5)
        for _ in range(3):
            assert all(np.array_equal(a, b) for a, b in zip(first, _score(x.cuda(), t.cuda(), 5)))


# ---- the layer and the scores as a program uses them -------------------------------------------

def _oracle_layer(W, X, r, bits_w):
    C = W.shape[1]
    s = ref.num_splits(C, r)
    sp = ref.split_weights(W, C, 1, s)
    xe = X[:, sp["chan_src"]]
    y = np.zeros((X.shape[0], W.shape[0]))
    steps_w, rows_w = [], []
    for n in range(W.shape[0]):
        q, sc = ref.quantize(sp["T_out"][n:n + 1], bits_w)
        rows_w.append(q[0].astype(np.float64))
        steps_w.append(float(sc[1]))
    for m in range(X.shape[0]):
        q, sc = ref.quantize(np.ascontiguousarray(xe[m:m + 1]), 8)
        y[m] = (np.stack(rows_w) @ q[0].astype(np.float64)) * (float(sc[1]) * np.array(steps_w))
    return y


@pytest.mark.parametrize("M,C,N,r,bits_w", [(1, 300, 50, 0.05, 8), (25, 300, 70, 0.05, 5), (70, 128, 33, 0.0, 8), (9, 64, 40, 0.3, 4)])
def test_token_layer_against_the_oracle(M, C, N, r, bits_w):
    from paper_1901_09504_amd.layer import TokenLayer, token_logprobs

    rng = np.random.default_rng(C + N)
    W = (rng.standard_normal((N, C)) * rng.random((N, 1))).astype(np.float32)
    W[rng.integers(0, N, 5), rng.integers(0, C, 5)] *= 8
    X = rng.standard_normal((M, C)).astype(np.float32)
    head = TokenLayer(N, C, r, bits_w=bits_w)
    head.prepare_weights(G.dev(W))
    y = head.forward(G.dev(X))
    torch.cuda.synchronize()
    want = _oracle_layer(W, X, r, bits_w)
    assert np.all(np.abs(y.cpu().numpy() - want) <= 4 * U * np.abs(want))
    t = torch.from_numpy(rng.integers(-1, N, M).astype(np.int32)).cuda()
    out = token_logprobs(y, t, 3)
    lp, ent, ids, top = _score(y, t, 3)
    assert np.array_equal(out["logprob"].cpu().numpy(), lp) and np.array_equal(out["entropy"].cpu().numpy(), ent)
    assert np.array_equal(out["top_ids"].cpu().numpy(), ids) and np.array_equal(out["top_logprobs"].cpu().numpy(), top)
    assert set(token_logprobs(y)) == {"entropy"}


def test_no_tokens_and_one():
    from paper_1901_09504_amd.layer import TokenLayer, token_logprobs

    head = TokenLayer(40, 100, 0.05, out_dtype=BF16)
    head.prepare_weights(torch.randn((40, 100), device="cuda"))
    y = head.forward(torch.empty((0, 100), dtype=F16, device="cuda"))
    assert y.shape == (0, 40) and y.dtype == BF16
    out = token_logprobs(y, torch.empty(0, dtype=torch.int32, device="cuda"), 2)
    assert [tuple(out[n].shape) for n in ("logprob", "entropy", "top_ids", "top_logprobs")] == [(0,), (0,), (0, 2), (0, 2)]
    x = torch.randn((5, 100), device="cuda").to(F16)
    every = head.forward(x).clone()
    for m in range(5):                                      # a token's outputs do not depend on its company
        assert torch.equal(head.forward(x[m:m + 1])[0], every[m])


def test_layer_that_grows_while_another_stream_works():
    """The buffers that a larger batch replaces are still the other stream's: what is allocated meanwhile does not land on them."""
    from paper_1901_09504_amd.layer import TokenLayer

    head = TokenLayer(6000, 1000, 0.05, max_rows=256)
    head.prepare_weights(torch.randn((6000, 1000), device="cuda"))
    small, large = torch.randn((256, 1000), device="cuda"), torch.randn((300, 1000), device="cuda")
    want = head.forward(small).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):
        y = head.forward(small, side)
    with torch.cuda.stream(side):
        kept = y.clone()
    del y
    head.forward(large)                                     # replaces codes, steps and outputs
    filler = [torch.full((256, 6000), 7.0, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(kept, want) and all(bool((f == 7.0).all()) for f in filler)


def test_logits_of_one_token_in_any_layout():
    from paper_1901_09504_amd.layer import token_logprobs

    x = torch.randn((5, 3), device="cuda")
    for col in (x[:, 1:2], x.t().contiguous().t()[:, 2:]):  # a column: its second stride means nothing
        out = token_logprobs(col, torch.zeros(5, dtype=torch.int32, device="cuda"), 1)
        assert not out["entropy"].any() and not out["logprob"].any() and not out["top_ids"].any()


def test_scoring_command():
    from paper_1901_09504_amd import score

    rows = score.run(tokens=300, hidden=256, vocab=1000)
    exact = rows[0][2]
    eight = [p for bits, _, p, _ in rows if bits == 8]
    four = [p for bits, _, p, _ in rows if bits == 4]
    assert 1 < exact < 1000 and all(abs(p / exact - 1) < 0.05 for p in eight)
    assert max(abs(p / exact - 1) for p in eight) < max(abs(p / exact - 1) for p in four)


# ---- long offsets, streams, graphs -----------------------------------------------------------

def test_offsets_beyond_32_bits():
    """Rows whose first element lies more than 2^32 elements into the tensor."""
    ld = (1 << 31) + 64
    buf = torch.empty(2 * ld + 4096, dtype=BF16, device="cuda")
    x, t = _logits(3, 4001, BF16, 4)
    v = buf.as_strided((3, 4001), (ld, 1))
    v.copy_(x)
    _check_scores(v, t, 5)
    q, step = _codes(v, 4001, 1, None, None, 0, 8)
    q2, step2 = _codes(x.cuda(), 4001, 1, None, None, 0, 8)
    assert np.array_equal(q, q2) and np.array_equal(step, step2)
    y = buf.as_strided((3, 100), (ld, 1))
    rng = np.random.default_rng(0)
    xq, wq = _random_codes(rng, 3, 200, 256), _random_codes(rng, 100, 200, 256)
    sx, sw = np.full(3, 0.01, np.float32), np.full(100, 0.02, np.float32)
    B.ocs_qgemm_rows(G.dev(xq), 256, G.dev(wq), 256, 3, 100, 200, 8, 8, G.dev(sx), G.dev(sw), None, y, ld)
    torch.cuda.synchronize()
    _check_y(y, xq[:, :200].astype(np.float64) @ wq[:, :200].astype(np.float64).T, sx, sw, None, BF16, 3, 100)


def test_codes_into_rows_whose_end_is_near_2_to_31():
    """The padding of such a row is walked past its end by less than a round; a 32-bit column would not hold that."""
    x = torch.randn((1, 100), generator=torch.Generator().manual_seed(2)).cuda()
    ldq = (1 << 31) - 16
    big = torch.full((ldq,), 77, dtype=torch.int8, device="cuda")
    step = torch.empty(1, device="cuda")
    B.ocs_split_quantize_rows(x, 1, 100, 1, 100, None, None, 0, 8, 1.0, big, ldq, step)
    q, want = _codes(x, 100, 1, None, None, 0, 8)
    assert np.array_equal(G.host(big[:100]), q[0, :100]) and G.host(step)[0] == want[0]
    assert not any(bool(part.any()) for part in big[100:].split(1 << 28))


def _chain_state(M=20, C=500, s=25, V=40001, k=5):
    rng = np.random.default_rng(M)
    src, depth = _lists(rng, C, s)
    st = dict(M=M, C=C, s=s, V=V, k=k, src=G.dev(src))
    st["x"] = torch.from_numpy(rng.standard_normal((M, C)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.standard_normal((V, C)).astype(np.float32)).cuda()
    st["ld"] = B.ocs_padded_cols(C + s)
    st["wq"], st["sw"] = torch.empty((V, st["ld"]), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    B.ocs_split_quantize_rows(w, V, C, 1, C, st["src"], G.dev(depth), s, 8, 1.0, st["wq"], st["ld"], st["sw"])
    st["xq"], st["sx"] = torch.empty((M, st["ld"]), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    st["y"] = torch.empty((M, V), device="cuda")
    st["t"] = torch.randint(V, (M,), dtype=torch.int32, device="cuda")
    st["out"] = [torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty((M, k), dtype=torch.int32, device="cuda"),
                 torch.empty((M, k), device="cuda")]
    st["ws"] = torch.empty(max(256, B.ocs_token_logprobs_workspace_bytes(M, V, k)), dtype=torch.uint8, device="cuda")
    return st


def _chain(st, stream=None):
    B.ocs_forward_rows(st["x"], st["M"], st["C"], 1, st["C"], st["src"], st["s"], 8, 1.0, st["xq"], st["ld"], st["sx"], st["wq"],
                       st["ld"], st["V"], 8, st["sw"], None, st["y"], st["V"], stream)
    lp, ent, ids, top = st["out"]
    B.ocs_token_logprobs(st["y"], st["M"], st["V"], st["V"], st["t"], st["k"], lp, ent, ids, top, st["ws"], stream)


def _results(st):
    return [t.clone() for t in (st["xq"], st["sx"], st["y"], *st["out"])]


@pytest.mark.parametrize("M", [1, 3, 20, 300])
def test_chain_on_another_stream_and_replayed_from_a_graph(M):
    st = _chain_state(M=M)
    _chain(st)
    torch.cuda.synchronize()
    want = _results(st)
    side = torch.cuda.Stream()
    for t in (st["xq"], st["sx"], st["y"], *st["out"]):
        t.zero_()
    torch.cuda.synchronize()
    _chain(st, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, _results(st)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(st)
    x0 = st["x"].clone()
    for i in range(4):
        st["x"].copy_(x0 if i % 2 == 0 else x0 * 0.5 + 1)
        for t in (st["xq"], st["sx"], st["y"], *st["out"]):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = _results(st)
        _chain(st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, _results(st))), i
