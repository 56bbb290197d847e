"""The quantized cache on the GPU, further: how fine the weights of the values are, and cases at the edges of what a call may be given."""
import numpy as np
import pytest
import torch

from paper_1901_09504_amd import binding as B
from tests import gpu_util as G
from tests import test_cache as C
from tests.test_cache import BF16, F16, F32, INT8, MX4, Pool, check_attention, fill

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    G.require_gpu()


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("new,held,window", [([1, 1, 1], [100, 333, 700], 0), ([1], [5000], 0), ([60, 75], [60, 400], 0), ([70], [2900], 1500)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_weights_of_the_values_have_16_bits_with_bf16_queries(monkeypatch, fmt, new, held, window, D):
    """Two bf16 numbers make a weight: the first is off by 2^-8 of it at most, the second by 2^-8 of what is left.  Values of both signs leave
    outputs far below the sum of their sizes, where one bf16 number would show."""
    monkeypatch.setitem(C.WEIGHT, BF16, 2.0 ** -16)
    pool = Pool(fmt, held, 2, D, 32, seed=D)
    fill(pool, 4)
    check_attention(pool, new, 4, BF16, window=window)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("T,Hq", [(100, 6), (400, 6), (37, 2)])
def test_offsets_that_do_not_ascend_stay_inside_the_tensors(fmt, T, Hq):
    """They are against the interface, and what comes out is nobody's; but nothing is read or written beyond the tensors, by either kernel and
    for sequences that a wave looks at together or searches."""
    H, D = 2, 64
    pool = Pool(fmt, [70], H, D, 16, seed=1)
    fill(pool, 1)
    rng = np.random.default_rng(T)
    lists = [[0, T, 0, T], [T, T, 0, 0, T], [T, 0], [5, -3, 2 ** 31 - 1, -2 ** 31, 9], [0, 0, T, 0, T // 2, 3, T], [T] * 40 + [0] * 25,
             rng.integers(-T, 2 * T, 30).tolist(), rng.integers(0, T + 1, 5).tolist(), rng.permutation(90).tolist(), [T] * 100 + [0] * 50,
             rng.integers(0, T + 1, 200).tolist()]
    for cu in lists:
        n = len(cu) - 1
        table = torch.full((n, 5), int(pool.table[0, 0]), dtype=torch.int32, device="cuda")
        starts = torch.from_numpy(rng.integers(-5, 60, n).astype(np.int32)).cuda()
        whole = torch.full((T + 64, Hq, D), 7.0, dtype=BF16, device="cuda")
        lses = torch.full((T + 64, Hq), 7.0, device="cuda")
        q, y, lse = torch.zeros((T + 64, Hq, D), dtype=BF16, device="cuda")[32:-32], whole[32:-32], lses[32:-32]
        for most in (70, 4000):                                              # in parts too
            ws = C.workspace(T, n, H, Hq, D, most)
            B.ocs_cache_attention(q, Hq * D, D, Hq, T, G.dev(np.array(cu, dtype=np.int64).astype(np.int32)), starts, n, most, *pool.args(table), 0.1,
                                  0, y, Hq * D, D, lse, ws)
        for t in (whole, lses):
            assert bool((t[:32] == 7).all()) and bool((t[-32:] == 7).all()), cu


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 224, 256])
@pytest.mark.parametrize("G_,dtype", [(1, F32), (3, BF16), (2, F16)])
@pytest.mark.parametrize("new", [3, 60, 100])
def test_a_value_with_one_block_that_is_no_number_is_none_for_those_who_see_it(D, G_, dtype, new):
    """In the first, a middle or the last block: every output of the tokens that see it is NaN, the others' are what they are without it."""
    held, at, blocks = 130, 128, D // 32
    for block, byte in ((0, 255), (blocks // 2, 254), (blocks - 1, 253), (blocks - 1, 255)):
        pool = Pool(MX4, [held], 2, D, 16, seed=8)
        fill(pool, 8)
        q = torch.randn((new, 2 * G_, D), generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
        cu, st, _ = C.tokens_of([new], [held - new])
        ys = []
        for bad in (False, True):
            if bad:
                page, row = pool.row(0, at)
                pool.scales[1][page, 1, row, block] = byte
            y = torch.full_like(q, 7.0)
            B.ocs_cache_attention(q, 2 * G_ * D, D, 2 * G_, new, cu, st, 1, held, *pool.args(), 0.1, 0, y, 2 * G_ * D, D, None,
                                  C.workspace(new, 1, 2, 2 * G_, D, held))
            ys.append(y)
        sees = torch.arange(held - new, held) >= at
        assert bool(ys[1][sees, G_:].isnan().all()), (block, byte)
        assert torch.equal(ys[1][~sees], ys[0][~sees]) and torch.equal(ys[1][:, :G_], ys[0][:, :G_]) and bool(ys[0].isfinite().all())


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [1, 60, 100])
def test_large_values_whose_weight_is_nothing_add_nothing(fmt, dtype, new):
    """Position 1500's score is 4096 above the others', which lie in parts of their own and hold values 2^140 times as large: their weights
    are 0, and the output is position 1500's value, its weight's and its own rounding off."""
    L = 2048
    pool = Pool(fmt, [L], 1, 64, 16, seed=12)
    k, v = torch.zeros((L, 1, 64), device="cuda"), torch.full((L, 1, 64), 2.0 ** 100, device="cuda")
    k[1500], v[1500] = 8, C.random_rows(1, 1, 64, F32, 13)[0] * 2.0 ** -40
    C.write(pool, k, v, [L], [0])
    q = torch.full((new, 1, 64), 8.0, dtype=dtype, device="cuda")
    y, lse = torch.zeros_like(q), torch.zeros((new, 1), device="cuda")
    cu, st, _ = C.tokens_of([new], [L - new])
    ws = C.workspace(new, 1, 1, 1, 64, L)
    assert ws is not None
    B.ocs_cache_attention(q, 64, 64, 1, new, cu, st, 1, L, *pool.args(), 1.0, 0, y, 64, 64, lse, ws)
    page, row = pool.row(0, 1500)
    want = pool.numbers(1)[page, 0, row]
    assert bool(((y[:, 0].double() - want).abs() <= want.abs() * (C.HALF_STEP[dtype] + 2.0 ** -15)).all())
    k1500 = pool.numbers(0)[page, 0, row]
    assert bool(((lse.double() - 8 * k1500.sum()).abs() <= 4096 * 2.0 ** -21).all())


@pytest.mark.parametrize("fmt,D", [(INT8, 64), (MX4, 128), (INT8, 160)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("window", [3, 5, 40, 0])
@pytest.mark.parametrize("columns", [2, 5, 6, 7])
def test_windows_over_the_end_of_the_table(fmt, D, dtype, window, columns):
    """Tokens on both sides of the table's last position: the later ones of a wave's see none of it, those before them do."""
    new, held = [90, 95], [146, 151]                                         # 32 tokens to a wave, from position 56 on
    pool = Pool(fmt, held, 1, D, 16, seed=3)
    pool.table = np.ascontiguousarray(pool.table[:, :columns])
    pool.held = [min(n, 16 * columns) for n in held]
    fill(pool, 3)
    pool.held = held
    check_attention(pool, new, 1, dtype, window=window)


@pytest.mark.parametrize("bits", [8, 4])
def test_an_append_that_fails_leaves_the_cache_as_it_was(monkeypatch, bits):
    from paper_1901_09504_amd.layer import TokenCache

    def state(cache):
        return [list(t) for t in cache.tables], list(cache.lengths), list(cache.spare)

    def fails(*_):
        raise RuntimeError("no copy")

    cache = TokenCache(2, 4, 2, 64, page_rows=16, bits=bits)
    rows = C.random_rows(40, 2, 64, F32, 1)
    for begun in (0, 5):
        if begun:
            cache.append(rows[:begun], rows[:begun], [begun], [1])
        before = state(cache)
        with pytest.raises(B.OcsError):                                      # an element type that no call takes
            cache.append(rows.double(), rows.double(), [40], [0])
        assert state(cache) == before
        with monkeypatch.context() as m, pytest.raises(RuntimeError, match="no copy"):
            m.setattr(TokenCache, "_on_device", fails)
            cache.append(rows[:38], rows[:38], [20, 18])
        assert state(cache) == before
    cache.append(rows[:31], rows[:31], [1, 30])
    assert cache.lengths == [1, 35] and [len(t) for t in cache.tables] == [1, 3] and not cache.spare
    want = TokenCache(2, 4, 2, 64, page_rows=16, bits=bits)
    want.append(torch.cat([rows[:1], rows[:5], rows[1:31]]), torch.cat([rows[:1], rows[:5], rows[1:31]]), [1, 35])
    assert all(torch.equal(a, b) for a, b in zip(cache.read(), want.read()))


def eight_bits(x):
    """fp32 rows [.., D] that are finite and not all zeros -> codes and steps of Eq. 1, each quotient and product rounded to 32 bits once."""
    T = np.abs(x).max(-1).astype(np.float64)
    factor, step = (127 / T).astype(np.float32), (T / 127).astype(np.float32)
    scaled = (x.astype(np.float64) * factor[..., None].astype(np.float64)).astype(np.float32)
    return np.rint(scaled).clip(-127, 127).astype(np.int8), step


def check_rows(fmt, dtype, H, D, P, new, held, starts, extra, seed):
    """Writes the tokens into a pool, compares every row of it with the definition (the others as they were), and what is read back."""
    pool = Pool(fmt, held, H, D, P, seed=seed, halved=seed % 2 == 1)
    before = [t.clone() for t in pool.codes + pool.scales]
    T = sum(new)
    rows = [C.random_rows(T + extra, H, D, dtype, seed + i) for i in (1, 2)]
    C.write(pool, *rows, new, starts)
    position = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, new)]).astype(np.int64)
    page = pool.table[np.repeat(np.arange(len(new)), new), position // P].astype(np.int64)
    at = torch.from_numpy(page * P + position % P).cuda()                    # [T], of [pages, P]
    assert len(at.unique()) == T
    for i in range(2):
        x = G.host(rows[i][:T].float())
        if pool.depth[i] is not None:
            x = (x * np.ldexp(np.float32(1), -G.host(pool.depth[i]).astype(np.int64)).astype(np.float32)).astype(np.float32)
        if fmt == INT8:
            codes, scales = eight_bits(x)
            few = [C.ref.quantize(np.ascontiguousarray(r[None]), 8, ldq=D) for r in x[:3, 0]]
            assert all(np.array_equal(q[0], c) and s[1] == t for (q, s), c, t in zip(few, codes[:3, 0], scales[:3, 0]))
        else:
            codes, scales = C.on_grids(x.reshape(-1, D))
            codes, scales = C.packed(codes, D // 2).reshape(T, H, -1), scales.reshape(T, H, -1)
        for now, was, new_rows in ((pool.codes[i], before[i], codes), (pool.scales[i], before[2 + i], scales)):
            if now.dim() == 3:
                now, was, new_rows = now[..., None], was[..., None], new_rows[..., None]
            want = was.transpose(1, 2).flatten(0, 1).contiguous()            # [pages * P, H, ..]
            want[at] = torch.from_numpy(np.ascontiguousarray(new_rows)).cuda()
            assert torch.equal(now.transpose(1, 2).flatten(0, 1).contiguous().view(torch.uint8), want.view(torch.uint8))
    back = C.read(pool, F32, new, starts, extra=extra)
    for i in range(2):
        want = pool.numbers(i).transpose(1, 2).flatten(0, 1)[at]
        assert bool(((back[i][:T].double() - want).abs() <= 2.0 ** -23 * 1.01 * want.abs()).all()) and bool((back[i][T:] == 7).all())


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("B_", [64, 65, 100, 300])
@pytest.mark.parametrize("kind", ["a token each", "an empty one in front", "empty ones among them", "tokens behind the last"])
def test_rows_of_many_sequences(fmt, B_, kind):
    rng = np.random.default_rng(B_)
    new, extra = [1] * B_, 0
    if kind == "an empty one in front":
        new[0] = 0
    elif kind == "empty ones among them":
        new = [int(n) for n in rng.choice([0, 0, 1, 2, 37], B_)]
    elif kind == "tokens behind the last":
        new, extra = [int(n) for n in rng.integers(0, 4, B_)], 9
    starts = [int(s) for s in rng.integers(0, 50, B_)]
    check_rows(fmt, BF16, 3, 64, 16, new, [s + n for s, n in zip(starts, new)], starts, extra, B_)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype,H,D,P,new", [(F32, 3, 256, 32, [2001, 0, 1500, 77]), (BF16, 5, 96, 16, [4099, 1]), (F16, 7, 32, 64, [9001]),
                                             (BF16, 1, 160, 48, [5000]), (F32, 8, 128, 64, [1, 2500]), (F16, 33, 64, 16, [1111, 0, 222])])
def test_rows_of_long_prompts(fmt, dtype, H, D, P, new):
    """Enough rows that a wave takes four times as many as it holds at once; heads that leave its last times part empty."""
    lanes = 4 if D <= 32 else 8 if D <= 64 else 16 if D <= 128 else 32
    assert -(-2 * H // (64 // lanes)) * sum(new) >= 16 * 256
    starts = [5 * i for i in range(len(new))]
    check_rows(fmt, dtype, H, D, P, new, [s + n for s, n in zip(starts, new)], starts, 2, H)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("G_,window", [(1, 0), (4, 37), (7, 1)])
def test_tiles_of_many_rows(fmt, dtype, D, G_, window):
    """Prompts among sequences without tokens and with one: from five eighths of a tile's rows to a sequence on they go by tiles."""
    new, held = ([170, 0, 129, 1, 64], [200, 3, 129, 90, 99]) if G_ == 1 else ([33, 0, 70, 1, 25], [133, 3, 70, 90, 26])
    if D > 128:
        new, held = [n // 2 for n in new], [h - n + n // 2 for h, n in zip(held, new)]
    assert 8 * sum(new) * G_ >= 5 * (128 if D <= 128 else 64) * len(new) or G_ == 1
    pool = Pool(fmt, held, 2, D, 16, seed=D + G_, halved=G_ == 4)
    fill(pool, G_)
    check_attention(pool, new, 2 * G_, dtype, window=window, seed=D, extra=2)


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_tiles_of_more_sequences_than_a_wave_has_lanes(fmt):
    rng = np.random.default_rng(5)
    new = [int(n) for n in rng.integers(0, 50, 70)]
    held = [n + int(e) for n, e in zip(new, rng.integers(0, 90, 70))]
    pool = Pool(fmt, held, 1, 64, 16, seed=2)
    fill(pool, 2)
    assert 8 * sum(new) * 4 >= 5 * 128 * 70
    check_attention(pool, new, 4, BF16, window=30)


def test_a_cache_that_is_captured_refuses_and_stays_as_it_was():
    from paper_1901_09504_amd.layer import TokenCache

    cache = TokenCache(1, 4, 2, 64, page_rows=16)
    rows = C.random_rows(20, 2, 64, BF16, 1)
    cache.append(rows, rows, [20])
    want, stream = cache.attend(rows, [20]), cache._stream
    for call in (lambda: cache.append(rows, rows, [20]), lambda: cache.attend(rows, [20]), lambda: cache.read()):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph), pytest.raises(AssertionError, match="captured"):
            call()
        assert cache.lengths == [20] and len(cache.tables[0]) == 2 and cache._stream == stream
    assert torch.equal(cache.attend(rows, [20]), want)


def test_only_sequences_are_freed():
    from paper_1901_09504_amd.layer import TokenCache

    cache = TokenCache(2, 4, 2, 64, page_rows=16)
    rows = C.random_rows(20, 2, 64, BF16, 1)
    cache.append(rows, rows, [3, 17])
    for none in (-1, 2):
        with pytest.raises(AssertionError):
            cache.free(none)
    assert cache.lengths == [3, 17] and [len(t) for t in cache.tables] == [1, 2]
    cache.free(0)
    cache.free(0)                                                            # nothing left of it: nothing happens
    assert cache.lengths == [0, 17] and sorted(cache.spare + cache.tables[1]) == [0, 1, 2, 3]


@pytest.mark.parametrize("length", [1, 5, 8, 9])
def test_scores_behind_a_cache_of_short_sequences(length):
    """8 tokens one by one behind the prompt, or as many as there are."""
    from paper_1901_09504_amd import score

    rows = score.run_cache(sequences=2, length=length, vocab=100)
    assert len(rows) == 5 and all(p >= 1 and 0 <= same <= 1 for _, _, p, same in rows)


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_a_long_run_of_generation_in_one_graph(fmt):
    """A step captured once for lengths that it does not know: positions advance on the device across pages and across the parts that the bound
    `most` gives, a sequence without tokens of its own comes and goes; every replay against the same calls made eagerly, and the last
    against 64 bits."""
    H, Hq, D, P, steps = 2, 8, 128, 64, 12
    n0 = [250, 1, 1532, 60]
    held = [n + 10 * steps for n in n0]
    pool, eager = (Pool(fmt, held, H, D, P, seed=3) for _ in range(2))
    for p in (pool, eager):
        fill(p, 3)
    most, T = 4096, 4
    cu = torch.arange(5, dtype=torch.int32, device="cuda")
    starts = torch.tensor(n0, dtype=torch.int32, device="cuda")
    kt, vt = (torch.empty((T, H, D), dtype=BF16, device="cuda") for _ in range(2))
    qt, y = (torch.empty((T, Hq, D), dtype=BF16, device="cuda") for _ in range(2))
    ws, other = C.workspace(T, 4, H, Hq, D, most), C.workspace(T, 4, H, Hq, D, most)
    assert ws is not None
    args = pool.args()

    def step(st, offsets, out, args, ws):
        B.ocs_cache_write(kt, H * D, D, vt, H * D, D, T, offsets, st, 4, *args)
        B.ocs_cache_attention(qt, Hq * D, D, Hq, T, offsets, st, 4, most, *args, 0.1, 0, out, Hq * D, D, None, ws)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(starts, cu, y, args, ws)
        starts.add_(cu.diff() * 10)                                          # (the positions between hold what fill() left there)
    eager_args, at = eager.args(), list(n0)
    for i in range(steps):
        new = [1, 0, 1, 1] if i % 3 == 2 else [1, 1, 1, 1]
        cu.copy_(torch.tensor([0] + list(np.cumsum(new))))
        kt.copy_(C.random_rows(T, H, D, BF16, 10 + i))
        vt.copy_(C.random_rows(T, H, D, BF16, 20 + i))
        qt.copy_(C.random_rows(T, Hq, D, BF16, 30 + i))
        graph.replay()
        got = y[:sum(new)].clone()
        torch.cuda.synchronize()
        want = torch.empty_like(y)
        step(torch.tensor(at, dtype=torch.int32, device="cuda"), cu.clone(), want, eager_args, other)
        assert torch.equal(got, want[:sum(new)]), i
        at = [a + 10 * n for a, n in zip(at, new)]
    assert starts.tolist() == at
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(pool.codes + pool.scales, eager.codes + eager.scales))
    pool.held = at
    check_attention(pool, [1] * 4, Hq, BF16, most=most, seed=1)
