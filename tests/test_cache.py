"""The quantized cache on the GPU: rows written bit for bit against Eq. 1 and the block grids, read back exactly, and attention over them
against 64 bits; lengths from none to long ones, pages that are missing or out of range, rubbish where nothing is seen, windows, strides,
layouts, streams, graphs and pools beyond 4 GB."""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import ref
from paper_1901_09504_amd import binding as B
from tests import gpu_util as G
from tests.test_mx import numbers, on_grids, packed

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
WEIGHT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -16}   # how far a weight of the values may be off: one, two or three bf16 numbers make it
INT8, MX4 = B.CACHE_INT8, B.CACHE_MX4


@pytest.fixture(autouse=True)
def _gpu():
    G.require_gpu()


class Pool:
    """Pages full of rubbish that is no number, a table with every sequence's pages scattered over them, and where it is on the host."""

    def __init__(self, fmt, held, H, D, P, seed=0, halved=False, spare=3):
        rng = np.random.default_rng(seed)
        need = [-(-L // P) for L in held]
        self.fmt, self.H, self.D, self.P, self.pages, self.held = fmt, H, D, P, sum(need) + spare, held
        order = rng.permutation(self.pages)
        self.table = np.full((len(held), max(max(need, default=1), 1) + 2), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.pages, H, P)
        width, per = (D, ()) if fmt == INT8 else (D // 2, (D // 32,))
        dtype = torch.int8 if fmt == INT8 else torch.uint8
        self.codes = [torch.randint(-128 if fmt == INT8 else 0, 128 if fmt == INT8 else 256, shape + (width,), dtype=dtype,
                                    generator=torch.Generator().manual_seed(seed + i)).cuda() for i in (1, 2)]
        if fmt == INT8:
            rubbish = torch.tensor([torch.nan, torch.inf, -torch.inf, 3e38])
            self.scales = [rubbish[torch.randint(0, 4, shape, generator=torch.Generator().manual_seed(seed + i))].cuda() for i in (3, 4)]
        else:
            self.scales = [torch.randint(253, 256, shape + per, dtype=torch.uint8, generator=torch.Generator().manual_seed(seed + i)).cuda()
                           for i in (3, 4)]
        self.depth = [torch.from_numpy(rng.integers(0, 4, (H, D)).astype(np.int32)).cuda() if halved else None for _ in range(2)]

    def args(self, table=None):
        t = G.dev(self.table) if table is None else table
        self._kept = t                                                       # (until the call's work is done)
        return (t, t.shape[1], t.stride(0), self.fmt, self.codes[0], self.scales[0], self.codes[1], self.scales[1], self.pages, self.P, self.H,
                self.D, self.depth[0], self.depth[1])

    def numbers(self, which):
        """[pages, H, P, D] in 64 bits on the device."""
        c, s = self.codes[which], self.scales[which]
        if self.fmt == INT8:
            v = c.double() * s.double()[..., None]
        else:
            both = torch.stack([c & 15, c >> 4], -1).flatten(-2).long()
            grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
            size = torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127))
            v = torch.cat([grid, -grid])[both] * size.repeat_interleave(32, -1)
        return v if self.depth[which] is None else v * torch.exp2(self.depth[which].double())[:, None, :]

    def row(self, b, j):
        return int(self.table[b, j // self.P]), j % self.P


def tokens_of(new, starts):
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return G.dev(cu), G.dev(np.array(starts, dtype=np.int32)), cu


def write(pool, k, v, new, starts, T=None):
    cu, st, _ = tokens_of(new, starts)
    B.ocs_cache_write(k, k.stride(0), k.stride(1), v, v.stride(0), v.stride(1), k.shape[0] if T is None else T, cu, st, len(new), *pool.args())


def read(pool, dtype, n, starts, extra=0):
    T = sum(n) + extra
    out = [torch.full((T, pool.H, pool.D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    cu, st, _ = tokens_of(n, starts)
    B.ocs_cache_read(out[0], out[0].stride(0), out[0].stride(1), out[1], out[1].stride(0), out[1].stride(1), T, cu, st, len(n), *pool.args())
    return out


def random_rows(T, H, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, H, D), generator=g) * torch.exp2(torch.randint(-6, 4, (T, H, 1), generator=g).float())
    x[:, :, ::11] *= 9
    return x.to(dtype).cuda()


def grid_rows(x, fmt, depth):
    """fp32 rows [n, D] -> what the pool holds of them."""
    if depth is not None:
        x = (x * np.ldexp(np.float32(1), -depth.astype(np.int64)).astype(np.float32)).astype(np.float32)
    if fmt == MX4:
        codes, scales = on_grids(x)
        bad = ~np.isfinite(x).all(1)
        codes[bad], scales[bad] = 0, 255
        return packed(codes, x.shape[1] // 2), scales
    got = [ref.quantize(np.ascontiguousarray(r[None]), 8, ldq=x.shape[1]) for r in x]
    return np.concatenate([q for q, _ in got]), np.array([s[1] for _, s in got], dtype=np.float32)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("H,D,P", [(1, 32, 16), (2, 64, 32), (3, 96, 16), (8, 128, 64), (5, 160, 48), (2, 192, 16), (1, 224, 16), (4, 256, 128)])
@pytest.mark.parametrize("halved", [False, True])
def test_rows_written_and_read(fmt, dtype, H, D, P, halved):
    new, held = [3, 0, 1, 40, 17], [3, 5, 70, 40, 129]
    starts = [h - n for h, n in zip(held, new)]
    pool = Pool(fmt, held, H, D, P, seed=D, halved=halved)
    before = [t.clone() for t in pool.codes + pool.scales]
    k, v = random_rows(sum(new), H, D, dtype, 1), random_rows(sum(new), H, D, dtype, 2)
    k[0, 0], v[1, H - 1] = 0, 0
    write(pool, k, v, new, starts)
    where = [pool.row(b, starts[b] + i) for b in range(len(new)) for i in range(new[b])]
    page, row = torch.tensor([w[0] for w in where]), torch.tensor([w[1] for w in where])
    touched = torch.zeros((pool.pages, P), dtype=torch.bool)
    touched[page, row] = True
    for i, x in enumerate((k, v)):
        depth = None if pool.depth[i] is None else np.tile(G.host(pool.depth[i]), (len(where), 1))
        codes, scales = grid_rows(G.host(x.float()).reshape(-1, D), fmt, depth)
        got, gs = G.host(pool.codes[i][page, :, row]), G.host(pool.scales[i][page, :, row])
        assert np.array_equal(got.reshape(codes.shape), codes)
        assert np.array_equal(gs.reshape(scales.shape).view(np.uint8), scales.view(np.uint8))
        rest = (~touched).cuda()[:, None, :].expand(-1, H, -1)
        assert torch.equal(pool.codes[i][rest], before[i][rest])             # every other row is as it was
        assert torch.equal(pool.scales[i][rest].view(torch.uint8), before[2 + i][rest].view(torch.uint8))
    back = read(pool, dtype, new, starts)
    for i in range(2):
        want = pool.numbers(i)[page.cuda(), :, row.cuda()]
        # a 32-bit product of code and step, then the type's rounding
        err = (back[i].double() - want).abs()
        assert bool((err <= (HALF_STEP[dtype] + (2.0 ** -24 if fmt == INT8 else 0)) * want.abs() * 1.01 + (2.0 ** -25 if dtype == F16 else 0)).all())


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_rows_of_any_layout(fmt):
    H, D = 3, 64
    pool, other = (Pool(fmt, [9, 8], H, D, 16, seed=4) for _ in range(2))
    k, v = random_rows(9, H, D, BF16, 1), random_rows(9, H, D, BF16, 2)
    write(pool, k, v, [5, 4], [4, 4])
    wide = torch.empty((H, 10, D + 7), dtype=BF16, device="cuda")
    kk, vv = wide[:, :9, 3:D + 3].transpose(0, 1), torch.empty((9, H + 2, D), dtype=BF16, device="cuda")[:, 1:H + 1]
    kk.copy_(k)
    vv.copy_(v)
    write(other, kk, vv, [5, 4], [4, 4])
    for a, b in zip(pool.codes + pool.scales, other.codes + other.scales):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    buf = torch.full((H, 9, D + 1), 7.0, device="cuda")
    cu, st, _ = tokens_of([5, 4], [4, 4])
    plain = read(pool, F32, [5, 4], [4, 4])
    out = torch.empty((9, H, D), device="cuda")
    B.ocs_cache_read(buf, D + 1, 9 * (D + 1), out, H * D, D, 9, cu, st, 2, *pool.args())
    assert torch.equal(buf[:, :, :D].transpose(0, 1), plain[0]) and torch.equal(out, plain[1]) and bool((buf[:, :, D] == 7).all())


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_positions_without_a_page_and_tokens_without_a_sequence(fmt):
    H, D, P = 2, 32, 16
    pool = Pool(fmt, [40, 20], H, D, P, seed=1)
    pool.table[0, 1] = -7
    pool.table[1, 0] = pool.pages
    before = [t.clone() for t in pool.codes + pool.scales]
    T = 60
    k, v = random_rows(T + 5, H, D, F32, 1), random_rows(T + 5, H, D, F32, 2)
    write(pool, k, v, [40, 20], [0, 0])
    out = read(pool, F32, [40, 20], [0, 0], extra=5)
    for x, y in zip((k, v), out):
        gone = torch.zeros(T, dtype=torch.bool)
        gone[16:32] = True
        gone[40:56] = True
        assert not bool(y[:T][gone].any()) and bool((y[T:] == 7).all())
        big = x[:T][~gone].abs().amax(-1, keepdim=True)
        assert bool(((y[:T][~gone] - x[:T][~gone]).abs() <= big * (1 / 200 if fmt == INT8 else 1 / 4)).all())
    used = {int(p) for p in pool.table[0, [0, 2]]} | {int(pool.table[1, 1])}
    for p in set(range(pool.pages)) - used:
        for a, b in zip(pool.codes + pool.scales, before):
            assert torch.equal(a[p].view(torch.uint8), b[p].view(torch.uint8))
    # positions beyond the table, before the sequence, and far beyond 32 bits of rows
    write(pool, k, v, [30, 30], [pool.table.shape[1] * P - 3, -40])
    for far in read(pool, F32, [30, 30], [pool.table.shape[1] * P, -31]):
        assert not bool(far.any())
    assert not any(bool(far.any()) for far in read(pool, F32, [30, 30], [2 ** 31 - 40, -2 ** 31]))


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("bad", [torch.nan, torch.inf])
def test_rows_that_are_no_numbers(fmt, bad):
    pool = Pool(fmt, [6], 2, 64, 16, seed=2)
    k, v = random_rows(6, 2, 64, F32, 1), random_rows(6, 2, 64, F32, 2)
    k[2, 1, 40], v[5, 0, 0] = bad, bad
    write(pool, k, v, [6], [0])
    for i, (t, h) in enumerate(((2, 1), (5, 0))):
        s = pool.scales[i][pool.table[0, 0], :, :6].float()
        s = s if fmt == INT8 else torch.where(s == 255, torch.nan, s).amin(-1)
        ok = s.isfinite()
        assert not bool(ok[h, t]) and int(ok.sum()) == 11
    if fmt == MX4:
        back = read(pool, F32, [6], [0])
        assert bool(back[0][2, 1].isnan().all()) and int(back[0].isnan().sum()) == 64


# ---- attention -------------------------------------------------------------------------------

def workspace(T, n, H, Hq, D, most, window=0):
    need = B.ocs_cache_attention_workspace_bytes(T, n, H, Hq, D, most, window)
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None


def fill(pool, seed):
    """Codes and scales of every position that the table has up to the sequences' ends; the rest stays rubbish."""
    g = torch.Generator().manual_seed(seed)
    for b, L in enumerate(pool.held):
        for p0 in range(0, L, pool.P):
            page, n = int(pool.table[b, p0 // pool.P]), min(pool.P, L - p0)
            if not 0 <= page < pool.pages:
                continue
            for i in range(2):
                if pool.fmt == INT8:
                    pool.scales[i][page, :, :n] = (torch.rand((pool.H, n), generator=g) * 0.02 + 0.001).cuda()
                else:
                    pool.scales[i][page, :, :n] = torch.randint(122, 128, (pool.H, n, pool.D // 32), dtype=torch.uint8, generator=g).cuda()


def seen_of(pool, b, p, window, most):
    lo = max(0, p - window + 1) if window else 0
    return [j for j in range(lo, min(p + 1, most, pool.table.shape[1] * pool.P)) if 0 <= pool.table[b, j // pool.P] < pool.pages]


def check_attention(pool, new, Hq, dtype, window=0, scale=None, seed=0, sharp=1.0, extra=0, most=None, lse=True, q=None, y=None):
    """One call against 64 bits.  A score is off by its 32-bit products' and sums' roundings: (D + 8) steps of 2^-23 of the sum of its
    products' sizes at most, and by 4 steps of itself as an exponent of 2; a weight by twice that, its own rounding and the exponential's; the
    sums by a step for each 32 positions, in which the order of the parts' joining is counted."""
    H, D, held = pool.H, pool.D, pool.held
    T, starts = sum(new), [L - n for L, n in zip(held, new)]
    scale = 1 / math.sqrt(D) if scale is None else scale
    most = max(held) if most is None else most
    if q is None:
        q = (torch.randn((T + extra, Hq, D), generator=torch.Generator().manual_seed(seed)) * sharp).to(dtype).cuda()
    if y is None:
        y = torch.full((T + extra, Hq, D), 7.0, dtype=dtype, device="cuda")
    out_lse = torch.full((T + extra, Hq), 7.0, device="cuda") if lse else None
    cu, st, host_cu = tokens_of(new, starts)
    ws = workspace(T + extra, len(new), H, Hq, D, most, window)
    B.ocs_cache_attention(q, q.stride(0), q.stride(1), Hq, T + extra, cu, st, len(new), most, *pool.args(), scale, window, y, y.stride(0),
                          y.stride(1), out_lse, ws)
    k, v = pool.numbers(0), pool.numbers(1)
    for b in range(len(new)):
        for i in range(new[b]):
            t, seen = int(host_cu[b]) + i, seen_of(pool, b, starts[b] + i, window, most)
            if not seen:
                assert not bool(y[t].any()) and (not lse or bool((out_lse[t] == -math.inf).all()))
                continue
            page = torch.tensor([int(pool.table[b, j // pool.P]) for j in seen], device="cuda")
            row = torch.tensor([j % pool.P for j in seen], device="cuda")
            kk = k[page, :, row].repeat_interleave(Hq // H, 1)               # [n, Hq, D]
            vv = v[page, :, row].repeat_interleave(Hq // H, 1)
            s = (kk * q[t].double()).sum(-1) * scale                         # [n, Hq]
            size = (kk * q[t].double()).abs().sum(-1) * abs(scale)
            want_lse = torch.logsumexp(s, 0)
            w = torch.exp(s - want_lse)
            want, spread = (w[..., None] * vv).sum(0), (w[..., None] * vv.abs()).sum(0)
            off = ((D + 8) * 2.0 ** -23 * size + 4 * 2.0 ** -23 * s.abs()).amax(0) + (len(seen) / 32 + 24) * 2.0 ** -23
            tol = spread * (2 * off + WEIGHT[dtype])[:, None] * 1.05 + HALF_STEP[dtype] * want.abs() + (2.0 ** -25 if dtype == F16 else 0)
            # Below 2^-126 a number may be 0: each of a weight's three parts at most, times a number of at most 128 steps, for every
            # position.  (Seen where a column's only weight is the last of a sharp row: 4.5e-39, off by 0.25e-39.)
            tol += len(seen) * 3 * 128 * 2.0 ** -126
            err = (y[t].double() - want).abs()
            assert bool((err <= tol).all()), (b, i, float((err / tol).max()))
            if lse:
                assert bool(((out_lse[t].double() - want_lse).abs() <= off + 2.0 ** -22 * want_lse.abs()).all()), (b, i)
    assert bool((y[T:] == 7).all()) and (not lse or bool((out_lse[T:] == 7).all()))
    return y[:T], out_lse[:T] if lse else None


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("halved", [False, True])
def test_single_tokens(fmt, dtype, D, halved):
    held = [1, 2, 15, 16, 17, 33, 64, 100, 257]
    pool = Pool(fmt, held, 2, D, 16, seed=D, halved=halved)
    fill(pool, D)
    check_attention(pool, [1] * len(held), 6, dtype, sharp=2.0)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("G,H,D,P,window", [(1, 1, 64, 16, 0), (4, 2, 128, 64, 0), (8, 1, 96, 32, 20), (3, 2, 128, 16, 1), (16, 1, 32, 16, 0),
                                            (5, 3, 64, 48, 33), (20, 1, 64, 16, 0), (1, 5, 256, 32, 64), (2, 2, 192, 16, 7)])
def test_tokens_of_many_lengths(fmt, dtype, G, H, D, P, window):
    new, held = [1, 0, 5, 16, 33, 2, 70, 0], [1, 9, 5, 100, 47, 130, 70, 0]
    pool = Pool(fmt, held, H, D, P, seed=G + D)
    fill(pool, G)
    check_attention(pool, new, G * H, dtype, window=window, seed=P, extra=3)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new,held,window", [([1], [5000], 0), ([1, 1], [3001, 17], 0), ([2, 1], [2500, 4099], 700), ([300], [1300], 0),
                                             ([300, 200], [310, 1200], 128), ([513], [513], 0)])
def test_long_sequences(fmt, dtype, new, held, window):
    pool = Pool(fmt, held, 1, 128, 64, seed=len(held))
    fill(pool, 5)
    check_attention(pool, new, 4, dtype, window=window)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("new,held", [([1, 1, 1], [100, 60, 3000]), ([20, 3, 40], [100, 60, 3000]), ([200, 3, 130], [300, 60, 3000])])
def test_missing_pages_and_tokens_that_see_nothing(fmt, new, held):
    pool = Pool(fmt, held, 2, 64, 16, seed=9)
    pool.table[0, :] = -1                                                    # a sequence without any page
    pool.table[1, 1:3] = pool.pages + 5
    pool.table[2, 3:150] = -2 ** 31
    pool.table[2, 187] = 2 ** 31 - 1
    fill(pool, 1)
    for window in (0, 40):
        check_attention(pool, new, 4, BF16, window=window)
    check_attention(pool, new, 4, F32, most=50)                              # nothing is looked at from there on
    check_attention(pool, new, 4, F32, most=0)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sharp_rows_and_large_scores(fmt, dtype):
    held = [200, 333, 31]
    pool = Pool(fmt, held, 2, 64, 16, seed=3)
    fill(pool, 2)
    for scale in (0.125, 3.0, -1.0, 0.0):
        check_attention(pool, [1, 40, 31], 4, dtype, scale=scale, sharp=4.0)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("many", [False, True])
def test_rows_that_are_no_numbers_reach_only_those_who_see_them(fmt, dtype, many):
    held = [90, 90]
    new = [60, 60] if many else [3, 3]
    pool = Pool(fmt, held, 1, 64, 16, seed=8)
    fill(pool, 8)
    at = 88
    for which, b in ((0, 0), (1, 1)):
        page, row = pool.row(b, at)
        pool.scales[which][page, :, row] = torch.nan if fmt == INT8 else 255
    q = torch.randn((sum(new), 2, 64), generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
    y = torch.empty_like(q)
    cu, st, _ = tokens_of(new, [90 - n for n in new])
    B.ocs_cache_attention(q, 128, 64, 2, sum(new), cu, st, 2, 90, *pool.args(), 0.1, 0, y, 128, 64, None,
                          workspace(sum(new), 2, 1, 2, 64, 90))
    sees = torch.zeros(sum(new), dtype=torch.bool)
    for b in range(2):
        sees[sum(new[:b]) + at - (90 - new[b]):sum(new[:b + 1])] = True
    assert bool(y[sees].isnan().all()) and not bool(y[~sees].isnan().any())


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [1, 60])
def test_a_value_that_is_no_number_far_below_the_largest_score(fmt, dtype, new):
    # its weight is 0 beside the largest, in a part of its own of the positions
    L = 2048
    pool = Pool(fmt, [L], 1, 64, 16, seed=12)
    k, v = torch.zeros((L, 1, 64), device="cuda"), random_rows(L, 1, 64, F32, 13)
    k[1500] = 8
    v[10, 0, 5] = torch.nan
    write(pool, k, v, [L], [0])
    assert workspace(new, 1, 1, 2, 64, L) is not None
    q = torch.full((new, 2, 64), 8.0, dtype=dtype, device="cuda")
    q[:, 1] = 0
    for window in (0, 1024):
        y = torch.zeros_like(q)
        cu, st, _ = tokens_of([new], [L - new])
        B.ocs_cache_attention(q, 128, 64, 2, new, cu, st, 1, L, *pool.args(), 1.0, window, y, 128, 64, None,
                              workspace(new, 1, 1, 2, 64, L, window))
        assert bool(y.isnan().all()) if window == 0 else bool(y.isfinite().all())
        if window:
            # position 1500's value: its weight and the output rounded, half a step each, sums and the quotient in 32 bits; of the others less
            # than 2048 times the largest value (2^9) times 2^-126
            page, row = pool.row(0, 1500)
            want = pool.numbers(1)[page, 0, row]
            assert bool(((y[:, 0].double() - want).abs() <= want.abs() * (torch.finfo(dtype).eps + 2.0 ** -22) + 2.0 ** -106).all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("new", [[1, 1], [40, 3]])
def test_layouts_of_queries_and_outputs(dtype, new):
    pool = Pool(INT8, [77, 40], 2, 96, 16, seed=6)
    fill(pool, 6)
    T = sum(new)
    plain, lse = check_attention(pool, new, 4, dtype)
    q = torch.empty((4, T + 1, 99), dtype=dtype, device="cuda")[:, :T, 1:97].transpose(0, 1)
    q.copy_(torch.randn((T, 4, 96), generator=torch.Generator().manual_seed(0)).to(dtype))
    y = torch.full((T, 5, 99), 7.0, dtype=dtype, device="cuda")
    got, _ = check_attention(pool, new, 4, dtype, q=q, y=y[:, 1:, 2:98], lse=False)
    assert torch.equal(got, plain)
    assert bool((y[:, 0] == 7).all()) and bool((y[:, :, :2] == 7).all()) and bool((y[:, :, 98:] == 7).all())


def test_many_sequences_and_the_search_for_them():
    """More sequences than a wave has lanes, most of them without tokens; offsets that are no offsets do not fault."""
    rng = np.random.default_rng(0)
    new = [int(n) for n in rng.choice([0, 0, 0, 1, 2, 19], 300)]
    held = [n + int(e) for n, e in zip(new, rng.integers(0, 40, 300))]
    pool = Pool(INT8, held, 1, 32, 16, seed=1)
    fill(pool, 1)
    check_attention(pool, new, 2, F32)
    T = sum(new)
    q = torch.zeros((T, 2, 32), device="cuda")
    y = torch.empty_like(q)
    for cu in (torch.full((301,), -5), torch.full((301,), 2 ** 30), torch.arange(300, -1, -1) * 7, torch.arange(301) * 1000):
        B.ocs_cache_attention(q, 64, 32, 2, T, cu.to(torch.int32).cuda(), torch.zeros(300, dtype=torch.int32, device="cuda"), 300, 59,
                              *pool.args(), 0.1, 0, y, 64, 32, None, workspace(T, 300, 1, 2, 32, 59))
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_a_pool_beyond_32_bits(fmt):
    H, D, P = 8, 256, 256
    pages = (2 ** 32 // (H * P * (D if fmt == INT8 else D // 2))) + 40
    pool = Pool(fmt, [300, 300], H, D, P, seed=0, spare=0)
    small = pool.pages
    pool.codes = [torch.zeros((pages,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda") for t in pool.codes]
    pool.scales = [torch.zeros((pages,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda") for t in pool.scales]
    pool.pages = pages
    pool.table[pool.table >= 0] += pages - small
    k, v = random_rows(600, H, D, BF16, 1), random_rows(600, H, D, BF16, 2)
    write(pool, k, v, [300, 300], [0, 0])
    near = Pool(fmt, [300, 300], H, D, P, seed=0, spare=0)
    write(near, k, v, [300, 300], [0, 0])
    for a, b in zip(read(pool, BF16, [300, 300], [0, 0]), read(near, BF16, [300, 300], [0, 0])):
        assert torch.equal(a, b)
    q = torch.randn((2, 16, D), device="cuda").to(BF16)
    ys = []
    for p in (pool, near):
        y = torch.empty_like(q)
        cu, st, _ = tokens_of([1, 1], [299, 299])
        ws = workspace(2, 2, H, 16, D, 300)
        B.ocs_cache_attention(q, 16 * D, D, 16, 2, cu, st, 2, 300, *p.args(), 0.06, 0, y, 16 * D, D, None, ws)
        ys.append(y)
    assert torch.equal(*ys)


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_a_run_of_generation_with_its_layers_in_a_graph(fmt):
    """Prompts written and attended, then tokens one by one: each step's write and attention are one captured graph, whose lengths advance
    on the device; every replay against the same calls made eagerly, with other work and synchronizations between."""
    H, Hq, D, P, n0 = 2, 4, 64, 16, [30, 7]
    steps, scale = 5, 0.125
    pool, eager = (Pool(fmt, [n + steps for n in n0], H, D, P, seed=3) for _ in range(2))
    k, v, q = (random_rows(sum(n0), h, D, BF16, s) for h, s in ((H, 1), (H, 2), (Hq, 3)))
    most = max(n0) + steps
    for p in (pool, eager):
        write(p, k, v, n0, [0, 0])
    cu = torch.arange(3, dtype=torch.int32, device="cuda")
    starts = torch.tensor(n0, dtype=torch.int32, device="cuda")
    kt, vt = (torch.empty((2, H, D), dtype=BF16, device="cuda") for _ in range(2))
    qt, y = (torch.empty((2, Hq, D), dtype=BF16, device="cuda") for _ in range(2))
    ws = workspace(2, 2, H, Hq, D, most)
    args = pool.args()

    def step(p, st, out, args):
        B.ocs_cache_write(kt, H * D, D, vt, H * D, D, 2, cu, st, 2, *args)
        B.ocs_cache_attention(qt, Hq * D, D, Hq, 2, cu, st, 2, most, *args, scale, 0, out, Hq * D, D, None, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(pool, starts, y, args)
        starts.add_(1)
    eager_args = eager.args()
    for i in range(steps):
        kt.copy_(random_rows(2, H, D, BF16, 10 + i))
        vt.copy_(random_rows(2, H, D, BF16, 20 + i))
        qt.copy_(random_rows(2, Hq, D, BF16, 30 + i))
        graph.replay()
        got = y.clone()
        torch.cuda.synchronize()
        want = torch.empty_like(y)
        step(eager, torch.tensor([n + i for n in n0], dtype=torch.int32, device="cuda"), want, eager_args)
        assert torch.equal(got, want), i
    assert starts.tolist() == [n + steps for n in n0]


# ---- the cache that keeps its pages ----------------------------------------------------------

def _pool_of(cache):
    """The tests' view of a TokenCache's sequences."""
    pool = Pool.__new__(Pool)
    pool.fmt, pool.H, pool.D, pool.P, pool.pages = cache.format, cache.heads, cache.D, cache.page_rows, cache.pages
    pool.held = list(cache.lengths)
    pool.table = np.full((cache.sequences, max(1, max(len(t) for t in cache.tables))), -1, dtype=np.int32)
    for b, t in enumerate(cache.tables):
        pool.table[b, :len(t)] = t
    pool.codes, pool.scales, pool.depth = [cache.keys, cache.values], [cache.key_scales, cache.value_scales], [cache.key_depth, cache.value_depth]
    return pool


@pytest.mark.parametrize("bits", [8, 4])
def test_sequences_come_grow_and_go(bits):
    from paper_1901_09504_amd.layer import TokenCache, outlier_depths

    H, Hq, D = 2, 6, 64
    sample = random_rows(100, H, D, F32, 5)
    depths = outlier_depths(sample, 0.1)
    assert depths.shape == (H, D) and int(depths.max()) >= 1 and bool((depths[:, 11::11] >= 0).all())
    cache = TokenCache(3, 12, H, D, page_rows=16, bits=bits, key_depth=depths)
    seed = 0
    for which, counts, freed in (([0, 2], [20, 5], None), (None, [1, 0, 1], None), ([1], [40], None), ([0, 1, 2], [1, 1, 1], 1), ([1, 0], [17, 30], None)):
        seq = [0, 1, 2] if which is None else which
        k, v, q = (random_rows(sum(counts), h, D, BF16, seed + i) for i, h in enumerate((H, H, Hq)))
        seed += 3
        cache.append(k, v, counts, which)
        y, lse = cache.attend(q, counts, which, with_lse=True)
        pool = _pool_of(cache)
        new = [0, 0, 0]
        for b, n in zip(seq, counts):
            new[b] = n
        order = [sum(counts[:seq.index(b)]) + i for b in range(3) for i in range(new[b])]     # the tests' tokens are in the sequences' order
        want, want_lse = check_attention(pool, new, Hq, BF16, q=q[order].contiguous())
        # the call's parts may be others than the checked one's, whose table is wider: both are within the tolerance of the 64-bit values
        assert bool(((y[order].float() - want.float()).abs() <= 2.0 ** -6 * want.float().abs() + 2.0 ** -6 * v.float().abs().max()).all())
        assert bool(((lse[order] - want_lse).abs() <= 1e-4 * (1 + want_lse.abs())).all())
        back = cache.read()
        assert back[0].shape == (sum(cache.lengths), H, D)
        if freed is not None:
            cache.free(freed)
            assert cache.lengths[freed] == 0
    assert sorted(cache.spare + sum(cache.tables, [])) == list(range(12))
    before = [list(t) for t in cache.tables], list(cache.lengths), list(cache.spare)
    with pytest.raises(MemoryError):
        cache.append(random_rows(200, H, D, BF16, 1), random_rows(200, H, D, BF16, 2), [200], [0])
    assert before == ([list(t) for t in cache.tables], list(cache.lengths), list(cache.spare))
    side = torch.cuda.Stream()
    plain = cache.read()
    with torch.cuda.stream(side):
        again = cache.read()
    side.synchronize()
    assert torch.equal(plain[0], again[0]) and torch.equal(plain[1], again[1])


def test_a_cache_refuses_what_does_not_fit():
    from paper_1901_09504_amd.layer import TokenCache

    cache = TokenCache(2, 4, 2, 32, page_rows=16)
    k = random_rows(3, 2, 32, F32, 1)
    for K, V, counts, which in ((k, k, [3], None), (k, k, [1, 1], None), (k, k, [1, 2], [0, 0]), (k, k.to(BF16), [1, 2], None), (k, k, [3], [2]),
                                (k.cpu(), k, [1, 2], None), (k[:, :1], k, [1, 2], None), (k, k, [4, -1], None)):
        with pytest.raises(AssertionError):
            cache.append(K, V, counts, which)
    cache.append(k, k, [1, 2])
    with pytest.raises(AssertionError):
        cache.attend(k, [2, 1])                                              # more queries than positions
    with pytest.raises(AssertionError):
        TokenCache(2, 4, 2, 32, bits=5)
    cache = TokenCache(2, 4, 2, 32)
    with pytest.MonkeyPatch.context() as m, pytest.raises(AssertionError, match="device"):
        m.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(device=torch.device("cuda", 1)))
        cache.read()
    with pytest.raises(B.OcsError):
        TokenCache(2, 4, 2, 48).append(random_rows(2, 2, 48, F32, 1), random_rows(2, 2, 48, F32, 1), [1, 1])


def test_scores_behind_a_quantized_cache():
    from paper_1901_09504_amd import score

    rows = score.run_cache(sequences=2, length=40, vocab=500)
    assert [(b, r) for b, r, _, _ in rows] == [(32, 0.0), (8, 0.0), (8, 0.1), (4, 0.0), (4, 0.1)]
    assert all(math.isfinite(p) and p >= 1 and 0 <= same <= 1 for _, _, p, same in rows)


# ---- what the calls above do not reach -------------------------------------------------------

@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("D,P", [(64, 16), (160, 1024), (224, 32)])
def test_prompts_of_more_sequences_than_a_wave_has_lanes(fmt, D, P):
    rng = np.random.default_rng(D)
    new = [int(n) for n in rng.integers(0, 60, 70)]
    held = [n + int(e) for n, e in zip(new, rng.integers(0, 90, 70))]
    pool = Pool(fmt, held, 1, D, P, seed=2)
    fill(pool, 2)
    check_attention(pool, new, 2, BF16, window=50)


@pytest.mark.parametrize("fmt", [INT8, MX4])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("new,held,window", [([70], [2900], 0), ([70], [2900], 1500), ([130, 3], [2050, 700], 0)])
def test_prompts_whose_positions_are_shared_by_workgroups(fmt, dtype, new, held, window):
    pool = Pool(fmt, held, 1, 64, 32, seed=7, halved=True)
    fill(pool, 7)
    assert B.ocs_cache_attention_workspace_bytes(sum(new), len(new), 1, 2, 64, max(held), window) > 0
    check_attention(pool, new, 2, dtype, window=window)


@pytest.mark.parametrize("new", [[1, 1], [90, 40]])
def test_a_captured_attention_in_parts_and_the_same_bits_each_time(new):
    """A graph of its own workspace on a side stream, eager calls of other lengths between the replays; no sum depends on an order that changes."""
    held = [2500, 1900]
    pool = Pool(INT8, held, 2, 128, 64, seed=1)
    fill(pool, 1)
    T, args = sum(new), pool.args()
    cu, st, _ = tokens_of(new, [h - n for h, n in zip(held, new)])
    q = torch.randn((T, 4, 128), device="cuda").to(BF16)
    ys = [torch.empty_like(q) for _ in range(2)]
    wss = [workspace(T, 2, 2, 4, 128, 2500) for _ in range(2)]
    assert wss[0] is not None

    def call(y, ws, stream=None):
        B.ocs_cache_attention(q, 512, 128, 4, T, cu, st, 2, 2500, *args, 0.1, 0, y, 512, 128, None, ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(ys[1], wss[1], stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(ys[0], wss[0])
    for seed in range(4):
        q.copy_(torch.randn((T, 4, 128), generator=torch.Generator().manual_seed(seed)))
        ys[0].fill_(3.0)
        graph.replay()
        got = ys[0].clone()
        torch.cuda.synchronize()
        call(ys[1], wss[1])
        assert torch.equal(got, ys[1])
        check_attention(pool, [1, 1], 4, F32, seed=seed)


def test_written_and_read_on_another_stream():
    pool, other = (Pool(MX4, [50], 2, 64, 16, seed=5) for _ in range(2))
    k, v = random_rows(50, 2, 64, F16, 1), random_rows(50, 2, 64, F16, 2)
    write(pool, k, v, [50], [0])
    cu, st, _ = tokens_of([50], [0])
    out = [torch.empty_like(k) for _ in range(2)]
    args = other.args()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.ocs_cache_write(k, 128, 64, v, 128, 64, 50, cu, st, 1, *args, stream=side)
    B.ocs_cache_read(out[0], 128, 64, out[1], 128, 64, 50, cu, st, 1, *args, stream=side)
    side.synchronize()
    for a, b in zip(out, read(pool, F16, [50], [0])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", [INT8, MX4])
def test_queries_that_are_no_numbers_stay_alone(fmt):
    pool = Pool(fmt, [100, 100], 1, 64, 16, seed=3)
    fill(pool, 3)
    for new in ([1, 1], [80, 80]):
        T = sum(new)
        q = torch.randn((T, 2, 64), generator=torch.Generator().manual_seed(1)).cuda()
        cu, st, _ = tokens_of(new, [100 - n for n in new])
        y, z = torch.empty_like(q), torch.empty_like(q)
        for to in (y, z):
            B.ocs_cache_attention(q, 128, 64, 2, T, cu, st, 2, 100, *pool.args(), 0.1, 0, to, 128, 64, None, workspace(T, 2, 1, 2, 64, 100))
            q[0, 1, 5] = torch.nan
        assert bool(z[0, 1].isnan().all())
        z[0, 1], y[0, 1] = 0, 0
        assert torch.equal(y, z)
