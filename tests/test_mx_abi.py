"""Refusals of the calls on microscaled 4-bit grids and of the quantized cache, on the host (no GPU): every argument error is found
before any device work, and no tokens are no work."""
import pytest
import torch

from paper_1901_09504_amd import binding as B

A = 1 << 20  # a fake, suitably aligned device address: validation never dereferences it


def _quantize(X=A, type=0, M=4, C=40, g=1, ldx=40, src=A, depth=None, s=3, q=A, ldq=32, sc=A, lds=16):
    return B.lib().ocs_split_quantize_mx(X, type, M, C, g, ldx, src, depth, s, q, ldq, sc, lds, None)


def _values(q=A, ldq=32, sc=A, lds=16, M=4, cols=43, Y=A, out=0, ldy=43):
    return B.lib().ocs_dequantize_mx(q, ldq, sc, lds, M, cols, Y, out, ldy, None)


def _product(xq=A, ldx=32, xs=A, ldxs=16, wq=A, ldw=32, ws=A, ldws=16, M=4, N=10, K=43, bias=None, Y=A, out=0, ldy=10):
    return B.lib().ocs_qgemm_mx(xq, ldx, xs, ldxs, wq, ldw, ws, ldws, M, N, K, bias, Y, out, ldy, None)


def _forward(X=A, type=0, M=4, C=40, g=1, ldx=40, src=A, s=3, q=A, ldq=32, sc=A, lds=16, wq=A, ldw=32, ws=A, ldws=16, N=10, bias=None, Y=A,
             out=0, ldy=10):
    return B.lib().ocs_forward_mx(X, type, M, C, g, ldx, src, s, q, ldq, sc, lds, wq, ldw, ws, ldws, N, bias, Y, out, ldy, None)


def test_pitches():
    for cols, q, s in ((0, 0, 0), (1, 128, 16), (256, 128, 16), (257, 256, 16), (512, 256, 16), (513, 384, 32), (4178, 2176, 144)):
        assert B.ocs_mx_code_pitch(cols) == q and B.ocs_mx_scale_pitch(cols) == s


def test_quantize_refusals():
    for name in ("X", "q", "sc", "src"):
        assert _quantize(**{name: None}) == -1, name
    assert _quantize(type=3) == -11
    for bad in (dict(M=-1), dict(C=0), dict(g=0), dict(ldx=39), dict(ldq=16), dict(lds=1), dict(M=(1 << 31) + 1), dict(ldq=1 << 32)):
        assert _quantize(**bad) == -2, bad
    assert _quantize(C=1, s=2, g=1 << 29, ldx=1 << 29, ldq=1 << 30, lds=1 << 27) == -2
    for bad in (dict(ldq=40), dict(lds=24), dict(q=A + 8), dict(sc=A + 4), dict(X=A + 2), dict(X=A + 1, type=1)):
        assert _quantize(**bad) == -3, bad
    assert _quantize(s=-1) == -5 and _quantize(C=7000, ldx=7000, s=1001, ldq=4016, lds=256) == -5


def test_values_refusals():
    for name in ("q", "sc", "Y"):
        assert _values(**{name: None}) == -1, name
    assert _values(out=3) == -11
    for bad in (dict(M=-1), dict(cols=0), dict(ldy=42), dict(ldq=16), dict(lds=0)):
        assert _values(**bad) == -2, bad
    for bad in (dict(ldq=40), dict(lds=17), dict(Y=A + 2), dict(q=A + 1)):
        assert _values(**bad) == -3, bad


def test_product_refusals():
    for name in ("xq", "xs", "wq", "ws", "Y"):
        assert _product(**{name: None}) == -1, name
    assert _product(out=7) == -11
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(ldx=16), dict(ldw=16), dict(ldxs=0), dict(ldws=0), dict(ldy=9), dict(M=(1 << 30) + 1)):
        assert _product(**bad) == -2, bad
    for bad in (dict(ldx=40), dict(xq=A + 4), dict(ws=A + 8), dict(Y=A + 2), dict(Y=A + 1, out=2), dict(bias=A + 3)):
        assert _product(**bad) == -3, bad


def test_forward_refusals():
    for name in ("X", "q", "sc", "src", "wq", "ws", "Y"):
        assert _forward(**{name: None}) == -1, name
    assert _forward(type=3) == -11 and _forward(out=3) == -11
    for bad in (dict(M=-1), dict(ldx=39), dict(ldq=16), dict(ldw=16), dict(N=0), dict(ldy=9)):
        assert _forward(**bad) == -2, bad
    assert _forward(ldq=40) == -3 and _forward(ldw=40) == -3 and _forward(Y=A + 2) == -3 and _forward(bias=A + 2) == -3 and _forward(s=-1) == -5


# ---- the cache -------------------------------------------------------------------------------

POOL = dict(table=A, cols=5, ldt=5, fmt=0, keys=A, ks=A, values=A, vs=A, pages=9, P=16, H=2, D=64, kd=None, vd=None)


def _rows(call, over):
    p = dict(K=A, ldk=128, hdk=64, V=A, ldv=128, hdv=64, type=0, T=3, cu=A, starts=A, Bn=2, **POOL)
    p.update(over)
    return call(*p.values(), None)


def _attend(**over):
    p = dict(Q=A, type=0, ldq=512, hdq=64, Hq=8, T=3, cu=A, starts=A, Bn=2, most=70, **POOL, scale=0.125, window=0, Y=A, ldy=512, hdy=64, lse=A,
             ws=A, wb=1 << 26)
    p.update(over)
    return B.lib().ocs_cache_attention(*p.values(), None)


BAD_POOL = [(dict(fmt=2), -9), (dict(fmt=-1), -9), (dict(cols=0), -2), (dict(ldt=4), -2), (dict(pages=0), -2), (dict(P=8), -2), (dict(P=40), -2),
            (dict(H=0), -2), (dict(D=0), -2), (dict(D=48), -2), (dict(D=288), -2), (dict(T=-1), -2), (dict(Bn=-1), -2), (dict(type=3), -11),
            (dict(pages=1 << 31, P=1 << 20), -2)]
BAD_POOL += [({name: None}, -1) for name in ("table", "keys", "ks", "values", "vs", "cu", "starts")]
BAD_POOL += [({name: A + 2}, -3) for name in ("table", "cu", "starts", "kd", "vd")]
BAD_POOL += [({name: A + 8}, -3) for name in ("keys", "ks", "values", "vs")]


@pytest.mark.parametrize("over,code", BAD_POOL, ids=str)
def test_pool_refusals(over, code):
    for call in (B.lib().ocs_cache_write, B.lib().ocs_cache_read):
        assert _rows(call, over) == code
    if over.get("H") != 0:
        assert _attend(**over) == code


def test_rows_refusals():
    for call in (B.lib().ocs_cache_write, B.lib().ocs_cache_read):
        for over, code in ((dict(K=None), -1), (dict(V=None), -1), (dict(K=A + 2), -3), (dict(V=A + 1, type=1), -3), (dict(ldk=-1), -2),
                           (dict(hdv=-64), -2)):
            assert _rows(call, over) == code, over
    # rows that are written must not lie in each other
    for over in (dict(ldk=63), dict(hdv=63)):
        assert _rows(B.lib().ocs_cache_read, over) == -2


def test_positions_whose_numbers_would_pass_32_bits():
    # blocks beyond the last one seen are counted in 32 bits
    for most in (0x7FFF0001, 0x7FFFFFFF):
        assert _attend(most=most, P=1 << 24, cols=128, ldt=128) == -2
        assert B.ocs_cache_attention_workspace_bytes(3, 2, 2, 8, 64, most) == 0
    assert B.ocs_cache_attention_workspace_bytes(3, 2, 2, 8, 64, 0x7FFF0000) > 0


def test_attention_refusals():
    for over, code in ((dict(Q=None), -1), (dict(Y=None), -1), (dict(Hq=7), -2), (dict(Hq=1), -2), (dict(Hq=0), -2), (dict(most=-1), -2),
                       (dict(most=1 << 31), -2), (dict(window=-1), -2), (dict(ldy=63), -2), (dict(hdy=32), -2), (dict(Q=A + 2), -3),
                       (dict(Y=A + 2), -3), (dict(lse=A + 1), -3), (dict(scale=float("nan")), -13), (dict(scale=float("inf")), -13),
                       (dict(T=1 << 28, Hq=64, H=1), -2)):
        assert _attend(**over) == code, over
    need = B.ocs_cache_attention_workspace_bytes(3, 2, 2, 8, 64, 100000)
    assert need > 0
    assert _attend(most=100000, ws=None) == -7 and _attend(most=100000, wb=need - 1) == -7 and _attend(most=100000, ws=A + 16) == -3
    assert B.ocs_cache_attention_workspace_bytes(3, 2, 2, 7, 64, 100000) == 0 and B.ocs_cache_attention_workspace_bytes(0, 2, 2, 8, 64, 100) == 0
    assert B.lib().ocs_strerror(-13) not in (b"unknown error code", b"")


def test_workspace_stays_small():
    for T, Bn in ((1, 1), (1, 200), (200, 200), (35, 1), (5000, 7), (100000, 50)):
        for H, Hq in ((1, 1), (8, 32), (16, 256)):
            for most in (1, 1000, 100000, 1 << 30):
                for window in (0, 100, 5000):
                    assert B.ocs_cache_attention_workspace_bytes(T, Bn, H, Hq, 256, most, window) <= 1 << 26


def test_no_tokens_are_no_work():
    assert _quantize(M=0, X=None, q=None, sc=None) == 0 and _values(M=0, q=None, sc=None, Y=None) == 0
    assert _product(M=0, xq=None, xs=None, Y=None) == 0 and _forward(M=0, X=None, q=None, sc=None, Y=None) == 0
    assert _product(M=0, N=0) == -2 and _forward(M=0, wq=None) == -1
    for none in (dict(T=0), dict(Bn=0)):
        for call in (B.lib().ocs_cache_write, B.lib().ocs_cache_read):
            assert _rows(call, dict(K=None, V=None, cu=None, starts=None, table=None, **none)) == 0
        assert _attend(Q=None, Y=None, cu=None, **none) == 0
    assert _attend(T=0, fmt=5) == -9


class _NullStream:
    cuda_stream = 0


def test_binding_refuses_other_element_types_and_counts():
    x = torch.zeros((2, 32), dtype=torch.float64)
    u = torch.zeros((2, 16), dtype=torch.uint8)
    with pytest.raises(B.OcsError) as e:
        B.ocs_split_quantize_mx(x, 2, 32, 1, 32, None, None, 0, u, 16, u, 16, stream=_NullStream)
    assert e.value.code == -11
    with pytest.raises(B.OcsError) as e:                                     # keys and values of two types
        B.ocs_cache_write(torch.zeros((1, 1, 32)), 32, 32, torch.zeros((1, 1, 32), dtype=torch.bfloat16), 32, 32, 1, None, None, 1, None, 1, 1, 0,
                          None, None, None, None, 1, 16, 1, 32, None, None, stream=_NullStream)
    assert e.value.code == -11
    with pytest.raises(TypeError):
        B.ocs_cache_read(1, 2, 3, stream=_NullStream)
