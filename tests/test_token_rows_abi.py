"""Refusals of the calls with a grid per row and of token scoring, on the host (no GPU): every argument error is found
before any device work, and no tokens are no work."""
import pytest
import torch

from paper_1901_09504_amd import binding as B

A = 1 << 20  # a fake, suitably aligned device address: validation never dereferences it


def _quantize(X=A, type=0, M=4, C=40, g=1, ldx=40, src=A, depth=None, s=3, bits=8, clip=1.0, Xq=A, ldq=48, step=A):
    return B.lib().ocs_split_quantize_rows(X, type, M, C, g, ldx, src, depth, s, bits, clip, Xq, ldq, step, None)


def _product(Xq=A, ldx=384, Wq=A, ldw=384, M=4, N=10, K=330, bx=8, bw=8, sx=A, sw=A, bias=None, Y=A, type=0, ldy=10):
    return B.lib().ocs_qgemm_rows(Xq, ldx, Wq, ldw, M, N, K, bx, bw, sx, sw, bias, Y, type, ldy, None)


def _forward(X=A, type=0, M=4, C=40, g=1, ldx=40, src=A, s=3, bits=8, clip=1.0, Xq=A, ldq=48, step=A, Wq=A, ldw=48, N=10, bw=8,
             sw=A, bias=None, Y=A, out=0, ldy=10):
    return B.lib().ocs_forward_rows(X, type, M, C, g, ldx, src, s, bits, clip, Xq, ldq, step, Wq, ldw, N, bw, sw, bias, Y, out, ldy,
                                    None)


def _score(x=A, type=0, M=4, V=100, ld=100, tokens=A, k=5, lp=A, ent=A, ids=A, top=A, ws=None, wb=0):
    return B.lib().ocs_token_logprobs(x, type, M, V, ld, tokens, k, lp, ent, ids, top, ws, wb, None)


def test_quantize_rows_refusals():
    for name in ("X", "Xq", "step", "src"):
        assert _quantize(**{name: None}) == -1, name
    assert _quantize(type=3) == -11 and _quantize(type=-1) == -11
    for bad in (dict(M=-1), dict(C=0), dict(g=0), dict(ldx=39), dict(ldq=32), dict(M=(1 << 31) + 1)):
        assert _quantize(**bad) == -2, bad
    assert _quantize(C=1, s=2, g=1 << 29, ldx=1 << 29, ldq=1 << 31) == -2            # (C + s) * g beyond 2^30
    assert _quantize(ldq=56) == -3 and _quantize(Xq=A + 8) == -3 and _quantize(X=A + 2) == -3 and _quantize(step=A + 2) == -3
    assert _quantize(X=A + 1, type=1) == -3
    assert _quantize(bits=1) == -4 and _quantize(bits=9) == -4
    assert _quantize(s=-1) == -5 and _quantize(C=7000, ldx=7000, s=1001, ldq=8016) == -5
    for clip in (0.0, -1.0, float("nan"), float("inf")):
        assert _quantize(clip=clip) == -10


def test_product_rows_refusals():
    for name in ("Xq", "Wq", "sx", "sw", "Y"):
        assert _product(**{name: None}) == -1, name
    assert _product(type=7) == -11
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(ldx=320), dict(ldw=320), dict(ldy=9), dict(M=(1 << 30) + 1)):
        assert _product(**bad) == -2, bad
    for bad in (dict(ldx=400), dict(Xq=A + 4), dict(Wq=A + 8), dict(Y=A + 2), dict(Y=A + 1, type=2), dict(sx=A + 1), dict(sw=A + 2),
                dict(bias=A + 3)):
        assert _product(**bad) == -3, bad
    assert _product(bx=1) == -4 and _product(bw=9) == -4
    assert _product(K=140000, ldx=140032, ldw=140032) == -6


def test_forward_rows_refusals():
    for name in ("X", "Xq", "step", "src", "Wq", "sw", "Y"):
        assert _forward(**{name: None}) == -1, name
    assert _forward(type=3) == -11 and _forward(out=3) == -11
    for bad in (dict(M=-1), dict(ldx=39), dict(ldq=32), dict(ldw=32), dict(N=0), dict(ldy=9)):
        assert _forward(**bad) == -2, bad
    assert _forward(ldq=56) == -3 and _forward(ldw=56) == -3 and _forward(Y=A + 2) == -3 and _forward(bias=A + 2) == -3
    assert _forward(bits=1) == -4 and _forward(bw=1) == -4 and _forward(s=-1) == -5 and _forward(clip=0.0) == -10


def test_token_logprobs_refusals():
    assert _score(x=None) == -1
    assert _score(tokens=None) == -1 and _score(lp=None) == -1                       # one without the other
    assert _score(ids=None) == -1 and _score(top=None) == -1
    assert _score(tokens=None, lp=None, ent=None, k=0) == -1                         # nothing is asked for
    assert _score(type=5) == -11
    for bad in (dict(M=-1), dict(V=0), dict(ld=99), dict(V=(1 << 30) + 1, ld=1 << 31)):
        assert _score(**bad) == -2, bad
    assert _score(k=-1) == -12 and _score(k=33) == -12 and _score(V=4, k=5) == -12
    for bad in (dict(x=A + 2), dict(x=A + 1, type=1), dict(tokens=A + 2), dict(lp=A + 1), dict(ent=A + 2), dict(ids=A + 2),
                dict(top=A + 2)):
        assert _score(**bad) == -3, bad
    # a long row for one token is shared by several workgroups, which meet in the workspace
    need = B.ocs_token_logprobs_workspace_bytes(1, 1 << 20, 5)
    assert need > 0
    assert _score(M=1, V=1 << 20, ld=1 << 20) == -7 and _score(M=1, V=1 << 20, ld=1 << 20, ws=A, wb=need - 1) == -7
    assert _score(M=1, V=1 << 20, ld=1 << 20, ws=A + 16, wb=need) == -3
    for M, V, k in ((0, 100, 5), (4, 0, 5), (4, 100, 33), (4, 100, -1), (-1, 100, 5)):
        assert B.ocs_token_logprobs_workspace_bytes(M, V, k) == 0


def test_workspace_stays_small():
    for M in (1, 2, 7, 20, 63, 64, 100, 255, 256, 700, 4096):
        for V in (1, 100, 33001, 131072, 1 << 20, 1 << 30):
            for k in (0, 1, min(V, 32)):
                assert B.ocs_token_logprobs_workspace_bytes(M, V, k) <= 1 << 20


def test_no_tokens_are_no_work():
    assert _quantize(M=0, X=None, Xq=None, step=None) == 0
    assert _product(M=0, Xq=None, sx=None, Y=None) == 0
    assert _forward(M=0, X=None, Xq=None, step=None, Y=None) == 0
    assert _score(M=0, x=None, tokens=None, lp=None, ent=None, ids=None, top=None) == 0
    # what is not per token is still checked
    assert _quantize(M=0, bits=9) == -4 and _product(M=0, N=0) == -2 and _forward(M=0, Wq=None) == -1 and _score(M=0, k=33) == -12


def test_error_texts():
    for code in (-11, -12):
        assert B.lib().ocs_strerror(code) not in (b"unknown error code", b"")


@pytest.mark.parametrize("dtype", [torch.float64, torch.int32])
def test_binding_refuses_other_element_types(dtype):
    x = torch.zeros((2, 8), dtype=dtype)
    f = torch.zeros(8)
    with pytest.raises(B.OcsError) as e:
        B.ocs_token_logprobs(x, 2, 8, 8, None, 0, None, f, None, None, stream=type("S", (), {"cuda_stream": 0}))
    assert e.value.code == -11


class _NullStream:
    cuda_stream = 0


def test_binding_refuses_arguments_of_other_kinds():
    """Python errors, not codes and not crashes; what fits neither 32 nor 64 bits is no smaller number."""
    x, f, i = torch.zeros((0, 8)), torch.zeros(0), torch.zeros(0, dtype=torch.int32)

    def score(x=x, M=0, V=8, ld=8, tokens=i, k=2, lp=f, ws=None, stream=_NullStream):
        B.ocs_token_logprobs(x, M, V, ld, tokens, k, lp, f, i, f, ws, stream)

    score()
    score(ws=torch.zeros(4, dtype=torch.uint8))
    for bad in (dict(M="0"), dict(V=None), dict(x=3), dict(tokens="x"), dict(k=1.5), dict(ws=7), dict(stream=3)):
        with pytest.raises((TypeError, AttributeError)):
            score(**bad)
    for bad in (dict(k=1 << 31), dict(k=-(1 << 31) - 1), dict(V=1 << 63), dict(M=1 << 70)):
        with pytest.raises(OverflowError):
            score(**bad)
    with pytest.raises(B.OcsError) as e:
        score(x=None)                                        # nothing has no element type
    assert e.value.code == -11


def test_binding_passes_every_argument_to_its_place():
    """One wrong argument at a time, and no tokens: the code tells which one arrived where."""
    x, q, f = torch.zeros((0, 40)), torch.zeros((0, 48), dtype=torch.int8), torch.zeros(0)
    src, w, sw, y = torch.zeros(43, dtype=torch.int32), torch.zeros((10, 48), dtype=torch.int8), torch.zeros(10), torch.zeros((0, 10))
    half = torch.zeros((0, 10), dtype=torch.float64)

    def quantize(x=x, M=0, C=40, g=1, ldx=40, src=src, s=3, bits=8, clip=1.0, ldq=48):
        B.ocs_split_quantize_rows(x, M, C, g, ldx, src, None, s, bits, clip, q, ldq, f, _NullStream)

    def product(ldx=48, w=w, ldw=48, M=0, N=10, K=43, bx=8, bw=8, sw=sw, bias=None, y=y, ldy=10):
        B.ocs_qgemm_rows(q, ldx, w, ldw, M, N, K, bx, bw, f, sw, bias, y, ldy, _NullStream)

    def forward(x=x, M=0, C=40, g=1, ldx=40, src=src, s=3, bits=8, clip=1.0, ldq=48, w=w, ldw=48, N=10, bw=8, sw=sw, bias=False, y=y, ldy=10):
        B.ocs_forward_rows(x, M, C, g, ldx, src, s, bits, clip, q, ldq, f, w, ldw, N, bw, sw, bias, y, ldy, _NullStream)

    quantize(), product(), forward(), forward(bias=sw), product(bias=sw)
    grids = [(dict(x=half), -11), (dict(C=0), -2), (dict(g=0), -2), (dict(ldx=39), -2), (dict(src=None), -1),
             (dict(s=-1), -5), (dict(bits=9), -4), (dict(clip=0.0), -10), (dict(ldq=32), -2), (dict(ldq=56), -3)]
    layer = [(dict(w=None), -1), (dict(ldw=32), -2), (dict(N=0), -2), (dict(bw=1), -4), (dict(sw=None), -1), (dict(y=half), -11),
             (dict(ldy=9), -2), (dict(ldw=56), -3)]
    own = [(dict(ldx=32), -2), (dict(ldx=56), -3), (dict(K=0), -2), (dict(K=49), -2), (dict(bx=1), -4)]
    for call, cases in ((quantize, grids), (forward, grids + layer), (product, own + layer)):
        for bad, code in cases:
            with pytest.raises(B.OcsError) as e:
                call(**bad)
            assert e.value.code == code, (call.__name__, bad, e.value.code)
