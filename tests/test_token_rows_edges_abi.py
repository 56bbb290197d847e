"""What the calls with a grid per row and token scoring accept and refuse, on the host (no GPU), where they have gone wrong."""
import pytest
import torch

from paper_1901_09504_amd import binding as B

A = 1 << 20  # a fake, suitably aligned device address: validation never dereferences it


# ---- layers wider than the channel selection serves ----------------------------------------------

def _quantize(C, s, g=1, M=0, src=A):
    ld = (C + s) * g
    return B.lib().ocs_split_quantize_rows(A, 0, M, C, g, C * g, src, None, s, 8, 1.0, A, -(-ld // 16) * 16, A, None)


def _forward(C, s, g=1, src=A):
    ld = -(-(C + s) * g // 128) * 128
    return B.lib().ocs_forward_rows(A, 0, 0, C, g, C * g, src, s, 8, 1.0, A, ld, A, A, ld, 10, 8, A, None, A, 0, 10, None)


@pytest.mark.parametrize("C", [8000, 8001, 8192, 11008, 14336, 65536, 100000])
def test_without_splits_the_selections_bound_does_not_hold(C):
    assert _quantize(C, 0) == 0 and _quantize(C, 0, src=None) == 0 and _quantize(C, 0, g=9) == 0
    assert _forward(C, 0) == 0 and _forward(C, 0, src=None) == 0


def test_with_splits_it_does():
    assert _quantize(7999, 1) == 0 and _quantize(8000, 1) == -5 and _quantize(8192, 410) == -5 and _forward(8192, 1) == -5
    assert _quantize(8192, -1) == -5


def test_other_bounds_hold_without_splits():
    assert _quantize(1 << 30, 0) == 0 and _quantize((1 << 30) + 1, 0) == -2 and _quantize(1 << 20, 0, g=1 << 11) == -2
    assert _forward(140000, 0) == -6                         # 140000 x 127 x 127 does not fit an accumulator


# ---- tensors of the host -------------------------------------------------------------------------

def test_tensors_of_the_host_are_refused_before_any_call(monkeypatch):
    """Their addresses mean nothing to the GPU: no call may be made with them."""
    from paper_1901_09504_amd import layer

    called = []
    for n in ("ocs_select_channels", "ocs_split_quantize_rows", "ocs_forward_rows", "ocs_token_logprobs", "alloc_workspace"):
        monkeypatch.setattr(layer.B, n, lambda *a, **k: called.append(a))
    head = object.__new__(layer.TokenLayer)
    head.N, head.K, head.C, head.g, head.s = 4, 8, 8, 1, 0
    with pytest.raises(AssertionError):
        head.prepare_weights(torch.zeros(4, 8))
    with pytest.raises(AssertionError):
        head.forward(torch.zeros(2, 8))
    with pytest.raises(AssertionError):
        layer.token_logprobs(torch.zeros(2, 8))
    with pytest.raises(AssertionError):
        layer.token_logprobs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), 3)
    assert not called
