"""The quantized cache on the GPU, further: how fine the weights of the values are, and cases at the edges of what a call may be given."""
import pytest
import torch

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
