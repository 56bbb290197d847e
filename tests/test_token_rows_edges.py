"""Layers with a grid per row and the scoring of tokens where they have gone wrong: a section for each."""
import numpy as np
import pytest
import torch

from paper_1901_09504_amd import binding as B
from tests import gpu_util as G

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def _gpu():
    G.require_gpu()


# ---- NaN ---------------------------------------------------------------------------------------

def _nan_rows(V, dtype):
    """Rows of logits with NaN in them: at token 0 alone, everywhere, at 0 and the end, in the second half, at 0 beside +inf and -inf."""
    x = torch.randn((5, V), generator=torch.Generator().manual_seed(V)).to(dtype)
    x[0, 0] = float("nan")
    x[1] = float("nan")
    x[2, 0] = x[2, V - 1] = float("nan")
    x[3, V // 2:] = -float("nan")
    x[4] = float("-inf")
    x[4, V // 2] = float("inf")
    x[4, 0] = float("nan")
    return x


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V,k", [(1, 1), (2, 1), (5, 5), (32, 32), (100, 7), (3000, 20), (33001, 32), (66001, 5), (131075, 20)])
def test_nan_at_any_token_comes_first(dtype, V, k):
    """NaN ahead of everything, the lowest index first, whatever index that is; every id is one of the row's."""
    x = _nan_rows(V, dtype)
    ids, top = torch.full((5, k), -7, dtype=torch.int32, device="cuda"), torch.zeros((5, k), device="cuda")
    lp, ent = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    need = B.ocs_token_logprobs_workspace_bytes(5, V, k)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    B.ocs_token_logprobs(x.cuda(), 5, V, V, torch.zeros(5, dtype=torch.int32, device="cuda"), k, lp, ent, ids, top, ws)
    ids = G.host(ids)
    v = x.double().numpy()
    for m in range(5):
        nan = np.isnan(v[m])
        order = np.lexsort((np.arange(V), -np.where(nan, 0.0, v[m]), ~nan))[:k]
        assert np.array_equal(ids[m], order), (m, ids[m], order)
    assert ids.min() >= 0 and ids.max() < V
    assert np.isnan(G.host(top)).all() and np.isnan(G.host(lp)).all() and np.isnan(G.host(ent)).all()
