"""Softmax attention where rows share a register, a reciprocal or a tile: queries of padding and queries that hold NaN in a step."""
import math

import pytest
import torch

from test_gpu_softmax import BF, DEV, F32, _compare, _inputs, _run, _slopes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("Hq,Hk,nq", [(1, 1, 12), (2, 2, 16), (4, 2, 5), (3, 1, 3), (6, 2, 5), (3, 1, 6)])
@pytest.mark.parametrize("cap", [0.0, 10.0])
def test_padding_among_the_queries_of_a_step_may_hold_anything(dtype, d, Hq, Hk, nq, cap):
    """Up to 16 rows a key head (18: the other kernels): a row of padding shares the products of its tile with rows that are not."""
    nk = 300
    Q, K, V, dO = _inputs(2, Hq, Hk, nq, nk, d, dtype)
    g = torch.Generator().manual_seed(nq)
    dk = torch.randint(0, 2, (2, nk), generator=g).int()
    dq = torch.randint(0, 2, (2, nq), generator=g).int()
    dq[0, 1::2] = -1                                           # every other query of one sequence, the end of the other
    dq[1, nq // 2:] = -1
    kw = dict(doc_q=dq, doc_k=dk, cap=cap, slopes=_slopes(Hq))
    got = _compare(Q, K, V, dO, **kw)
    pad = (dq < 0).to(DEV)
    for bad in (math.nan, math.inf):
        Q.transpose(1, 2)[pad] = bad
        dO.transpose(1, 2)[pad] = bad
        again = _run(Q, K, V, dO, **kw)
        for k in got:
            assert torch.equal(got[k], again[k]), (k, bad)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Hq,nq", [(12, 1), (5, 3), (16, 1), (1, 13)])
@pytest.mark.parametrize("cap", [0.0, 10.0])
def test_a_query_that_holds_nan_spoils_its_own_row_only(dtype, Hq, nq, cap):
    Q, K, V, _ = _inputs(2, Hq, 1, nq, 600, 64, dtype)
    ref = _run(Q, K, V, cap=cap)
    h, i = 2 % Hq, nq // 3
    Q[0, h, i] = math.nan
    got = _run(Q, K, V, cap=cap)
    assert torch.isnan(got["O"][0, h, i]).all() and torch.isnan(got["lse"][0, h, i])
    for k in ("O", "lse"):
        got[k][0, h, i] = ref[k][0, h, i]
        assert torch.equal(got[k], ref[k]), k
