"""Softmax attention where rows share a register, a reciprocal or a tile: queries of padding and queries that hold NaN in a step;
caps far above and far below the scores; long rows of 128 channels, the kernel with two query tiles a CTA."""
import math

import pytest
import torch

from attention_reference import attention, check
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


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d,nq,nk", [(64, 1, 700), (128, 12, 700), (32, 90, 90), (64, 200, 700), (128, 200, 700)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [1e4, 1e6, 1e9, 3e38])
def test_a_large_cap_tends_to_no_cap(dtype, d, nq, nk, bias, cap):
    """The tolerance is that of uncapped scores: s (1 - (s / cap)^2 / 3) differs from s by 3e-6 of it where |s| < 30 and the cap is 1e4, in
    the reference as in the kernel; the factor of the cap costs a kernel a few half steps of the score, not of the cap.  (1 - tanh^2 is off by a
    half step or two of 32 bits, beside the four that a gradient's tolerance has.)"""
    Q, K, V, dO = _inputs(2, 2, 1, nq, nk, d, dtype, sigma=4.0)
    kw = dict(causal=True, slopes=_slopes(2) if bias else None)
    got = _run(Q, K, V, dO, cap=cap, **kw)
    val, _ = attention(Q, K, V, dO, dtype=dtype, cap=cap, **kw)
    _, tol = attention(Q, K, V, dO, dtype=dtype, **kw)
    print(check(got, val, tol))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d,nq,nk", [(64, 3, 700), (64, 200, 700), (128, 200, 700)])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [100.0, 128.0, 129.0, 1000.0])
def test_scores_on_both_sides_of_the_cap(dtype, d, nq, nk, bias, cap):
    Q, K, V, dO = _inputs(1, 2, 2, nq, nk, d, dtype, sigma=0.7 * cap)
    Q[:, :, ::3] *= 0.01
    _compare(Q, K, V, dO, causal=True, cap=cap, slopes=_slopes(2) if bias else None)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 150])
@pytest.mark.parametrize("cap", [1e-30, 1e-39])
def test_a_tiny_cap_leaves_equal_weights(dtype, nq, cap):
    Q, K, V, dO = _inputs(1, 2, 2, nq, 300, 64, dtype)
    Q[:, 0, 0] = 0.0                                           # products of zero: tanh(0) whatever the cap
    got = _run(Q, K, V, dO, cap=cap)
    val, tol = attention(Q, K, V, dtype=dtype, cap=cap)
    check({k: got[k] for k in ("O", "lse")}, val, tol)
    for k in ("dQ", "dK", "dV"):
        assert torch.isfinite(got[k]).all(), k


def _underflow(Q, K, V, dO):
    """What A and ds below 2^-126, the smallest normal number of 32 bits (and of bf16), may take from the gradients: far from its query a key with a
    distance bias has nothing else.  Either may come out as zero.  A pair of dV then misses 2^-126 |dO|; one of dK or dQ misses scale
    2^-126 (1 + |dP - delta|) of its query or key, and |dP - delta| <= 2 |dO|_2 |V|_2 since O is a mean of the V (the cap's factor is at most 1)."""
    q, k, v, g = (t.cpu().double().abs() for t in (Q, K, V, dO))
    reach = 2.0 ** -126 / math.sqrt(q.shape[-1]) * (1 + 2 * float(g.norm(dim=-1).max() * v.norm(dim=-1).max()))
    group = q.shape[1] // k.shape[1]
    per_key_head = lambda t: t.sum(2, keepdim=True).unflatten(1, (-1, group)).sum(2)
    per_query_head = lambda t: t.sum(2, keepdim=True).repeat_interleave(group, 1)
    return dict(dQ=reach * per_query_head(k), dK=reach * per_key_head(q), dV=2.0 ** -126 * per_key_head(g))


WIDE = [(1, 2, 513, 513), (2, 2, 129, 1030), (1, 2, 300, 2100), (1, 1, 700, 900)]


@pytest.mark.parametrize("B,H,nq,nk", WIDE)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("bias", [False, True])
def test_long_rows_of_wide_heads(B, H, nq, nk, causal, cap, bias):
    """128 channels, more than 128 queries and 512 keys: two query tiles a CTA, and beyond 1024 keys parts that are joined."""
    kw = dict(causal=causal, cap=cap, slopes=_slopes(2 * H) if bias else None)
    if causal and bias:
        kw["prefix"] = torch.full((B,), nk // 3, dtype=torch.int32)
    x = _inputs(B, 2 * H, H, nq, nk, 128, BF, sigma=2.0)
    got = _run(*x, **kw)
    val, tol = attention(*x, dtype=BF, **kw)
    for k, t in _underflow(*x).items():
        tol[k] += t
    print(check(got, val, tol))


@pytest.mark.parametrize("n", [700, 1333])
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_documents_in_long_rows_of_wide_heads(n, cap):
    Q, K, V, dO = _inputs(2, 2, 1, n, n, 128, BF, packed=True)
    at = torch.arange(n)
    doc = torch.stack([at // 290, torch.where(at < n - 200, at // 517, -1)]).int()
    kw = dict(doc_q=doc, doc_k=doc, causal=True, cap=cap)
    got = _compare(Q, K, V, dO, **kw)
    pad = (doc < 0).to(DEV)
    for t in (Q, K, V, dO):
        t.transpose(1, 2)[pad] = math.nan
    again = _run(Q, K, V, dO, **kw)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("nq,nk", [(150, 600), (400, 1500)])
@pytest.mark.parametrize("causal", [False, True])
def test_filled_length_in_long_rows_of_wide_heads(nq, nk, causal):
    Q, K, V, dO = _inputs(5, 2, 2, nq, nk, 128, BF)
    kv = torch.tensor([nk, 0, 1, nk - 129, 520], dtype=torch.int32)
    kw = dict(kv_len=kv, causal=causal, cap=10.0, slopes=_slopes(2))
    got = _compare(Q, K, V, dO, **kw)
    for b, n in enumerate(kv.tolist()):
        K[b, :, n:] = math.nan
        V[b, :, n:] = math.inf
    again = _run(Q, K, V, dO, **kw)
    for k in got:
        assert torch.equal(got[k], again[k]), k


def test_long_rows_of_many_wide_heads():
    """Query tiles fill the GPU: two tiles a CTA, keys not split."""
    Q, K, V, _ = _inputs(4, 40, 10, 300, 1100, 128, BF)
    _compare(Q, K, V, causal=True)


def _rounded(t):
    return t.to(BF).double()


def _without_correction(Q, K, V, dO, cap):
    """Errors of dQ and dK, relative to their norms, if delta = dO . O is taken from the stored O as it is (64 bits but for the roundings)."""
    q, k, v, g = (t.cpu().double() for t in (Q, K, V, dO))
    scale = 1 / math.sqrt(q.shape[-1])
    t = torch.tanh(q @ k.transpose(-1, -2) * scale / cap) if cap else None
    s, bend = (cap * t, 1 - t * t) if cap else (q @ k.transpose(-1, -2) * scale, 1.0)
    A = torch.softmax(s, -1)
    dP, out = g @ v.transpose(-1, -2), A @ v
    back = lambda O, store: [store(x) for ds in (store(A * (dP - (g * O).sum(-1, keepdim=True)) * bend),) for x in (ds @ k * scale, ds.transpose(-1, -2) @ q * scale)]
    return [float((x - y).norm() / y.norm()) for x, y in zip(back(_rounded(out), _rounded), back(out, lambda x: x))]


@pytest.mark.parametrize("n,sigma,cap", [(16, 3.0, 0.0), (16, 6.0, 0.0), (16, 3.0, 8.0), (197, 6.0, 0.0)])
def test_gradients_of_peaked_rows_are_as_good_as_their_roundings(n, sigma, cap):
    """A rounding to bf16 is uniform within half a step: 2^-8 / sqrt(3) of the value where the mantissa is 1, half of it near 2, 1.7e-3 in the
    mean square.  dQ and dK see two of them that are independent, ds and their own: 2.35e-3 of the norm, and a tenth more for the
    scatter over 32 heads.  The rounding of the stored O, through delta, would come on top of it."""
    bound = 1.1 * 2.35e-3
    Q, K, V, dO = _inputs(8, 4, 4, n, n, 64, BF, sigma=sigma)
    assert min(_without_correction(Q, K, V, dO, cap)) > 1.05 * bound
    got = _run(Q, K, V, dO, cap=cap)
    val, _ = attention(Q, K, V, dO, dtype=BF, cap=cap)
    for k in ("dQ", "dK"):
        err = float((got[k].cpu().double() - val[k]).norm() / val[k].norm())
        print(k, err)
        assert err < bound, (k, err)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [2, 140])
def test_overlapping_rows_and_a_bias_that_grows_with_distance(dtype, nq):
    """Windows over one buffer, a row eight elements behind the last; negative slopes, so that the farthest key weighs most and A of the
    nearest lies below 2^-126."""
    nk, d = 300, 64
    g = torch.Generator().manual_seed(4)
    windows = lambda n: torch.randn(2, 2, n * 8 + d, generator=g).to(dtype).to(DEV).as_strided((2, 2, n, d), (2 * (n * 8 + d), n * 8 + d, 8, 1))
    Q, K, V, dO = windows(nq), windows(nk), windows(nk), windows(nq)
    kw = dict(causal=True, slopes=torch.tensor([-0.3, -0.01]))
    got = _run(Q, K, V, dO, **kw)
    val, tol = attention(Q, K, V, dO, dtype=dtype, **kw)
    for k, t in _underflow(Q, K, V, dO).items():
        tol[k] += t
    print(check(got, val, tol))
