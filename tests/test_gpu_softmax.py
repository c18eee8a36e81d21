"""Softmax attention with capped, biased and masked scores against its definition in 64 bits, element by element."""
import math

import pytest
import torch

import paper_2604_20368_b200 as ln
from attention_reference import attention, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _inputs(B, Hq, Hk, nq, nk, d, dtype, seed=0, sigma=1.0, packed=False):
    g = torch.Generator().manual_seed(seed + 1000 * nq + nk)
    normal = lambda *s: torch.randn(*s, generator=g)
    if packed:
        x = normal(B, nq, Hq + 2 * Hk, d)
        x[:, :, :Hq] *= sigma
        Q, K, V = (t.transpose(1, 2) for t in x.to(dtype).to(DEV).split([Hq, Hk, Hk], 2))
    else:
        Q, K, V = ((normal(B, h, n, d) * s).to(dtype).to(DEV) for h, n, s in ((Hq, nq, sigma), (Hk, nk, 1.0), (Hk, nk, 1.0)))
    return Q, K, V, normal(B, Hq, nq, d).to(dtype).to(DEV)


def _run(Q, K, V, dO=None, **kw):
    kw = {k: (v.to(DEV) if torch.is_tensor(v) else v) for k, v in kw.items()}
    sp = ln.SoftmaxAttention(**kw)
    status = torch.full((Q.shape[0] * Q.shape[1],), -1, dtype=torch.int32, device=DEV)
    O, lse = ln.softmax_attention_fwd(sp, Q, K, V, dev_status=status)
    got = dict(O=O, lse=lse)
    assert int(status.abs().max()) == 0
    if dO is not None:
        status.fill_(-1)
        got["dQ"], got["dK"], got["dV"] = ln.softmax_attention_bwd(sp, Q, K, V, O, lse, dO, dev_status=status)
        assert int(status.abs().max()) == 0
    return got


def _compare(Q, K, V, dO=None, **kw):
    got = _run(Q, K, V, dO, **kw)
    val, tol = attention(Q, K, V, dO, dtype=Q.dtype, **kw)
    print({k: f"{v:.2f}" for k, v in check(got, val, tol).items()})
    return got


def _slopes(H):
    return torch.exp2(-8.0 * torch.arange(1, H + 1) / H)


def _docs(B, n, seed, pad=True, kinds=4):
    g = torch.Generator().manual_seed(seed)
    cuts = torch.randint(0, n + 1, (B, kinds), generator=g).sort(1).values
    d = (torch.arange(n)[None, :, None] >= cuts[:, None, :]).sum(-1).int()
    return torch.where(d == kinds, -1, d).int() if pad else d


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("nq,nk", [(1, 1), (197, 197), (64, 64), (65, 129), (128, 257), (300, 77)])
def test_lengths_and_head_dims(dtype, d, nq, nk):
    _compare(*_inputs(2, 2, 2, nq, nk, d, dtype))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq,nk", [(1, 1), (197, 197), (256, 256), (100, 333), (333, 100), (2, 300), (513, 513)])
@pytest.mark.parametrize("extra", ["none", "prefix", "cap", "bias", "all"])
def test_causal(dtype, nq, nk, extra):
    kw = dict(causal=True)
    if extra in ("prefix", "all"):
        kw["prefix"] = torch.tensor([min(nk, 70), 0, nk + 5], dtype=torch.int32)
    if extra in ("cap", "all"):
        kw["cap"] = 5.0
    if extra in ("bias", "all"):
        kw["slopes"] = _slopes(4)
    _compare(*_inputs(3, 4, 2, nq, nk, 64, dtype, sigma=2.0), **kw)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (8.0, True)])
def test_documents_with_padding(dtype, d, causal, cap, bias):
    n = 421
    Q, K, V, dO = _inputs(3, 2, 1, n, n, d, dtype, packed=True)
    doc = _docs(3, n, d)
    doc[2] = -1                                                # nothing at all in one batch element
    kw = dict(doc_q=doc, doc_k=doc, causal=causal, cap=cap, slopes=_slopes(2) if bias else None)
    got = _compare(Q, K, V, dO, **kw)
    empty = (doc < 0)[:, None].expand(3, 2, n).to(DEV)
    assert (got["O"][empty] == 0).all() and (got["lse"][empty] == -math.inf).all() and (got["dQ"][empty] == 0).all()
    # the rows of padding may hold anything
    pad = (doc < 0).to(DEV)
    for t in (Q, K, V, dO):
        t.transpose(1, 2)[pad] = float("nan")
    dO.transpose(1, 2)[pad] = float("inf")
    again = _run(Q, K, V, dO, **kw)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype", [F32, BF])
def test_documents_in_any_order_and_other_ids_for_keys(dtype):
    nq, nk = 150, 290
    g = torch.Generator().manual_seed(5)
    dq = torch.randint(-1, 3, (2, nq), generator=g).int()
    dk = torch.randint(-1, 5, (2, nk), generator=g).int()
    dk[1][dk[1] == 2] = 2147483647                             # document 2 has no key in the second batch element
    _compare(*_inputs(2, 3, 3, nq, nk, 64, dtype), doc_q=dq, doc_k=dk)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 3, 90, 200])
@pytest.mark.parametrize("causal", [False, True])
def test_filled_length_of_a_cache(dtype, nq, causal):
    nk = 260
    Q, K, V, dO = _inputs(6, 4, 2, nq, nk, 64, dtype)
    kv = torch.tensor([nk, 0, 1, 130, -3, nk + 7], dtype=torch.int32)
    kw = dict(kv_len=kv, causal=causal, cap=10.0, slopes=_slopes(4))
    got = _compare(Q, K, V, dO, **kw)
    for b, n in enumerate(kv.clamp(0, nk).tolist()):
        K[b, :, n:] = float("nan")
        V[b, :, n:] = float("inf")
        assert (got["dK"][b, :, n:] == 0).all() and (got["dV"][b, :, n:] == 0).all()
    again = _run(Q, K, V, dO, **kw)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Hq,Hk", [(8, 1), (6, 3), (5, 5)])
@pytest.mark.parametrize("nq", [1, 2, 140])
def test_shared_heads(dtype, Hq, Hk, nq):
    _compare(*_inputs(2, Hq, Hk, nq, 140, 128, dtype), causal=True, slopes=_slopes(Hq))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("Hq,Hk,nq", [(1, 1, 1), (4, 1, 1), (8, 4, 2), (16, 1, 1), (2, 2, 16), (3, 1, 5), (6, 2, 6)])
def test_steps_over_a_long_cache(dtype, d, Hq, Hk, nq):
    """Few queries, keys split over many CTAs: with up to 16 rows a key head the step kernels, with 18 the others."""
    nk = 5003
    Q, K, V, _ = _inputs(3, Hq, Hk, nq, nk, d, dtype, sigma=3.0)
    kv = torch.tensor([nk, 517, 4999], dtype=torch.int32)
    _compare(Q, K, V)
    _compare(Q, K, V, causal=True, kv_len=kv, cap=15.0, slopes=_slopes(Hq), prefix=torch.tensor([0, 516, 5003], dtype=torch.int32))
    dk = _docs(3, nk, 1)
    _compare(Q, K, V, doc_q=dk[:, 2000:2000 + nq].contiguous(), doc_k=dk, kv_len=kv)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 3, 30])
@pytest.mark.parametrize("cap", [0.0, 10.0])
def test_padding_between_the_keys_of_a_step_may_hold_anything(dtype, nq, cap):
    nk = 600
    g = torch.Generator().manual_seed(7)
    Q, K, V, dO = _inputs(2, 4, 2, nq, nk, 64, dtype)
    dk = torch.randint(-1, 2, (2, nk), generator=g).int()
    dq = torch.randint(0, 2, (2, nq), generator=g).int()
    kw = dict(doc_q=dq, doc_k=dk, cap=cap, slopes=_slopes(4))
    got = _compare(Q, K, V, dO, **kw)
    pad = (dk < 0).to(DEV)
    K.transpose(1, 2)[pad] = float("nan")
    V.transpose(1, 2)[pad] = float("inf")
    again = _run(Q, K, V, dO, **kw)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype", [F32, BF])
def test_long_row_and_large_scores(dtype):
    # scores of +-100 and more: the running maximum moves, the exponentials span the whole range
    Q, K, V, dO = _inputs(1, 2, 2, 130, 2100, 64, dtype, sigma=30.0)
    _compare(Q, K, V, dO)
    _compare(Q, K, V, dO, cap=30.0, causal=True)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 70])
def test_strides(dtype, nq):
    """Slices of a projection, broadcast batch, outputs inside larger buffers whose other elements stay as they are."""
    B, H, nk, d = 3, 2, 140, 64
    Q, K, V, dO = _inputs(B, H, H, nq, nk, d, dtype)
    wide = torch.randn(B, nk, 3, H, d + 32, device=DEV).to(dtype)
    K, V = wide[:, :, 1, :, 8:8 + d].transpose(1, 2), wide[:1, :, 2, :, 16:16 + d].transpose(1, 2).expand(B, H, nk, d)
    hold = {k: torch.full((B, n + 2, H + 1, d + 16), 7.0, dtype=dtype, device=DEV) for k, n in (("O", nq), ("dQ", nq), ("dK", nk), ("dV", nk))}
    out = {k: t[:, 1:-1, :H, 8:8 + d].transpose(1, 2) for k, t in hold.items()}
    sp = ln.SoftmaxAttention(causal=True)
    _, lse = ln.softmax_attention_fwd(sp, Q, K, V, O=out["O"])
    ln.softmax_attention_bwd(sp, Q, K, V, out["O"], lse, dO, dQ=out["dQ"], dK=out["dK"], dV=out["dV"])
    val, tol = attention(Q, K, V, dO, dtype=dtype, causal=True)
    check(dict(out, lse=lse), val, tol)
    for k, t in hold.items():
        rest = torch.ones_like(t, dtype=torch.bool)
        rest[:, 1:-1, :H, 8:8 + d] = False
        assert (t[rest] == 7.0).all(), k


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 100])
def test_offsets_beyond_32_bits(dtype, nq):
    """Batch elements more than 2^31 elements apart in one buffer."""
    step, d, nk = (1 << 31) + 64, 64, 130
    buf = torch.zeros(step + 3 * 2 * nk * d, dtype=dtype, device=DEV)
    view = lambda k, n: buf.as_strided((2, 2, n, d), (step, n * d, d, 1), k * 2 * nk * d)
    Q, K, V, dO = _inputs(2, 2, 2, nq, nk, d, dtype)
    q, k, v = view(0, nq), view(1, nk), view(2, nk)
    q.copy_(Q); k.copy_(K); v.copy_(V)
    got, ref = _run(q, k, v, dO, causal=True), _run(Q, K, V, dO, causal=True)
    for x in ref:
        assert torch.equal(got[x], ref[x]), x


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("nq", [1, 200])
def test_same_bits_every_time_and_in_graphs_and_on_streams(dtype, nq):
    Q, K, V, dO = _inputs(2, 4, 2, nq, 700, 64, dtype)
    doc = torch.arange(700)[None].expand(2, 700).div(300, rounding_mode="floor").int().contiguous().to(DEV)
    sp = ln.SoftmaxAttention(causal=True, cap=20.0, doc_q=doc[:, 700 - nq:].contiguous(), doc_k=doc)

    def step():
        O, lse = ln.softmax_attention_fwd(sp, Q, K, V)
        return (O, lse) + ln.softmax_attention_bwd(sp, Q, K, V, O, lse, dO)
    ref = [t.clone() for t in step()]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(step(), ref))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        held = step()
    keep = Q.clone()
    for s in (1.0, 0.5, 1.0):                                   # replays read what the inputs hold then
        Q.copy_(keep * s)
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        now = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, now))
    # two calls at once, each with its own workspace
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = [ln.softmax_attention_fwd(sp, Q, K, V, stream=s) for s in streams]
        grads = [ln.softmax_attention_bwd(sp, Q, K, V, o, l, dO, stream=s) for s, (o, l) in zip(streams, outs)]
        torch.cuda.synchronize()
        for (o, l), g in zip(outs, grads):
            assert all(torch.equal(a, b) for a, b in zip((o, l) + g, ref))


@pytest.mark.parametrize("kw", [dict(), dict(causal=True, cap=4.0), dict(slopes=True)])
def test_gradients_against_differences(kw):
    """Directional derivatives of the fp32 forward pass: central differences with step t in a direction of unit norm are off by
    O(t^2) of the third derivative and by the forward error 2 u S / t, S = |dO||O| the absolute sum of the product; t = 2^-6
    balances them near 1e-3 of the gradient's norm."""
    if kw.get("slopes"):
        kw = dict(slopes=_slopes(2))
    Q, K, V, dO = _inputs(1, 2, 2, 40, 40, 32, F32, sigma=1.0)
    got = _run(Q, K, V, dO, **kw)
    f = lambda *x: float((_run(*x, **kw)["O"].double() * dO.double()).sum())
    g = torch.Generator().manual_seed(3)
    for at, name in enumerate(("dQ", "dK", "dV")):
        D = torch.randn(Q.shape, generator=g).to(DEV)
        D /= D.norm()
        t = 2.0 ** -6
        plus, minus = ([x + s * t * D if k == at else x for k, x in enumerate((Q, K, V))] for s in (1, -1))
        diff = (f(*plus) - f(*minus)) / (2 * t)
        assert abs(diff - float((got[name].double() * D.double()).sum())) < 5e-3 * float(got[name].norm()), name


def test_prepared_heads_feed_both_attentions():
    """Norms and rotation, then softmax attention and the Laplacian path on the same prepared heads, and back."""
    B, H, n, d = 2, 4, 197, 64
    g = torch.Generator().manual_seed(11)
    qkv = torch.randn(B, n, 3, H, d, generator=g).to(BF).to(DEV)
    Q, K, V = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    gq, gk = (torch.rand(d, generator=g).to(DEV) + 0.5 for _ in range(2))
    rope = ln.Rope(d, ln.rope_frequencies(d)[0].to(DEV))
    Qr, Kr = ln.qk_norm_rope_fwd(rope, Q, K, gq, gk)
    sp = ln.SoftmaxAttention(cap=30.0)
    dO = torch.randn(B, H, n, d, generator=g).to(BF).to(DEV)
    O, lse = ln.softmax_attention_fwd(sp, Qr, Kr, V)
    dQr, dKr, dV = ln.softmax_attention_bwd(sp, Qr, Kr, V, O, lse, dO)
    dQ, dK, dgq, dgk = ln.qk_norm_rope_bwd(rope, Q, K, dQr, dKr, gq, gk)
    # the same chain in 64 bits, with the prepared heads and their gradients rounded where they are stored
    leaf = lambda t: t.detach().double().requires_grad_()
    q, k, a, c = leaf(Q), leaf(K), leaf(gq), leaf(gk)
    ang = torch.arange(n, device=DEV).double()[:, None] * ln.rope_frequencies(d)[0].to(DEV)

    def prepare(x, gain):
        x = gain * x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        u, v = x[..., :d // 2], x[..., d // 2:]
        return torch.cat((u * ang.cos() - v * ang.sin(), u * ang.sin() + v * ang.cos()), -1)
    qr, kr = prepare(q, a), prepare(k, c)
    s = 30 * torch.tanh(qr @ kr.transpose(-1, -2) / math.sqrt(d) / 30)
    out = torch.softmax(s, -1) @ V.double()
    out.backward(dO.double())
    rel = lambda x, y: float((x.double() - y.detach()).norm() / y.detach().norm())
    # roundings to bf16 of at most 2^-8 a value: the prepared heads (two), A, ds, O, the gradients of the prepared heads and the
    # results: eight at most, none of them amplified in the norm
    for x, y in ((O, out), (dQ, q.grad), (dK, k.grad), (dgq, a.grad), (dgk, c.grad)):
        assert rel(x, y) < 8 * 2.0 ** -8
    # and the Laplacian path takes the prepared heads as they are
    p = ln.Problem(B, H, n, d, 49, float(d), 6, prefix=1, gh=14, gw=14, mh=7, mw=7)
    saved = torch.empty(ln.laplace_nystrom_saved_bytes(p), dtype=torch.uint8, device=DEV)
    Vc = V.contiguous()
    ln.laplace_nystrom_fwd(p, Qr, Kr, Vc, saved=saved)
    dQl, dKl, _, _ = ln.laplace_nystrom_bwd(p, Qr, Kr, Vc, dO, saved)
    for t in ln.qk_norm_rope_bwd(rope, Q, K, dQl, dKl, gq, gk):
        assert torch.isfinite(t).all()


def test_refusals_on_the_device():
    Q, K, V, dO = _inputs(2, 4, 2, 20, 30, 64, BF)
    ok = ln.SoftmaxAttention()
    for args in ((Q, K[:, :, :29], V), (Q, K.float(), V), (Q, K, V.cpu()), (Q, K.transpose(2, 3), V), (Q[0], K, V)):
        with pytest.raises(ValueError):
            ln.softmax_attention_fwd(ok, *args)
    I = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    for bad in (dict(kv_len=I(3)), dict(kv_len=I(2).long()), dict(doc_q=I(2, 20), doc_k=I(2, 20)), dict(slopes=torch.ones(2, device=DEV)),
                dict(causal=True, prefix=I(2).cpu())):
        with pytest.raises(ValueError):
            ln.softmax_attention_fwd(ln.SoftmaxAttention(**bad), Q, K, V)
    for bad in (dict(prefix=I(2)), dict(doc_q=I(2, 20)), dict(cap=-1.0), dict(cap=math.inf), dict(scale=math.nan)):
        with pytest.raises(ln.LnError):
            ln.softmax_attention_fwd(ln.SoftmaxAttention(**bad), Q, K, V)
    with pytest.raises(ln.LnError):                             # rows of the output overlap
        ln.softmax_attention_fwd(ok, Q, K, V, O=Q[:, :1].expand(2, 4, 20, 64))
    with pytest.raises(ln.LnError):                             # rows that do not start on 16 bytes
        ln.softmax_attention_fwd(ok, Q, torch.zeros(2, 2, 30, 68, dtype=BF, device=DEV)[..., 4:], V)
    with pytest.raises(ln.LnError):                             # heads do not divide
        ln.softmax_attention_fwd(ok, Q[:, :3], K, V)
    with pytest.raises(ln.LnError):                             # head dim
        ln.softmax_attention_fwd(ok, Q[..., :48], K[..., :48], V[..., :48])
    with pytest.raises(ln.LnError):
        ln.softmax_attention_fwd(ln.SoftmaxAttention(doc_q=I(2, 20), doc_k=I(2, 30)), Q, K, V, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
