"""Host side of the query / key preparation and of softmax attention, without a GPU: frequencies, tables, sizes, refusals, and the
reference's own gradients against differences."""
import ctypes
import math

import pytest
import torch

import paper_2604_20368_b200 as ln
from attention_reference import attention
from paper_2604_20368_b200 import binding

FAKE = ctypes.c_void_p(4096)                       # never dereferenced: validation fails first
NEAR = ctypes.c_void_p(4100)                       # not on 16 bytes


class View(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


def _view(data=FAKE, b=16384, h=2048, t=64):
    return ctypes.byref(View(data.value if data else None, b, h, t))


def _rope(**kw):
    c = binding._CRope(64, 64, 0, 1, FAKE.value, 1.0, None, 0, 0, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _softmax(**kw):
    c = binding._CSoftmax(2, 4, 2, 24, 24, 64, 1, 0.125, 0.0, 0, None, None, None, None, None)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("kw,status", [
    (dict(d=96), -2), (dict(r=24), -2), (dict(r=128), -1), (dict(r=-16), -1), (dict(dtype=2), -1), (dict(turns=None), -1), (dict(r=0), -1),
    (dict(turns=4100), -1), (dict(factor=math.nan), -1), (dict(pos=4097), -1)])
def test_rope_refusals(kw, status):
    p = _rope(**kw)
    for entry in ("rope_fwd", "rope_bwd"):
        assert getattr(binding.lib(), entry)(ctypes.byref(p), 2, 8, 8, 8, _view(), _view(), _view(), _view(), None) == status
    assert binding.lib().qk_norm_rope_bwd_workspace_bytes(ctypes.byref(p), 2, 8, 8, 8) == 0


def test_rope_sizes_and_views():
    L, p = binding.lib(), _rope()
    call = lambda B, n, Hq, Hk, *v: L.rope_fwd(ctypes.byref(p), B, n, Hq, Hk, *v, None)
    ok = _view()
    for bad in ((0, 8, 8, 8), (2, 0, 8, 8), (2, 8, 0, 8), (2, 8, 8, -1)):
        assert call(*bad, ok, ok, ok, ok) == -1
    assert call(2, (1 << 30) + 1, 8, 8, ok, ok, ok, ok) == -2
    assert call(1 << 14, 1 << 14, 8, 8, ok, ok, ok, ok) == -2            # 2^32 rows
    for bad in (_view(None), _view(NEAR), _view(t=60), _view(h=-2048)):
        assert call(2, 8, 8, 8, bad, ok, ok, ok) == -1
        assert call(2, 8, 8, 8, ok, ok, ok, bad) == -1
    assert call(2, 8, 8, 8, ok, ok, ok, _view(h=0)) == -1                # rows of an output overlap
    assert call(2, 8, 8, 8, ok, ok, ok, _view(b=7 * 2048 + 7 * 64)) == -1
    assert L.qk_norm_rope_fwd(ctypes.byref(p), 2, 8, 8, 8, -1.0, None, None, ok, ok, ok, ok, None) == -1
    assert L.qk_norm_rope_fwd(ctypes.byref(p), 2, 8, 8, 8, 1e-6, NEAR, None, ok, ok, ok, ok, None) == -1
    need = L.qk_norm_rope_bwd_workspace_bytes(ctypes.byref(p), 2, 8, 8, 8)
    assert need > 0
    back = lambda ws, size: L.qk_norm_rope_bwd(ctypes.byref(p), 2, 8, 8, 8, 1e-6, None, None, ok, ok, ok, ok, ok, ok, FAKE, None, ws, size, None)
    assert back(FAKE, need - 1) == -3 and back(None, need) == -1


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), -1), (dict(nq=0), -1), (dict(nk=-1), -1), (dict(Hk=3), -1), (dict(d=96), -2), (dict(dtype=5), -1), (dict(B=40000), -2),
    (dict(nk=(1 << 30) + 1), -2), (dict(scale=math.inf), -1), (dict(scale=0.0), -1), (dict(cap=-1.0), -1), (dict(cap=math.nan), -1), (dict(causal=2), -1),
    (dict(prefix=4096), -1), (dict(doc_q=4096), -1), (dict(doc_k=4096), -1), (dict(kv_len=4098), -1)])
def test_softmax_refusals(kw, status):
    L, p, ok = binding.lib(), _softmax(**kw), _view()
    assert L.softmax_attention_workspace_bytes(ctypes.byref(p), 0) == 0
    assert L.softmax_attention_fwd(ctypes.byref(p), ok, ok, ok, ok, FAKE, FAKE, 1 << 40, None, None) == status
    assert L.softmax_attention_bwd(ctypes.byref(p), ok, ok, ok, ok, FAKE, ok, ok, ok, ok, FAKE, 1 << 40, None, None) == status


def test_softmax_views_and_workspace():
    L, p, ok = binding.lib(), _softmax(doc_q=4096, doc_k=4096), _view()
    assert L.softmax_attention_workspace_bytes(ctypes.byref(_softmax()), 0) > 0
    for backward in (0, 1):
        need = L.softmax_attention_workspace_bytes(ctypes.byref(p), backward)
        assert need > 0
        if backward:
            call = lambda q, o, ws, size: L.softmax_attention_bwd(ctypes.byref(p), q, ok, ok, ok, FAKE, ok, o, ok, ok, ws, size, None, None)
        else:
            call = lambda q, o, ws, size: L.softmax_attention_fwd(ctypes.byref(p), q, ok, ok, o, FAKE, ws, size, None, None)
        assert call(ok, ok, FAKE, need - 1) == -3
        assert call(ok, ok, None, need) == -1 and call(ok, ok, NEAR, need) == -1
        assert call(_view(t=68), ok, FAKE, need) == -1 and call(_view(None), ok, FAKE, need) == -1
        assert call(ok, _view(t=32), FAKE, need) == -1 and call(_view(t=0), ok, FAKE, need) == -1
    assert L.softmax_attention_fwd(ctypes.byref(p), ok, ok, ok, ok, None, FAKE, 1 << 40, None, None) == -1
    # a step splits its keys over CTAs and needs room for their parts; more than 2^22 - 64 queries, or keys of a backward pass
    step, short = _softmax(nq=1, nk=1 << 20), _softmax(nq=1, nk=8)
    assert L.softmax_attention_workspace_bytes(ctypes.byref(step), 0) > L.softmax_attention_workspace_bytes(ctypes.byref(short), 0) > 0
    assert L.softmax_attention_fwd(ctypes.byref(step), ok, ok, ok, ok, FAKE, FAKE, 256, None, None) == -3
    assert L.softmax_attention_workspace_bytes(ctypes.byref(_softmax(nq=1, nk=1 << 25)), 0) > 0
    assert L.softmax_attention_workspace_bytes(ctypes.byref(_softmax(nq=1, nk=1 << 25)), 1) == 0
    assert L.softmax_attention_workspace_bytes(ctypes.byref(_softmax(nq=1 << 23)), 0) == 0


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(1, 2, 4, 64)
    rope = ln.Rope(64, ln.rope_frequencies(64)[0])
    for call in (lambda: ln.rope_fwd(rope, x), lambda: ln.rope_bwd(rope, x), lambda: ln.qk_norm_rope_fwd(rope, x, x),
                 lambda: ln.qk_norm_rope_bwd(rope, x, x, x, x), lambda: ln.softmax_attention_fwd(ln.SoftmaxAttention(), x, x, x),
                 lambda: ln.softmax_attention_bwd(ln.SoftmaxAttention(), x, x, x, x, torch.zeros(1, 2, 4), x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ln.rope_fwd(ln.Rope(32), x)


def test_table_holds_the_fraction_of_a_turn():
    freq = torch.tensor([1.0, 0.01, 7.5, -0.3, 2 * math.pi, 1e-7], dtype=torch.float64)
    rope = ln.Rope(64, freq)
    assert rope.r == 12 and rope.turns.dtype == torch.int64
    for f, t in zip(freq.tolist(), rope.turns.tolist()):
        part = (t % 2 ** 64) / 2 ** 64
        assert 0 <= part <= 1 and abs((f / (2 * math.pi) - part + 0.5) % 1 - 0.5) < 1e-15
    assert ln.Rope(64).turns is None
    with pytest.raises(ValueError):
        ln.Rope(64, [math.nan])


def test_scaled_frequencies():
    plain, one = ln.rope_frequencies(64)
    assert one == 1.0 and torch.allclose(plain, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32))
    assert torch.equal(ln.rope_frequencies(64, scaling=dict(kind="linear", factor=4.0))[0], plain / 4)
    ntk, _ = ln.rope_frequencies(64, scaling=dict(kind="ntk", factor=4.0))
    assert ntk[0] == 1.0 and abs(float(ntk[-1] / plain[-1]) - 0.25) < 1e-12
    for kind in ("yarn", "bands"):
        f, factor = ln.rope_frequencies(128, scaling=dict(kind=kind, factor=8.0, original=4096))
        base, _ = ln.rope_frequencies(128)
        assert torch.allclose(f[:8], base[:8]) and torch.allclose(f[-8:], base[-8:] / 8)        # fast pairs stay, slow ones scale
        assert ((f <= base * (1 + 1e-12)) & (f >= base / 8 * (1 - 1e-12))).all()
        assert factor == pytest.approx(0.1 * math.log(8.0) + 1 if kind == "yarn" else 1.0)
    for bad in (dict(kind="none", factor=2.0), dict(kind="linear", factor=0.5)):
        with pytest.raises(ValueError):
            ln.rope_frequencies(64, scaling=bad)
    with pytest.raises(ValueError):
        ln.rope_frequencies(63)


@pytest.mark.parametrize("kw", [dict(), dict(causal=True, cap=2.0, prefix=torch.tensor([3, 0])), dict(cap=3.0, kv_len=torch.tensor([5, 0])),
                                dict(doc_q=torch.tensor([[0, 0, -1, 1, 1, 2]] * 2), doc_k=torch.tensor([[0, 1, 1, -1, 0, 0, 5]] * 2))])
def test_reference_gradients_against_differences(kw):
    g = torch.Generator().manual_seed(0)
    x = [torch.randn(2, h, n, 4, generator=g, dtype=torch.float64) for h, n in ((4, 6), (2, 7), (2, 7))]
    dO = torch.randn(2, 4, 6, 4, generator=g, dtype=torch.float64)
    kw = dict(kw, slopes=torch.tensor([0.5, 0.1, 0.2, 0.3]))
    val, _ = attention(*x, dO, **kw)
    f = lambda y: float((attention(*y, **kw)[0]["O"] * dO).sum())
    for at, name in enumerate(("dQ", "dK", "dV")):
        D = torch.randn(x[at].shape, generator=g, dtype=torch.float64)
        diff = (f([t + 1e-5 * D if k == at else t for k, t in enumerate(x)]) - f([t - 1e-5 * D if k == at else t for k, t in enumerate(x)])) / 2e-5
        assert abs(diff - float((val[name] * D).sum())) < 1e-7 * float(val[name].abs().sum() + 1)
