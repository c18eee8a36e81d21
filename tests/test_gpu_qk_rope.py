"""Rotary positions and head norms against their definitions in 64 bits, element by element."""
import math

import pytest
import torch

import paper_2604_20368_b200 as ln

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _half(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


def _turn(x, pos, freq, factor, interleaved, sign=1.0):
    """Definition in 64 bits: x [B, H, n, d], pos [B, n]."""
    r = 2 * freq.numel()
    ang = pos.double()[:, None, :, None] * freq
    c, s = ang.cos() * factor, ang.sin() * factor * sign
    y = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def _reach(x, r, interleaved):
    """|x| and its partner's |x| added: what the two terms of a rotated channel are at most, over the factor."""
    y = x.abs().clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


def _within(got, ref, size, dtype, steps):
    """|got - ref| <= half a step of the storage type + `steps` half steps of 32 bits of `size` (the terms that are added)."""
    x = got.detach().cpu().double()
    assert x.shape == ref.shape and not torch.isnan(x).any()
    err, tol = (x - ref).abs(), _half(dtype) * ref.abs() + steps * 2.0 ** -24 * size + 1e-37
    assert (err <= tol).all(), float((err / tol).max())


def _case(B, Hq, Hk, n, d, r, interleaved, dtype, seed=0, scaling=None, packed=False, far=False):
    g = torch.Generator().manual_seed(seed + n + d)
    if packed:
        x = torch.randn(B, n, Hq + 2 * Hk, d, generator=g).to(dtype).to(DEV)
        Q, K = x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + Hk].transpose(1, 2)
    else:
        Q, K = (torch.randn(B, h, n, d, generator=g).to(dtype).to(DEV) for h in (Hq, Hk))
    freq, factor = ln.rope_frequencies(r, scaling=scaling)
    rope = ln.Rope(d, freq, interleaved=interleaved, factor=factor, device=DEV)
    lo, hi = (-5, 5000) if not far else (10 ** 6, 2 ** 31 - 1)
    pos = torch.randint(lo, hi, (B, n), generator=g, dtype=torch.int32)
    dY = [torch.randn(t.shape, generator=g).to(dtype).to(DEV) for t in (Q, K)]
    return Q, K, freq, factor, rope, pos, dY


SHAPES = [(1, 1, 1, 1, 64, 64), (3, 5, 2, 7, 64, 32), (2, 6, 6, 197, 64, 64), (2, 3, 1, 33, 32, 16), (1, 8, 2, 130, 128, 128),
          (4, 2, 2, 65, 128, 48), (17, 16, 4, 1, 128, 64), (2, 40, 40, 3, 32, 32)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("packed", [False, True])
def test_rotation_and_its_transpose(dtype, interleaved, shape, packed):
    Q, K, freq, factor, rope, pos, (dq, dk) = _case(*shape, interleaved, dtype, packed=packed, scaling=dict(kind="yarn", factor=4.0, original=512))
    out = ln.rope_fwd(rope, Q, K, pos=pos.to(DEV)) + ln.rope_bwd(rope, dq, dk, pos=pos.to(DEV))
    # sine and cosine to 2 ulp each with the rounding of the phase (pi half steps), the factor, two products, one sum: 12 half steps
    for got, x, sign in zip(out, (Q, K, dq, dk), (1.0, 1.0, -1.0, -1.0)):
        x = x.cpu().double()
        _within(got, _turn(x, pos, freq, factor, interleaved, sign), factor * _reach(x, shape[5], interleaved), dtype, 12)
        assert torch.equal(got[..., shape[5]:].cpu().double(), x[..., shape[5]:])     # the other channels are copied


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_keep_their_angle(interleaved):
    Q, K, freq, factor, rope, pos, _ = _case(2, 2, 2, 50, 64, 64, interleaved, F32, far=True)
    Qr, _ = ln.rope_fwd(rope, Q, K, pos=pos.to(DEV))
    # the angle in exact arithmetic: positions up to 2^31 leave a double only 2^-22 of a turn
    from fractions import Fraction
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937511")
    ang = torch.tensor([[[float(Fraction(f) * int(p) % two_pi) for f in freq.tolist()] for p in row] for row in pos], dtype=torch.float64)
    x = Q.cpu().double()
    ref = x.clone()
    a, b = (slice(0, 64, 2), slice(1, 64, 2)) if interleaved else (slice(0, 32), slice(32, 64))
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    ref[..., a], ref[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    # the table holds 2^-64 of a turn: at 2^31 the phase is off by 2^-33 turns = 2^-30.3 rad, under one half step of 32 bits more
    _within(Qr, ref, _reach(x, 64, interleaved), F32, 13)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_start_shared_positions_no_keys_and_in_place(dtype):
    Q, K, freq, factor, rope, _, _ = _case(3, 2, 2, 21, 64, 64, False, dtype)
    start = 100000
    pos = torch.arange(start, start + 21, dtype=torch.int32)
    a = ln.rope_fwd(rope, Q, K, start=start)
    b = ln.rope_fwd(rope, Q, K, pos=pos.to(DEV))
    c = ln.rope_fwd(rope, Q, K, pos=pos[None].expand(3, 21).contiguous().to(DEV))
    d, none = ln.rope_fwd(rope, Q, start=start)
    assert none is None
    wide = torch.stack([pos, pos * 0], 1).to(DEV)                # positions with a stride
    e = ln.rope_fwd(rope, Q, K, pos=wide[:, 0])
    for x in (b, c, e):
        assert torch.equal(a[0], x[0]) and torch.equal(a[1], x[1])
    assert torch.equal(a[0], d)
    Q2, K2 = Q.clone(), K.clone()
    ln.rope_fwd(rope, Q2, K2, start=start, Qr=Q2, Kr=K2)
    assert torch.equal(a[0], Q2) and torch.equal(a[1], K2)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gains", [False, True])
def test_norm_with_rotation_and_gradients(dtype, interleaved, shape, gains):
    B, Hq, Hk, n, d, r = shape
    Q, K, freq, factor, rope, pos, dY = _case(*shape, interleaved, dtype, packed=True, scaling=dict(kind="linear", factor=8.0))
    Q[0, 0, 0] = 0.0                                             # a row of zeros: rstd = eps^-1/2, gradient through it alone
    g = torch.Generator().manual_seed(1)
    gain = [torch.rand(d, generator=g) + 0.5 if gains else None for _ in range(2)]
    gd = [None if x is None else x.to(DEV) for x in gain]
    eps, P = 1e-5, pos.to(DEV)
    Qr, Kr = ln.qk_norm_rope_fwd(rope, Q, K, *gd, eps=eps, pos=P)
    dQ, dK, dgq, dgk = ln.qk_norm_rope_bwd(rope, Q, K, *dY, *gd, eps=eps, pos=P)
    for x, y, dy, dx, w, dg in ((Q, Qr, dY[0], dQ, gain[0], dgq), (K, Kr, dY[1], dK, gain[1], dgk)):
        X, D = x.cpu().double(), dy.cpu().double()
        W = torch.ones(d, dtype=torch.float64) if w is None else w.double()
        rstd = (X.square().mean(-1, keepdim=True) + eps).rsqrt()
        # the sum of squares (d / E + log steps), rsqrt to 2 ulp, two products on top of the rotation: d / 8 + 24 half steps
        steps = d / 8 + 24
        _within(y, _turn(X * rstd * W, pos, freq, factor, interleaved), factor * _reach(X * rstd * W, r, interleaved), dtype, steps)
        t = _turn(D, pos, freq, factor, interleaved, -1.0)
        size = factor * _reach(D, r, interleaved)                # what t's rounding is measured against
        u = t * W
        ref = rstd * (u - X * rstd ** 2 * (u * X).mean(-1, keepdim=True))
        big = rstd * (size * W + X.abs() * rstd ** 2 * (size * W * X.abs()).mean(-1, keepdim=True))
        _within(dx, ref, big, dtype, 4 * steps)
        if w is not None:
            # rows are added in 32 bits by a lane, then across lanes and CTAs: rows / (lanes) + steps half steps of the absolute sum
            rows = X[..., 0].numel()
            _within(dg, (t * X * rstd).sum((0, 1, 2)), (size * X.abs() * rstd).sum((0, 1, 2)), F32, steps + rows)
        else:
            assert dg is None


def test_norm_alone_and_without_keys():
    Q, _, _, _, _, _, (dq, _) = _case(2, 3, 1, 19, 64, 64, False, F32)
    rope = ln.Rope(64)
    Qr, none = ln.qk_norm_rope_fwd(rope, Q, None, eps=0.0)
    assert none is None
    X = Q.cpu().double()
    ref = X / X.square().mean(-1, keepdim=True).sqrt()
    _within(Qr, ref, ref.abs(), F32, 20)
    gq = torch.ones(64, device=DEV)
    dQ, dK, dgq, dgk = ln.qk_norm_rope_bwd(rope, Q, None, dq, None, gq, None, eps=0.0)
    assert dK is None and dgk is None and torch.isfinite(dgq).all() and torch.isfinite(dQ).all()


def test_gradients_against_differences():
    """Central differences of the fp32 forward pass in a direction of unit norm, step t = 2^-6: off by O(t^2) and by
    2^-23 S / t, S = |dY||Y|; both below 1e-3 of the gradient's norm at this size."""
    Q, K, freq, factor, rope, pos, dY = _case(1, 2, 2, 9, 64, 32, False, F32)
    P = pos.to(DEV)
    g = torch.Generator().manual_seed(2)
    x = [Q, K, torch.rand(64, generator=g).to(DEV) + 0.5, torch.rand(64, generator=g).to(DEV) + 0.5]
    grads = ln.qk_norm_rope_bwd(rope, Q, K, *dY, x[2], x[3], pos=P)
    f = lambda y: sum(float((a.double() * b.double()).sum()) for a, b in zip(ln.qk_norm_rope_fwd(rope, *y, pos=P), dY))
    for at, grad in enumerate(grads):
        D = torch.randn(x[at].shape, generator=g).to(DEV)
        D /= D.norm()
        t = 2.0 ** -6
        diff = (f([y + t * D if k == at else y for k, y in enumerate(x)]) - f([y - t * D if k == at else y for k, y in enumerate(x)])) / (2 * t)
        assert abs(diff - float((grad.double() * D.double()).sum())) < 5e-3 * float(grad.norm()), at


@pytest.mark.parametrize("dtype", [F32, BF])
def test_outputs_inside_a_cache_and_far_offsets(dtype):
    """Keys written at one position of a cache, whose other rows stay as they are; batch elements 2^31 elements apart."""
    step = (1 << 31) + 64
    buf = torch.zeros(step + 4 * 10 * 64, dtype=dtype, device=DEV)
    cache = buf.as_strided((2, 4, 10, 64), (step, 640, 64, 1))
    Q, K, _, _, rope, pos, _ = _case(2, 4, 4, 1, 64, 64, True, dtype)
    P = pos.to(DEV)
    Qr, Kr = ln.qk_norm_rope_fwd(rope, Q, K, pos=P)
    ln.qk_norm_rope_fwd(rope, Q, K, pos=P, Kr=cache[:, :, 7:8])
    assert torch.equal(cache[:, :, 7:8], Kr)
    assert not cache[:, :, :7].any() and not cache[:, :, 8:].any()


def test_same_bits_every_time_in_graphs_and_on_streams():
    Q, K, _, _, rope, pos, dY = _case(4, 6, 2, 500, 64, 64, False, BF, packed=True)
    P = pos.to(DEV)
    gq, gk = (torch.rand(64, device=DEV) + 0.5 for _ in range(2))
    step = lambda **kw: ln.qk_norm_rope_fwd(rope, Q, K, gq, gk, pos=P, **kw) + ln.qk_norm_rope_bwd(rope, Q, K, *dY, gq, gk, pos=P, **kw)
    ref = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = step(stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    P.add_(3)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_refusals_on_the_device():
    Q, K, freq, _, rope, pos, (dq, dk) = _case(2, 4, 2, 8, 64, 64, False, BF)
    P = pos.to(DEV)
    for kw in (dict(pos=P.long()), dict(pos=P[:, :7]), dict(pos=pos), dict(pos=P[None])):
        with pytest.raises(ValueError):
            ln.rope_fwd(rope, Q, K, **kw)
    for a, b in ((Q, K.float()), (Q, K[:, :, :7]), (Q.transpose(2, 3), K), (Q[0], K), (Q.cpu(), K.cpu())):
        with pytest.raises(ValueError):
            ln.rope_fwd(rope, a, b, pos=P)
    with pytest.raises(ValueError):
        ln.qk_norm_rope_fwd(rope, Q, K, torch.ones(64, device=DEV).half(), None, pos=P)
    with pytest.raises(ln.LnError):                              # overlapping rows of an output
        ln.rope_fwd(rope, Q, K, pos=P, Qr=Q[:, :1].expand(2, 4, 8, 64))
    with pytest.raises(ln.LnError):
        ln.qk_norm_rope_fwd(rope, Q, K, eps=-1.0, pos=P)
    with pytest.raises(ln.LnError):                              # 24 rotated channels
        ln.rope_fwd(ln.Rope(64, freq[:12], device=DEV), Q, K, pos=P)
    with pytest.raises(ln.LnError):
        ln.rope_fwd(ln.Rope(64, freq, factor=math.inf, device=DEV), Q, K, pos=P)
    with pytest.raises(ln.LnError):                              # rows that do not start on 16 bytes
        ln.rope_fwd(rope, torch.zeros(2, 4, 8, 68, dtype=BF, device=DEV)[..., 4:], K, pos=P)
