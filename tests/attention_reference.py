"""Softmax attention with capped, biased and masked scores in 64 bits, with its gradients and, for every output, the sums of
absolute values that the rounding errors of a kernel are measured against.  Plain loops over batch elements and heads."""
import math

import torch


def bounds(dtype):
    """(half a step of the storage type relative to the value, half a step of the operands of a matrix product)."""
    return (2.0 ** -8, 2.0 ** -8) if dtype == torch.bfloat16 else (2.0 ** -24, 0.0)


def mask(b, nq, nk, causal=False, prefix=None, doc_q=None, doc_k=None, kv_len=None):
    """Allowed pairs [nq, nk] of batch element b, and the distance of every pair."""
    length = nk if kv_len is None else min(max(int(kv_len[b]), 0), nk)
    i, j = torch.arange(nq)[:, None] + length - nq, torch.arange(nk)[None]
    ok = (j < length).expand(nq, nk).clone()
    if causal:
        ok &= (j <= i) | (j < (0 if prefix is None else int(prefix[b])))
    if doc_q is not None:
        ok &= (doc_q[b][:, None] == doc_k[b][None]) & (doc_k[b][None] >= 0)
    return ok, (i - j).abs().double()


def attention(Q, K, V, dO=None, scale=None, cap=0.0, slopes=None, dtype=torch.float32, **masks):
    """Returns (values, tolerances): dicts of O, lse and, given dO, dQ, dK, dV, in double on the CPU.

    Tolerances, element by element.  With h the half step of the storage type, o that of rounded product operands (A and ds are
    rounded to bf16 for the tensor cores; fp32 storage keeps 24 bits) and u = 2^-24:
      score       a dot product of d terms in 32 bits is off by at most d u sum|q k|, so x is off by e_s = d u scale sum|q||k| plus
                  8 u |x| for the scale, cap and bias steps; the forward pass and the backward pass each make that error, and
                  ex2 is off by 2^-22: a probability is off by  e_p = 2 e_s + 2^-21  of its value
      O           (h + n u) |O| + (o + e_p + n u) (A |V|)
      lse         e_s + 4 u |lse| + (n u + 2^-21)
      delta       off by e_d = h sum|dO||O| (the stored O) + the error of O that the tolerance above allows, through |dO|
      ds          A bend scale (dP - delta): off by (o + e_p + 4 u) |ds| + A scale (d u |dO||V| + e_d) + cap error
      dQ, dK, dV  h |value| + the errors of ds (A) through |K|, |Q| (|dO|) + n u of the absolute sums
    """
    Q, K, V = (t.detach().cpu().double() for t in (Q, K, V))
    B, Hq, nq, d = Q.shape
    Hk, nk = K.shape[1:3]
    G = Hq // Hk
    scale = 1 / math.sqrt(d) if scale is None else scale
    masks = {k: (None if v is None else v.cpu() if torch.is_tensor(v) else v) for k, v in masks.items()}
    h, o = bounds(dtype)
    u, n = 2.0 ** -24, max(nq * G, nk)
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    val = dict(O=z(B, Hq, nq, d), lse=torch.full((B, Hq, nq), -math.inf, dtype=torch.float64))
    tol = dict(O=z(B, Hq, nq, d), lse=z(B, Hq, nq))
    if dO is not None:
        dO = dO.detach().cpu().double()
        for x, s in (("dQ", Q.shape), ("dK", K.shape), ("dV", V.shape)):
            val[x], tol[x] = z(*s), z(*s)
    clean = lambda t, used: torch.where(used[:, None], t, torch.zeros((), dtype=torch.float64))
    for b in range(B):
        ok, dist = mask(b, nq, nk, **masks)
        # what no pair uses may hold anything
        rows, cols = ok.any(1), ok.any(0)
        for hq in range(Hq):
            q, k, v = clean(Q[b, hq], rows), clean(K[b, hq // G], cols), clean(V[b, hq // G], cols)
            raw = scale * (q @ k.T)
            t = torch.tanh(raw / cap) if cap else None
            s = cap * t if cap else raw
            bend = 1 - t * t if cap else torch.ones_like(s)
            if slopes is not None:
                s = s - float(slopes[hq]) * dist
            e_s = d * u * scale * (q.abs() @ k.abs().T) + 8 * u * (s.abs() + raw.abs() + (cap or 0.0))
            s = s.masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(s, 1)
            A = torch.where(ok, torch.exp(s - torch.where(rows, lse, 0.0)[:, None]), 0.0)
            e_p = 2 * e_s + 2.0 ** -21 + 8 * u * torch.where(rows, lse, 0.0).abs()[:, None]
            out = A @ v
            val["O"][b, hq], val["lse"][b, hq] = out, lse
            tol["O"][b, hq] = (h + n * u) * out.abs() + ((o + e_p + n * u) * A) @ v.abs() + 1e-37
            tol["lse"][b, hq] = torch.where(rows, e_s.masked_fill(~ok, 0).amax(1) + 4 * u * lse.abs() + n * u + 2.0 ** -21, 0.0)
            if dO is None:
                continue
            g = clean(dO[b, hq], rows)
            dP, delta = g @ v.T, (g * out).sum(1, keepdim=True)
            ds = A * bend * (dP - delta) * scale
            e_d = (g.abs() * (tol["O"][b, hq] + 4 * u * out.abs())).sum(1, keepdim=True) + d * u * (g.abs() * out.abs()).sum(1, keepdim=True)
            # 1 - t^2: t is off by 4 u, and moves by the error of the score over the cap
            e_b = (8 * u + 2 * e_s / cap) if cap else 0.0
            e_ds = (o + e_p + 4 * u) * ds.abs() + A * scale * (bend * (d * u * (g.abs() @ v.abs().T) + e_d) + e_b * (dP - delta).abs())
            val["dQ"][b, hq] = ds @ k
            val["dK"][b, hq // G] += ds.T @ q
            val["dV"][b, hq // G] += A.T @ g
            tol["dQ"][b, hq] = (e_ds + n * u * ds.abs()) @ k.abs()
            tol["dK"][b, hq // G] += (e_ds + n * u * ds.abs()).T @ q.abs()
            tol["dV"][b, hq // G] += ((o + e_p + n * u) * A).T @ g.abs()
    for x in ("dQ", "dK", "dV"):
        if dO is not None:
            tol[x] += h * val[x].abs() + 1e-37
    return val, tol


def check(got, val, tol):
    """Every element of every output within its tolerance; infinities in the same places.  Returns the largest share used."""
    worst = {}
    for name, ref in val.items():
        x = got[name].detach().cpu().double()
        assert x.shape == ref.shape, name
        assert not torch.isnan(x).any(), name
        inf = torch.isinf(ref)
        assert torch.equal(torch.isinf(x), inf) and torch.equal(x[inf], ref[inf]), name
        err, t = (x - ref).abs()[~inf], tol[name][~inf]
        share = torch.where(err == 0, 0.0, err / t)
        worst[name] = float(share.max()) if share.numel() else 0.0
        assert worst[name] <= 1.0, (name, worst[name], float(err.max()))
    return worst
