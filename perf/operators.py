"""Timed cases of the query / key preparation and of the softmax attention that stands beside the Laplacian one.

Three operators, all through the public entry points:
  rope   rotary positions on queries and keys (rope_fwd, and rope_bwd where `train`): interleaved or half layout, the whole
         head or its first channels, plain or scaled frequencies
  qkn    RMS norm of every query and key head and the rotation in the same pass (qk_norm_rope_fwd, qk_norm_rope_bwd)
  attn   softmax attention whose scores may be capped by a tanh, biased by distance, and masked: causal, with a prefix
         that everybody sees, by document, by the filled length of a cache (softmax_attention_fwd, softmax_attention_bwd)
Tensors are [B, H, n, d] views: `packed` ones are slices of the projection's [B, n, Hq + 2 Hk, d] output.  Sizes are those
of perf/cases.py and of paper_2604_20368_b200/synth.py where they exist; inputs are synthetic.

The plain forms compute in 32 bits (angles in 64) with elementary torch operations and round once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------ cases
def _rope(name, kind, B, Hq, Hk, n, d, r, layout="half", scaling="none", start=0, restart=0, packed=True, train=True, dtype="bf16"):
    """r: rotated channels; start: position of the first token; restart: positions start again every so many tokens (0: never)."""
    c = dict(kind=kind, B=B, Hq=Hq, Hk=Hk, n=n, d=d, r=r, layout=layout, scaling=scaling, start=start, restart=restart,
             packed=packed, train=train, dtype=dtype)
    return dict(name=name, **c) if name else c


def _attn(name, B, Hq, Hk, nq, nk, d, causal=False, prefix=0, cap=0.0, bias=False, docs=0, ragged=False, packed=True, train=True,
          dtype="bf16", sigma=1.0):
    """prefix: longest prefix of a batch element; docs: documents per sequence, with padding behind the last (0: no documents);
    ragged: the keys of a batch element end before nk (filled length of a cache)."""
    c = dict(kind="attn", B=B, Hq=Hq, Hk=Hk, nq=nq, nk=nk, d=d, causal=causal, prefix=prefix, cap=cap, bias=bias, docs=docs,
             ragged=ragged, packed=packed, train=train, dtype=dtype, sigma=sigma)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one new token of each of sixteen sequences far into a long context: the smallest call, latency alone
        _rope("rope_step", "rope", 16, 8, 8, 1, 128, 128, scaling="yarn", start=50175, packed=False, train=False),
        # training step of a layer with wide heads, half of each head rotated
        _rope("rope_train", "rope", 16, 8, 8, 4096, 128, 64, layout="half"),
        # 224 x 224 tokens per head, trained on 56 x 56: frequencies scaled for the longer sequence
        _rope("rope_hires224", "rope", 8, 2, 2, 50176, 64, 64, layout="interleaved", scaling="linear", packed=False, train=False),
        # the serving step of a layer that norms its queries and keys: eight query heads share two key heads
        _rope("qkn_step", "qkn", 16, 8, 2, 1, 128, 128, scaling="bands", start=4095, packed=True, train=False),
        # DeiT-Small-shaped training step: 197 tokens, an odd number
        _rope("qkn_deit_train", "qkn", 64, 6, 6, 197, 64, 64, layout="interleaved"),
        # packed documents of a long-sequence training step, positions start again with every document
        _rope("qkn_train", "qkn", 16, 8, 2, 4096, 128, 128, restart=1000),
        # one new token against a long cache whose sequences have different lengths
        _attn("attn_step", 16, 8, 2, 1, 50176, 128, causal=True, ragged=True, packed=False, train=False),
        # DeiT-Small-shaped training step: many small heads, 197 tokens, every token sees every token
        _attn("attn_deit_train", 64, 6, 6, 197, 197, 64),
        # causal training step with capped scores, eight query heads on two key heads
        _attn("attn_capped_train", 4, 8, 2, 4096, 4096, 128, causal=True, cap=20.0, sigma=3.0),
        # images of different sizes packed into one sequence of 112 x 112 tokens: nobody sees another image
        _attn("attn_docs_train", 2, 2, 2, 12544, 12544, 64, docs=12),
        # prompt of a model with distance bias behind a prefix that sees itself both ways, an odd length; forward only
        _attn("attn_prefix_bias", 1, 3, 3, 12545, 12545, 64, causal=True, prefix=999, bias=True, packed=False, train=False),
        # fp32 storage, the precision a user checks gradients or trains small models in
        _attn("attn_f32_train", 8, 4, 4, 784, 784, 64, causal=True, bias=True, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "qkn", "attn", "attn", "attn"])
    d = rng.choice([32, 64, 64, 128, 128])
    Hk = rng.choice([1, 2, 3, 4, 6, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind != "attn":
        Hq = Hk * rng.choice([1, 1, 2, 4])
        n = rng.choice([1, _log_int(rng, 1, 50176), _log_int(rng, 16, 50176)])
        B = _log_int(rng, 1, max(1, min(64, (1 << 26) // (n * (Hq + Hk) * d))))
        return _rope(None, kind, B, Hq, Hk, n, d, rng.choice([d, d, d // 2]), layout=rng.choice(["half", "interleaved"]),
                     scaling=rng.choice(["none", "linear", "ntk", "yarn", "bands"]), start=rng.choice([0, _log_int(rng, 1, 1000000)]),
                     restart=rng.choice([0, 0, _log_int(rng, 2, 4096)]), packed=rng.random() < 0.6, train=rng.random() < 0.6, dtype=dtype)
    step = rng.random() < 0.25                       # a serving step: few queries at the end of a long cache
    G = rng.choice([1, 2, 4, 8] if step else [1, 1, 2, 4])
    Hq = Hk * G
    cap, bias = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3
    sigma = rng.choice([1.0, 3.0])
    if step:
        nk = _log_int(rng, 1, 50176)
        B = _log_int(rng, 1, max(1, min(64, (1 << 27) // (nk * Hk * d))))
        return _attn(None, B, Hq, Hk, min(nk, rng.choice([1, 1, 1, 2])), nk, d, causal=True, cap=cap, bias=bias, ragged=rng.random() < 0.7,
                     packed=False, train=False, dtype=dtype, sigma=sigma)
    most = (1 << 29) // (1 if dtype == "bf16" else 32)          # pairs of a call
    train = rng.random() < 0.6
    n = _log_int(rng, 16, 12545 if dtype == "bf16" else 2048)
    B = _log_int(rng, 1, max(1, min(64, most // (n * n * Hq))))
    Hq, Hk = (Hq, Hk) if B * Hq * n * n <= most else (G, 1)
    docs = rng.choice([0, 0, rng.randint(1, 12)])
    causal = rng.random() < 0.6
    nq = n if docs or train or rng.random() < 0.6 else rng.randint(1, n)
    return _attn(None, B, Hq, Hk, nq, n, d, causal=causal, prefix=rng.choice([0, rng.randint(1, n)]) if causal and not docs else 0, cap=cap,
                 bias=bias, docs=docs, ragged=not train and not docs and rng.random() < 0.3, packed=nq == n and rng.random() < 0.6,
                 train=train, dtype=dtype, sigma=sigma)


# ------------------------------------------------------------------------------------------ inputs
def _frequencies(r, scaling):
    """Radians per position of each rotated channel pair, in 64 bits, and the factor on cosine and sine."""
    i = torch.arange(r // 2, dtype=torch.float64)
    base, factor, original = 10000.0, 16.0, 3136
    if scaling == "linear":                          # every position divided by the factor
        return base ** (-2 * i / r) / factor, 1.0
    if scaling == "ntk":                             # a larger base: the slowest pair slows down by the factor
        return (base * factor ** (r / (r - 2.0) if r > 2 else 1.0)) ** (-2 * i / r), 1.0
    f = base ** (-2 * i / r)
    turns = original * f / (2 * math.pi)             # turns that a pair makes over the original length
    if scaling == "yarn":                            # a ramp over the pair's index between 32 turns and one turn
        at = lambda t: r * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    if scaling == "bands":                           # a ramp over the turns themselves between four and one
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _views(case, normal, nq, nk, dt):
    """Q, K, V as [B, H, n, d] views: slices of one [B, n, Hq + 2 Hk, d] projection, or tensors of their own."""
    B, Hq, Hk, d = case["B"], case["Hq"], case["Hk"], case["d"]
    if case["packed"]:
        x = normal(B, nk, Hq + 2 * Hk, d).to(dt)
        return tuple(t.transpose(1, 2) for t in x.split([Hq, Hk, Hk], 2))
    return normal(B, Hq, nq, d).to(dt), normal(B, Hk, nk, d).to(dt), normal(B, Hk, nk, d).to(dt)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, device=dev, generator=gen)
    integers = lambda lo, hi, *shape: torch.randint(lo, hi, shape, device=dev, generator=gen, dtype=torch.int32)
    B, Hq, Hk, d, dt = case["B"], case["Hq"], case["Hk"], case["d"], TYPES[case["dtype"]]
    st = dict(case=case)
    if case["kind"] != "attn":
        n = case["n"]
        st["Q"], st["K"], _ = _views(case, normal, n, n, dt)
        pos = torch.arange(n, device=dev, dtype=torch.int32)[None].expand(B, n) + case["start"]
        if case["restart"]:                          # document boundaries fall elsewhere in every batch element
            pos = (pos + integers(0, case["restart"], B, 1)) % case["restart"]
        elif n == 1:                                 # sequences of different lengths
            pos = pos - integers(0, max(1, case["start"] // 2), B, 1)
        st["pos"] = pos.contiguous()
        f, factor = _frequencies(case["r"], case["scaling"])
        st["freq"], st["factor"] = f.to(dev), factor
        if case["kind"] == "qkn":
            st["gq"], st["gk"] = (1 + 0.2 * normal(d) for _ in range(2))
        if case["train"]:
            st["dQr"], st["dKr"] = normal(B, Hq, n, d).to(dt), normal(B, Hk, n, d).to(dt)
        if own:
            import paper_2604_20368_b200 as ln
            st["rope"] = ln.Rope(d, st["freq"], interleaved=case["layout"] == "interleaved", factor=factor)
        return st
    nq, nk = case["nq"], case["nk"]
    Q, st["K"], st["V"] = _views(case, normal, nq, nk, dt)
    st["Q"] = Q.mul_(case["sigma"])
    st["scale"] = 1.0 / math.sqrt(d)
    st["prefix"] = integers(case["prefix"] // 2, case["prefix"] + 1, B) if case["prefix"] else None
    st["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=dev) / Hq).float() if case["bias"] else None
    st["kv_len"] = integers(max(nq, nk // 2), nk + 1, B) if case["ragged"] else None
    st["doc"] = None
    if case["docs"]:                                 # lengths of a random partition; what is behind the last document is padding
        cuts = (torch.rand((B, case["docs"]), device=dev, generator=gen) * nk).int().sort(1).values
        doc = (torch.arange(nk, device=dev)[None, :, None] >= cuts[:, None, :]).sum(-1).int()
        st["doc"] = torch.where(doc == case["docs"], -1, doc) if case["docs"] > 1 else doc
    if case["train"]:
        st["dO"] = normal(B, Hq, nq, d).to(dt)
    return st


# ------------------------------------------------------------------------------------------ passes
def run(state):
    kind, train = state["case"]["kind"], state["case"]["train"]
    if own:
        return _own_attn(state) if kind == "attn" else _own_rope(state)
    if kind == "attn":
        return _plain_attn(state)
    cos, sin = _angles(state)
    out = {}
    for x, g, dy in (("Q", "gq", "dQr"), ("K", "gk", "dKr")):
        X = state[x].float()
        y, dg = X, None
        if kind == "qkn":
            rstd = torch.rsqrt((X * X).mean(-1, keepdim=True) + 1e-6)
            xhat = X * rstd
            y = xhat * state[g]
        out[x + "r"] = _turn(y, cos, sin, state["case"]["layout"]).to(state[x].dtype)
        if train:
            dY = _turn(state[dy].float(), cos, -sin, state["case"]["layout"])
            dx = dY
            if kind == "qkn":
                out["d" + g] = (dY * xhat).double().sum((0, 1, 2)).float()
                t = dY * state[g]
                dx = rstd * (t - xhat * (t * xhat).mean(-1, keepdim=True))
            out["d" + x] = dx.to(state[x].dtype)
    return out


def _angles(state):
    """Cosine and sine [B, 1, n, r / 2], formed in 64 bits."""
    a = state["pos"].double()[:, None, :, None] * state["freq"]
    return (torch.cos(a) * state["factor"]).float(), (torch.sin(a) * state["factor"]).float()


def _turn(x, cos, sin, layout):
    r = 2 * cos.shape[-1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if layout == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    u, v = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((u, v), -1).flatten(-2) if layout == "interleaved" else torch.cat((u, v), -1)
    return torch.cat((y, x[..., r:]), -1)


def _own_rope(state):
    import paper_2604_20368_b200 as ln
    kind, train, rope, pos = state["case"]["kind"], state["case"]["train"], state["rope"], state["pos"]
    Q, K = state["Q"], state["K"]
    if kind == "rope":
        Qr, Kr = ln.rope_fwd(rope, Q, K, pos=pos)
        if not train:
            return dict(Qr=Qr, Kr=Kr)
        dQ, dK = ln.rope_bwd(rope, state["dQr"], state["dKr"], pos=pos)
        return dict(Qr=Qr, dQ=dQ, Kr=Kr, dK=dK)
    Qr, Kr = ln.qk_norm_rope_fwd(rope, Q, K, state["gq"], state["gk"], eps=1e-6, pos=pos)
    if not train:
        return dict(Qr=Qr, Kr=Kr)
    dQ, dK, dgq, dgk = ln.qk_norm_rope_bwd(rope, Q, K, state["dQr"], state["dKr"], state["gq"], state["gk"], eps=1e-6, pos=pos)
    return dict(Qr=Qr, dgq=dgq, dQ=dQ, Kr=Kr, dgk=dgk, dK=dK)


def _own_attn(state):
    import paper_2604_20368_b200 as ln
    sp = ln.SoftmaxAttention(scale=state["scale"], cap=state["case"]["cap"], causal=state["case"]["causal"], prefix=state["prefix"],
                             slopes=state["slopes"], doc_q=state["doc"], doc_k=state["doc"], kv_len=state["kv_len"])
    O, lse = ln.softmax_attention_fwd(sp, state["Q"], state["K"], state["V"])
    if not state["case"]["train"]:
        return dict(O=O, lse=lse)
    dQ, dK, dV = ln.softmax_attention_bwd(sp, state["Q"], state["K"], state["V"], O, lse, state["dO"])
    return dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV)


def _allowed(state):
    """Which pairs the masks leave, [B, 1, 1, nq or 1, nk], and each pair's distance [B, 1, 1, nq, nk] (B may be 1).  The last
    query stands at the last key."""
    case = state["case"]
    nq, nk, dev = case["nq"], case["nk"], state["K"].device
    j = torch.arange(nk, device=dev)
    end = state["kv_len"].long()[:, None, None] if state["kv_len"] is not None else torch.full((1, 1, 1), nk, device=dev)
    at = torch.arange(nq, device=dev)[None, :, None] + end - nq
    ok = j < end
    if case["causal"]:
        seen = j <= at
        if state["prefix"] is not None:
            seen = seen | (j < state["prefix"][:, None, None])
        ok = ok & seen
    if state["doc"] is not None:
        ok = ok & (state["doc"][:, :, None] == state["doc"][:, None, :]) & (state["doc"][:, None, :] >= 0)
    return ok[:, None, None], (at - j).abs()[:, None, None]


def _plain_attn(state):
    case = state["case"]
    B, Hq, Hk, nq, d = case["B"], case["Hq"], case["Hk"], case["nq"], case["d"]
    G, cap = Hq // Hk, case["cap"]
    grouped = lambda t: t.float().reshape(B, Hk, G, -1, d)
    q, k, v = grouped(state["Q"]), state["K"].float()[:, :, None], state["V"].float()[:, :, None]
    ok, dist = _allowed(state)
    s = q @ k.transpose(-1, -2) * state["scale"]
    if cap:
        t = torch.tanh(s / cap)
        s = cap * t
    if case["bias"]:
        s = s - state["slopes"].reshape(1, Hk, G, 1, 1) * dist
    s = torch.where(ok, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.where(ok, torch.exp(s - top), 0.0)
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)
    p = p / torch.where(total > 0, total, 1.0)
    O = p @ v
    heads = lambda t, h: t.reshape(B, h, -1, d).to(state["Q"].dtype)
    out = dict(O=heads(O, Hq), lse=lse.reshape(B, Hq, nq))
    if case["train"]:
        dO = grouped(state["dO"])
        ds = p * (dO @ v.transpose(-1, -2) - (dO * O).sum(-1, keepdim=True))
        if cap:
            ds = ds * (1 - t * t)
        ds = ds * state["scale"]
        out["dQ"] = heads(ds @ k, Hq)
        out["dK"] = heads((ds.transpose(-1, -2) @ q).sum(2), Hk)
        out["dV"] = heads((p.transpose(-1, -2) @ dO).sum(2), Hk)
    return out


# ------------------------------------------------------------------------------------------ work
def _pairs(case):
    """Pairs of a query and a key that the masks leave in one head and batch element, in expectation."""
    nq, nk = case["nq"], case["nk"]
    if case["docs"]:                                 # E[sum of squared lengths] of a uniform partition, the last part left out
        k = case["docs"]
        full = nk * nk * (1.0 if k == 1 else 2.0 * k / ((k + 1) * (k + 2)))
        return full / 2 if case["causal"] else full
    keys = nk * (0.75 if case["ragged"] else 1.0)
    if not case["causal"]:
        return nq * keys
    prefix = 0.75 * case["prefix"]
    rows = min(nq, keys)
    return rows * (keys - rows / 2) + (max(0.0, prefix - (keys - rows)) ** 2 / 2)


def work(case):
    """Inputs once, outputs once.  Rotation 6 operations a rotated pair, norm 4 (forward) and 9 (backward) a channel; 4 d
    operations a pair of the masks forward and 10 d backward (five products)."""
    e = 2 if case["dtype"] == "bf16" else 4
    B, Hq, Hk, d = case["B"], case["Hq"], case["Hk"], case["d"]
    if case["kind"] != "attn":
        rows = B * case["n"] * (Hq + Hk)
        norm = case["kind"] == "qkn"
        passes = 2 if not case["train"] else (5 if norm else 4)
        flops = rows * (3 * case["r"] + (4 * d if norm else 0)) + (rows * (3 * case["r"] + (9 * d if norm else 0)) if case["train"] else 0)
        return {"bytes": rows * d * e * passes + 4 * B * case["n"], "flops": flops}
    q, kv = B * Hq * case["nq"] * d * e, 2 * B * Hk * case["nk"] * d * e * (0.75 if case["ragged"] else 1.0)
    flops = B * Hq * _pairs(case) * d * (14 if case["train"] else 4)
    return {"bytes": (4 * q + 2 * kv if case["train"] else 2 * q + kv) + 4 * B * Hq * case["nq"], "flops": flops}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The operators' definitions in 64 bits, a batch element and a head at a time."""
    if case["kind"] == "attn" and case["B"] * case["Hq"] * case["nq"] * case["nk"] * case["d"] > 1 << 38:
        return None
    st = prepare(case, seed)
    return _exact_attn(case, st) if case["kind"] == "attn" else _exact_rope(case, st)


def _exact_rope(case, st):
    r, d, dev = case["r"], case["d"], st["Q"].device
    # channel c turns with its partner as y = x cos + x[partner] sign sin
    c = torch.arange(r, device=dev)
    if case["layout"] == "interleaved":
        partner, sign, pair = c ^ 1, torch.where(c % 2 == 0, -1.0, 1.0).double(), c // 2
    else:
        partner, sign, pair = (c + r // 2) % r, torch.where(c < r // 2, -1.0, 1.0).double(), c % (r // 2)
    out = {}
    for x, g in (("Q", "gq"), ("K", "gk")):
        Y, dX, dg = [], [], torch.zeros(d, dtype=torch.float64, device=dev)
        for b in range(case["B"]):
            phase = torch.outer(st["pos"][b].double(), st["freq"])[:, pair]
            co, si = phase.cos() * st["factor"], phase.sin() * st["factor"] * sign
            X = st[x][b].double()
            w = st[g].double() if case["kind"] == "qkn" else None
            ms = (X.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt()
            N = X / ms * w if w is not None else X
            R = N.clone()
            R[..., :r] = N[..., :r] * co + N[..., partner] * si
            Y.append(R)
            if case["train"]:
                D = st["d" + x + "r"][b].double()
                # the transpose: channel c receives its own cosine and its partner's sine
                E = D.clone()
                E[..., :r] = D[..., :r] * co + D[..., partner] * si[:, partner]
                if w is not None:
                    dg += (E * X / ms).sum((0, 1))
                    E = E * w / ms
                    E = E - X / ms.pow(2) * ((E * X).sum(-1, keepdim=True) / d)
                dX.append(E)
        out[x + "r"] = torch.stack(Y)
        if case["train"]:
            if case["kind"] == "qkn":
                out["d" + g] = dg
            out["d" + x] = torch.stack(dX)
    return out


def _exact_attn(case, st):
    B, Hq, Hk, nq, nk, d = (case[k] for k in ("B", "Hq", "Hk", "nq", "nk", "d"))
    dev, f64, G = st["Q"].device, torch.float64, Hq // Hk
    zeros = lambda h, n: torch.zeros(B, h, n, d, dtype=f64, device=dev)
    out = dict(O=zeros(Hq, nq), lse=torch.full((B, Hq, nq), -math.inf, dtype=f64, device=dev))
    if case["train"]:
        out |= dict(dQ=zeros(Hq, nq), dK=zeros(Hk, nk), dV=zeros(Hk, nk))
    for b in range(B):
        n = int(st["kv_len"][b]) if st["kv_len"] is not None else nk
        i, j = torch.arange(n - nq, n, device=dev)[:, None], torch.arange(n, device=dev)[None]
        hidden = torch.zeros(nq, n, dtype=torch.bool, device=dev)
        if case["causal"]:
            hidden |= j > i
            if st["prefix"] is not None:
                hidden &= j >= int(st["prefix"][b])
        if st["doc"] is not None:
            dq, dk = st["doc"][b, :, None], st["doc"][b, None, :n]
            hidden |= (dq != dk) | (dk < 0)
        live = ~hidden.all(1)
        for h in range(Hq):
            Q, K, V = st["Q"][b, h].to(f64), st["K"][b, h // G, :n].to(f64), st["V"][b, h // G, :n].to(f64)
            z = (Q @ K.T).mul_(st["scale"])
            slope = None
            if case["cap"]:
                z = z.div_(case["cap"]).tanh_()
                if case["train"]:
                    slope = 1 - z * z
                z = z.mul_(case["cap"])
            if case["bias"]:
                z -= float(st["slopes"][h]) * (i - j).abs()
            z.masked_fill_(hidden, -math.inf)
            L = torch.logsumexp(z, 1)
            out["lse"][b, h] = L
            A = torch.where(live[:, None], (z - L[:, None]).exp_(), 0.0)
            del z
            out["O"][b, h] = A @ V
            if case["train"]:
                D = st["dO"][b, h].to(f64)
                out["dV"][b, h // G, :n] += A.T @ D
                A *= D @ V.T - (D * out["O"][b, h]).sum(1, keepdim=True)
                if slope is not None:
                    A *= slope
                A *= st["scale"]
                out["dQ"][b, h] = A @ K
                out["dK"][b, h // G, :n] += A.T @ Q
    return out
