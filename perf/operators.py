"""The calls by which the operators over packed sequences, caches and normed
heads are measured, each beside its plain form.

A case is a dict of plain values with a ``kind``; lengths are texts of numbers:

  packed  causal attention over packed sequences, forward: sequence s has the
          s-th of the ``q`` queries and the s-th of the ``k`` keys, the queries
          being the last ones of the keys
  step    the same, forward and backward
  decode  ``nq`` new tokens of every sequence against its rows of a cache (the
          new ones among them), ``k`` rows of ``cap``
  prefix  the same behind ``P`` rows that all sequences share
  norm    RMS norm of every query and key head and the position rotation
  norm_bwd  its gradients, those of the weights among them

``prepare`` makes what a program holds before the call, ``run`` is one pass, and
``exact`` is the same result from the definition in 64 bits.
"""

import math

import torch

own = False
D = 128                   # head width, the only one the library builds
DEV = "cuda:0"
EPS = 1e-6


# ------------------------------------------------------------------- cases

def listed():
    return [
        # A few short prompts, one of a single token: launches and latency.
        dict(name="packed_chat", kind="packed", q="7 1 130 33 64", k="7 1 130 33 64", Hq=32, Hkv=8,
             causal=True),
        # Prompts served in pieces: the next queries of each behind what its cache holds.
        dict(name="packed_context_32k", kind="packed", q="2048 512 1 777 130 1024",
             k="32768 20000 9001 777 4226 16384", Hq=32, Hkv=8, causal=True),
        # A short training batch of documents of odd lengths on one GPU's share of heads.
        dict(name="step_docs_2k", kind="step", q="700 1 411 128 257 551", k="700 1 411 128 257 551",
             Hq=4, Hkv=1, causal=True),
        # A long-context training batch: one long document and what fills the row up.
        dict(name="step_docs_64k", kind="step", q="32768 8191 12000 513 4000 2 6000 2062",
             k="32768 8191 12000 513 4000 2 6000 2062", Hq=8, Hkv=1, causal=True),
        # One long conversation, one new token.
        dict(name="decode_one_128k", kind="decode", k="131071", cap=131072, nq=1, Hq=8, Hkv=1),
        # A serving batch of all heads, lengths from one row to a long cache.
        dict(name="decode_batch_24", kind="decode", cap=16384, nq=1, Hq=32, Hkv=8,
             k="1 16384 300 4097 8000 127 12345 2048 640 5555 9999 33 15000 7000 1025 256 3500 11111 "
               "90 6144 2500 800 4444 13000"),
        # Four drafted tokens of three answers to one question.
        dict(name="prefix_draft", kind="prefix", P=1000, k="4 150 61", cap=256, nq=4, Hq=8, Hkv=1),
        # Many answers to one long prompt, all heads.
        dict(name="prefix_batch_64", kind="prefix", P=16384, cap=1024, nq=1, Hq=64, Hkv=8,
             k=" ".join(str(1 + 37 * i * i % 1024) for i in range(64))),
        # The new tokens of a small serving batch, all heads of a wide model.
        dict(name="norm_tokens", kind="norm", T=8, Hq=64, Hkv=8, base=1000000.0, w32=False),
        # The queries and keys of a long training batch.
        dict(name="norm_64k", kind="norm", T=65536, Hq=32, Hkv=8, base=500000.0, w32=False),
        # A short batch of odd length, weights kept in fp32.
        dict(name="norm_bwd_1k", kind="norm_bwd", T=1001, Hq=32, Hkv=8, base=10000.0, w32=True),
        # A long training batch of all heads of a wide model.
        dict(name="norm_bwd_64k", kind="norm_bwd", T=65536, Hq=64, Hkv=8, base=1000000.0, w32=False),
    ]


def _log_int(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(lens):
    return " ".join(str(n) for n in lens)


def _lens(text):
    return [int(n) for n in text.split()]


def draw(rng):
    top = {w: max(work(c)[w] for c in listed()) for w in ("bytes", "flops")}
    while True:
        kind = rng.choice(["packed", "packed", "step", "step", "decode", "prefix", "norm", "norm_bwd"])
        Hkv = rng.choice([1, 1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 5, 8])
        c = dict(kind=kind, Hq=Hq, Hkv=Hkv)
        if kind in ("packed", "step"):
            q = [_log_int(rng, 1, 32768) for _ in range(_log_int(rng, 1, 40))]
            k = q
            if rng.random() < (0.5 if kind == "packed" else 0.2):
                # Most sequences have earlier keys, some have fewer keys than queries.
                k = [max(0, n + rng.choice([0, _log_int(rng, 1, 16384), -_log_int(rng, 1, n)]))
                     for n in q]
            c.update(q=_text(q), k=_text(k), causal=rng.random() < 0.8)
        elif kind in ("decode", "prefix"):
            cap = _log_int(rng, 16, 131072 if kind == "decode" else 4096)
            k = [_log_int(rng, 1, cap) for _ in range(_log_int(rng, 1, 96))]
            c.update(k=_text(k), cap=cap, nq=rng.choice([1, 1, 1, 2, 4, 7]))
            if kind == "prefix":
                c.update(P=_log_int(rng, 1, 32768))
            if len(k) * cap * Hkv * 4 * D > 1 << 33:
                continue
        else:
            c.update(T=_log_int(rng, 1, 131072), base=rng.choice([10000.0, 500000.0, 1000000.0]),
                     w32=rng.random() < 0.3)
        w = work(c)
        if w["bytes"] <= top["bytes"] and w["flops"] <= top["flops"]:
            return c


# -------------------------------------------------------------------- work

def _pairs(Lq, Lk, causal):
    """Visible (query, key) pairs of one head: query i sees Lk - Lq + i + 1 keys."""
    if not causal:
        return Lq * Lk
    n = min(Lq, Lk)              # queries that see any key
    return n * (Lk - n) + n * (n + 1) // 2


def work(c):
    """4 d per visible (query, key, head) triple forward, 2.5 times that
    backward; every valid row read once, every result written once."""
    Hq, Hkv = c["Hq"], c["Hkv"]
    row = 2 * D
    if c["kind"] in ("norm", "norm_bwd"):
        n = c["T"] * (Hq + Hkv)
        back = c["kind"] == "norm_bwd"
        weights = 2 * D * (4 if c["w32"] else 2)
        return {"bytes": n * row * (3 if back else 2) + 8 * c["T"] + weights * (2 if back else 1),
                "flops": n * D * (16 if back else 7)}
    k = _lens(c["k"])
    if c["kind"] in ("decode", "prefix"):
        nq, P, B = c["nq"], c.get("P", 0), len(k)
        pairs = sum(_pairs(nq, n, True) + nq * P for n in k)
        return {"bytes": Hkv * 2 * row * (sum(k) + P) + B * nq * Hq * (2 * row + 4) + 4 * B,
                "flops": 4 * D * Hq * pairs}
    q = _lens(c["q"])
    pairs = sum(_pairs(a, b, c["causal"]) for a, b in zip(q, k))
    heads_q, heads_k = sum(q) * Hq, sum(k) * Hkv
    if c["kind"] == "packed":
        return {"bytes": heads_q * (2 * row + 4) + heads_k * 2 * row, "flops": 4 * D * Hq * pairs}
    return {"bytes": heads_q * (4 * row + 4) + heads_k * 4 * row, "flops": 14 * D * Hq * pairs}


# ----------------------------------------------------------------- prepare

def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
        if x.numel():
            x.normal_(generator=g)
        return x

    Hq, Hkv, kind = c["Hq"], c["Hkv"], c["kind"]
    st = {"case": c}
    if kind in ("packed", "step"):
        q, k = _lens(c["q"]), _lens(c["k"])
        st["cu_q"], st["cu_k"] = _cu(q), _cu(k)
        if q == k:
            # one projection's rows: [Q heads | K heads | V heads]
            qkv = normal(sum(q), Hq + 2 * Hkv, D)
            st["q"], st["k"], st["v"] = qkv.split([Hq, Hkv, Hkv], 1)
        else:
            st["q"], kv = normal(sum(q), Hq, D), normal(sum(k), 2 * Hkv, D)
            st["k"], st["v"] = kv.split([Hkv, Hkv], 1)
        if kind == "step":
            st["dout"] = normal(sum(q), Hq, D)
        if own:
            from paper_2602_21196_amd import upipe
            st["plan"] = upipe.VarlenPlan(st["cu_q"], st["cu_k"], Hq=Hq, Hkv=Hkv,
                                          causal=c["causal"], device=DEV)
    elif kind in ("decode", "prefix"):
        k = _lens(c["k"])
        B = len(k)
        st["q"] = normal(B, c["nq"], Hq, D)
        st["k"], st["v"] = normal(B, c["cap"], Hkv, D), normal(B, c["cap"], Hkv, D)
        st["lens"] = torch.tensor(k, dtype=torch.int32, device=DEV)
        if kind == "prefix":
            st["kp"], st["vp"] = normal(c["P"], Hkv, D), normal(c["P"], Hkv, D)
    else:
        T = c["T"]
        qkv = normal(T, Hq + 2 * Hkv, D)
        st["q"], st["k"], _ = qkv.split([Hq, Hkv, Hkv], 1)
        wt = torch.float32 if c["w32"] else torch.bfloat16
        st["wq"], st["wk"] = ((1 + 0.1 * normal(D).float()).to(wt) for _ in range(2))
        # packed sequences: positions start anew at each
        cut = torch.randint(0, T, (max(1, T // 3000),), device=DEV, generator=g)
        start = torch.zeros(T, dtype=torch.int64, device=DEV)
        start[cut] = cut
        st["positions"] = torch.arange(T, device=DEV) - torch.cummax(start, 0).values
        if kind == "norm_bwd":
            st["dq"], st["dk"] = normal(T, Hq, D), normal(T, Hkv, D)
    return st


# ------------------------------------------------------------- plain forms

CHUNK = 1 << 28           # scores formed at a time


def _visible(i0, i1, Lq, Lk, causal):
    """Mask [i1 - i0, Lk] of what the queries i0.. see."""
    j = torch.arange(Lk, device=DEV)
    i = torch.arange(i0, i1, device=DEV)[:, None]
    return (j <= i + (Lk - Lq)) if causal else torch.ones_like(j <= i)


def _probs(q, k, see):
    """Probabilities and row log-sum-exps of q [Hkv, n, G, d] against k [Hkv, Lk, d]."""
    h, n, G, _ = q.shape
    s = torch.matmul(q.reshape(h, n * G, D), k.transpose(1, 2)) * (1 / math.sqrt(D))
    s = s.view(h, n, G, -1).masked_fill_(~see[None, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min_(-1e30)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    some = l > 0
    p = p.div_(torch.where(some, l, 1.0))
    return p, torch.where(some, m + l.log(), -math.inf).squeeze(-1)


def _packed_plain(st):
    c = st["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    G = Hq // Hkv
    cu_q, cu_k = st["cu_q"], st["cu_k"]
    back = "dout" in st
    q, k, v = st["q"], st["k"], st["v"]
    o = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((Hq, q.shape[0]), dtype=torch.float32, device=DEV)
    if back:
        dq = torch.empty_like(o)
        dk = torch.empty(k.shape, dtype=torch.bfloat16, device=DEV)
        dv = torch.empty_like(dk)
    for a, b, x, y in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        Lq, Lk = b - a, y - x
        if Lk == 0:
            o[a:b] = 0
            lse[:, a:b] = -math.inf
            if back:
                dq[a:b] = 0
            continue
        ks, vs = (t[x:y].float().transpose(0, 1).contiguous() for t in (k, v))
        if back:
            dks, dvs = torch.zeros_like(ks), torch.zeros_like(vs)
        step = max(1, CHUNK // (Hq * Lk))
        for i0 in range(0, Lq, step):
            i1 = min(Lq, i0 + step)
            n = i1 - i0
            see = _visible(i0, i1, Lq, Lk, c["causal"])
            qs = q[a + i0:a + i1].float().view(n, Hkv, G, D).transpose(0, 1)
            p, ls = _probs(qs, ks, see)
            p = p.view(Hkv, n * G, Lk)
            os = torch.matmul(p, vs)
            o[a + i0:a + i1] = os.view(Hkv, n, G, D).transpose(0, 1).reshape(n, Hq, D)
            lse[:, a + i0:a + i1] = ls.transpose(1, 2).reshape(Hq, n)
            if back:
                do = st["dout"][a + i0:a + i1].float().view(n, Hkv, G, D).transpose(0, 1)
                do = do.reshape(Hkv, n * G, D)
                dvs += torch.matmul(p.transpose(1, 2), do)
                ds = torch.matmul(do, vs.transpose(1, 2)).sub_((do * os).sum(-1, keepdim=True))
                ds = ds.mul_(p).mul_(1 / math.sqrt(D))
                dks += torch.matmul(ds.transpose(1, 2), qs.reshape(Hkv, n * G, D))
                dq[a + i0:a + i1] = torch.matmul(ds, ks).view(Hkv, n, G, D).transpose(0, 1).reshape(
                    n, Hq, D)
        if back:
            dk[x:y] = dks.transpose(0, 1)
            dv[x:y] = dvs.transpose(0, 1)
    return (o, lse, dq, dk, dv) if back else (o, lse)


def _decode_plain(st):
    q, lens = st["q"], st["lens"]
    B, nq, Hq, _ = q.shape
    Hkv = st["k"].shape[2]
    G = Hq // Hkv
    cap = st["k"].shape[1]
    P = st["kp"].shape[0] if "kp" in st else 0
    qs = q.float().view(B, nq, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B * Hkv, nq * G, D)
    k, v = (st[t].float().transpose(1, 2).reshape(B * Hkv, cap, D) for t in ("k", "v"))
    j = torch.arange(cap, device=DEV)
    t = torch.arange(nq, device=DEV)
    see = j < (lens[:, None, None] - (nq - 1) + t[:, None]).clamp_max(cap)          # [B, nq, cap]
    see = see[:, None, :, None, :].expand(B, Hkv, nq, G, cap).reshape(B * Hkv, nq * G, cap)
    s = torch.matmul(qs, k.transpose(1, 2)).masked_fill_(~see, -math.inf)
    if P:
        kp, vp = (st[t].float().transpose(0, 1) for t in ("kp", "vp"))              # [Hkv, P, d]
        rows = qs.view(B, Hkv, nq * G, D).transpose(0, 1).reshape(Hkv, B * nq * G, D)
        sp = torch.matmul(rows, kp.transpose(1, 2)).view(Hkv, B, nq * G, P).transpose(0, 1)
        s = torch.cat([s, sp.reshape(B * Hkv, nq * G, P)], -1)
    s = s * (1 / math.sqrt(D))
    m = s.amax(-1, keepdim=True).clamp_min(-1e30)
    e = (s - m).exp()
    l = e.sum(-1, keepdim=True)
    some = l > 0
    w = e / torch.where(some, l, 1.0)
    live = (j < lens[:, None])[:, None, :, None].expand(B, Hkv, cap, 1).reshape(B * Hkv, cap, 1)
    o = torch.matmul(w[..., :cap], torch.where(live, v, 0.0))
    if P:
        wp = w[..., cap:].reshape(B, Hkv, nq * G, P).transpose(0, 1).reshape(Hkv, B * nq * G, P)
        op = torch.matmul(wp, vp).view(Hkv, B, nq * G, D).transpose(0, 1)
        o = o + op.reshape(B * Hkv, nq * G, D)
    lse = torch.where(some, m + l.log(), -math.inf).view(B, Hkv, nq, G)
    o = o.view(B, Hkv, nq, G, D).permute(0, 2, 1, 3, 4).reshape(B, nq, Hq, D).bfloat16()
    return o, lse.permute(0, 1, 3, 2).reshape(B, Hq, nq).contiguous()


def _angles(st):
    e = torch.arange(D // 2, dtype=torch.float64, device=DEV)
    a = st["positions"].double()[:, None] * st["case"]["base"] ** (-2 * e / D)
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _norm_plain(st):
    cos, sin = _angles(st)
    out = []
    for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])):
        x = x.float()
        n = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float()
        a, b = n[..., :D // 2], n[..., D // 2:]
        out.append(torch.cat([a * cos - b * sin, b * cos + a * sin], -1).bfloat16())
    return tuple(out)


def _norm_bwd_plain(st):
    cos, sin = _angles(st)
    dxs, dws = [], []
    for x, w, dy in ((st["q"], st["wq"], st["dq"]), (st["k"], st["wk"], st["dk"])):
        a, b = dy[..., :D // 2].float(), dy[..., D // 2:].float()
        g = torch.cat([a * cos + b * sin, b * cos - a * sin], -1)
        x = x.float()
        r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        xr = x * r
        dws.append((g * xr).double().sum((0, 1)).to(w.dtype))
        g = g * w.float()
        dxs.append((r * (g - xr * (g * xr).mean(-1, keepdim=True))).bfloat16())
    return (*dxs, *dws)


# --------------------------------------------------------------------- run

def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"packed": _packed_plain, "step": _packed_plain, "decode": _decode_plain,
                "prefix": _decode_plain, "norm": _norm_plain, "norm_bwd": _norm_bwd_plain}[kind](st)
    from paper_2602_21196_amd import upipe
    base = st["case"].get("base")
    if kind == "packed":
        return upipe.attn_fwd_varlen(st["q"], st["k"], st["v"], st["plan"])
    if kind == "step":
        o, lse = upipe.attn_fwd_varlen(st["q"], st["k"], st["v"], st["plan"])
        return (o, lse, *upipe.attn_bwd_varlen(st["q"], st["k"], st["v"], o, lse, st["dout"],
                                               st["plan"]))
    if kind in ("decode", "prefix"):
        return upipe.attn_decode(st["q"], st["k"], st["v"], st["lens"], k_prefix=st.get("kp"),
                                 v_prefix=st.get("vp"))
    if kind == "norm":
        return upipe.qk_norm_rope(st["q"], st["k"], st["wq"], st["wk"], st["positions"], base,
                                  eps=EPS)
    return upipe.qk_norm_rope_bwd(st["q"], st["k"], st["wq"], st["wk"], st["positions"], base,
                                  st["dq"], st["dk"], eps=EPS)


# ------------------------------------------------------------------- exact

def _attend64(q, k, v, see):
    """softmax(q k^T / sqrt d) v of [n, d] rows, and the log-sum-exps; see [n, m]."""
    s = (q @ k.T / math.sqrt(D)).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
    return p @ v, lse


def _exact_packed(st):
    c = st["case"]
    G, cu_q, cu_k = c["Hq"] // c["Hkv"], st["cu_q"], st["cu_k"]
    leaves = [st[t].double() for t in ("q", "k", "v")]
    q, k, v = leaves
    back = "dout" in st
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.full((c["Hq"], q.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    grads = [torch.zeros_like(t) for t in leaves] if back else []
    for a, b, x, y in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        if a == b or x == y:
            continue
        see = torch.ones((b - a, y - x), dtype=torch.bool, device=DEV)
        first = a                  # rows before it see nothing
        if c["causal"]:
            see = see.tril_((y - x) - (b - a))
            first = max(a, b - (y - x))
        blk = max(1, (1 << 29) // (y - x))
        for h in range(c["Hq"]):
            for i in range(first, b, blk):
                e = min(b, i + blk)
                part = [t.detach().requires_grad_(back)
                        for t in (q[i:e, h], k[x:y, h // G], v[x:y, h // G])]
                oh, lh = _attend64(*part, see[i - a:e - a])
                o[i:e, h], lse[h, i:e] = oh.detach(), lh.detach()
                if back:
                    gq, gk, gv = torch.autograd.grad(oh, part, st["dout"][i:e, h].double())
                    grads[0][i:e, h] += gq
                    grads[1][x:y, h // G] += gk
                    grads[2][x:y, h // G] += gv
    return (o, lse, *grads)


def _exact_decode(st):
    q, lens = st["q"].double(), st["lens"].tolist()
    B, nq, Hq, _ = q.shape
    G = Hq // st["k"].shape[2]
    P = st["kp"].shape[0] if "kp" in st else 0
    o = torch.zeros_like(q)
    lse = torch.full((B, Hq, nq), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        see = torch.ones((nq, P + n), dtype=torch.bool, device=DEV).tril_(P + n - nq)
        see[:, :P] = True
        for g in range(Hq // G):
            k, v = st["k"][b, :n, g].double(), st["v"][b, :n, g].double()
            if P:
                k = torch.cat([st["kp"][:, g].double(), k])
                v = torch.cat([st["vp"][:, g].double(), v])
            for h in range(g * G, g * G + G):
                o[b, :, h], lse[b, h] = _attend64(q[b, :, h], k, v, see)
    return o, lse


def _rotation64(st):
    theta = [st["case"]["base"] ** (-i / (D // 2)) for i in range(D // 2)]
    turn = torch.outer(st["positions"].double(), torch.tensor(theta, dtype=torch.float64, device=DEV))
    return torch.polar(torch.ones_like(turn), turn)[:, None]


def _exact_norm(st):
    rot = _rotation64(st)
    back = "dq" in st
    ys, dxs, dws = [], [], []
    for t in "qk":
        x = st[t].double().requires_grad_(back)
        w = st["w" + t].double().requires_grad_(back)
        n = w * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS)
        z = torch.complex(n[..., :D // 2], n[..., D // 2:]) * rot
        y = torch.cat([z.real, z.imag], -1)
        if back:
            dx, dw = torch.autograd.grad(y, (x, w), st["d" + t].double())
            dxs.append(dx)
            dws.append(dw)
        else:
            ys.append(y)
    return (*dxs, *dws) if back else tuple(ys)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("packed", "step"):
        return _exact_packed(st)
    return _exact_decode(st) if kind in ("decode", "prefix") else _exact_norm(st)
