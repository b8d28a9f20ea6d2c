"""Attention over packed sequences from its definition in 64 bits, with the sizes
that arithmetic errors are measured by (test infrastructure)."""

import math

import torch

D = 128
SCALE = 1 / math.sqrt(D)


def visible(Lq, Lk, causal, device):
    see = torch.ones((Lq, Lk), dtype=torch.bool, device=device)
    return see.tril_(Lk - Lq) if causal else see


def attend(q, k, v, see):
    """One head: q [n, d], k, v [m, d] float64, see [n, m].
    Returns o, lse, P, the largest sum of |q k| / sqrt d of a visible key."""
    s = (q @ k.T) * SCALE
    s = s.masked_fill(~see, -math.inf)
    m = s.amax(1, keepdim=True).clamp_min(-1e30) if k.shape[0] else s.new_zeros((q.shape[0], 1))
    e = torch.exp(s - m)
    l = e.sum(1, keepdim=True)
    some = l > 0
    p = e / torch.where(some, l, 1.0)
    lse = torch.where(some, m + l.log(), -math.inf)[:, 0]
    size = (q.abs() @ k.abs().T * SCALE).masked_fill(~see, 0)
    size = size.amax(1) if k.shape[0] else lse.new_zeros(q.shape[0])
    return p @ v, lse, p, size


class Packed:
    """Results of packed sequences: o, lse, and the sums of weights times absolute
    values (a_o) and the largest score sizes (s_lse); with dout the gradients and the
    sizes of their terms."""

    def __init__(self, q, k, v, cu_q, cu_k, causal, dout=None):
        dev = q.device
        q, k, v = q.double(), k.double(), v.double()
        Hq, Hkv = q.shape[1], k.shape[1]
        G = Hq // Hkv
        self.o, self.a_o = torch.zeros_like(q), torch.zeros_like(q)
        self.lse = torch.full((Hq, q.shape[0]), -math.inf, dtype=torch.float64, device=dev)
        self.s_lse = torch.zeros_like(self.lse)
        if dout is not None:
            dout = dout.double()
            self.dq, self.dk, self.dv = (torch.zeros_like(t) for t in (q, k, v))
            self.a_dq, self.a_dk, self.a_dv = (torch.zeros_like(t) for t in (q, k, v))
        for a, b, x, y in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
            if b == a:
                continue
            see = visible(b - a, y - x, causal, dev)
            for h in range(Hq):
                g = h // G
                qs, ks, vs = q[a:b, h], k[x:y, g], v[x:y, g]
                o, lse, p, size = attend(qs, ks, vs, see)
                self.o[a:b, h], self.lse[h, a:b] = o, lse
                self.a_o[a:b, h], self.s_lse[h, a:b] = p @ vs.abs(), size
                if dout is None or y == x:
                    continue
                do = dout[a:b, h]
                dp = do @ vs.T
                big = do.abs() @ vs.abs().T
                row = (do * o).sum(1, keepdim=True)
                ds = p * (dp - row)
                # what errors of relative size e in P, dP, D make of dS: e times this
                ads = p * (big + (do.abs() * (p @ vs.abs())).sum(1, keepdim=True))
                self.dv[x:y, g] += p.T @ do
                self.a_dv[x:y, g] += p.T @ do.abs()
                self.dq[a:b, h] = ds @ ks * SCALE
                self.a_dq[a:b, h] = ads @ ks.abs() * SCALE
                self.dk[x:y, g] += ds.T @ qs * SCALE
                self.a_dk[x:y, g] += ads.T @ qs.abs() * SCALE


# Unit roundoffs.
BF16, FP32 = 2.0 ** -8, 2.0 ** -24


def score_error(size):
    """Error of a score: 128 fp32 products and sums of absolute size `size`, one
    scaling, the log2 e in front of the hardware's exp2 (good to 2 units itself)."""
    return (D + 4) * FP32 * size + 4 * FP32


def check(name, got, ref, bound):
    """|got - ref| <= bound everywhere; infinities where the reference has them."""
    got = got.double()
    same = torch.isinf(ref) & (got == ref)
    err = torch.where(same, 0.0, (got - ref).abs())
    ok = err <= bound
    worst = float((err / (bound + 1e-300)).max()) if err.numel() else 0.0
    print(f"  {name}: worst error / bound {worst:.3f}", flush=True)
    assert bool(ok.all()), (name, worst, int((~ok).sum()))


def check_forward(o, lse, ref, rows=slice(None)):
    """o: half a step of the result, and of every weight before its product with v, and
    the scores' error in the weights (twice: the weight and the sum it is divided by)."""
    es = score_error(ref.s_lse)
    w = BF16 + 2 * es.T[..., None] + 8 * FP32
    check("o", o[rows], ref.o[rows], (BF16 * ref.o.abs() + (1 + BF16) * w * ref.a_o)[rows] + 1e-30)
    fin = torch.where(torch.isinf(ref.lse), 0.0, ref.lse)
    check("lse", lse[:, rows], ref.lse[:, rows], (es + 4 * FP32 * fin.abs() + 8 * FP32)[:, rows])


def check_backward(dq, dk, dv, ref, rows_q=slice(None), rows_k=slice(None)):
    """Half a step of each result, and: dv has half a step of every weight and the
    weight's error (score, and lse, which has the score's error again); dS has that too, half
    a step of its own, and D's error, which is o's: half a step of o and of the weights that
    formed it.  All relative to the sums of absolute terms."""
    es = float(score_error(ref.s_lse.max())) if ref.s_lse.numel() else 0.0
    ep = 3 * es + 16 * FP32
    cv = BF16 + (1 + BF16) * ep
    cs = BF16 + ep + 2 * (BF16 + 2 * es + 8 * FP32) + 8 * BF16 * BF16 + (D + 8) * FP32
    for name, got, want, size, c, rows in (("dq", dq, ref.dq, ref.a_dq, cs, rows_q),
                                           ("dk", dk, ref.dk, ref.a_dk, cs, rows_k),
                                           ("dv", dv, ref.dv, ref.a_dv, cv, rows_k)):
        check(name, got[rows], want[rows],
              (BF16 * want.abs() + (1 + BF16) * c * size)[rows] + 1e-30)
