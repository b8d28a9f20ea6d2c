"""The packed calls together, as a model's block uses them: projection, norm of the heads
with their rotation, attention over packed sequences, output projection, and back; then
new tokens one by one from the caches that the prompts filled.

Against the same in 64 bits by torch's autograd, to the bar of the attention block's own
tests (tol.py): relative Frobenius norm 1e-2, of which every bf16 tensor between two
calls takes up to 2^-9 / sqrt(3) on average."""

import pytest
import torch

from paper_2602_21196_amd import upipe
from tol import REL_FROB

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, BASE, EPS = 128, 1e4, 1e-6


def _normal(shape, seed, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (std * torch.randn(shape, generator=g, device=DEV)).bfloat16()


def _norm_rope64(x, w, pos):
    n = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w
    e = torch.arange(D // 2, dtype=torch.float64, device=DEV)
    a = pos.double()[:, None, None] * BASE ** (-2 * e / D)
    u, v = n[..., :D // 2], n[..., D // 2:]
    return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], -1)


def _attend64(q, k, v, cu):
    out, G = [], q.shape[1] // k.shape[1]
    for a, b in zip(cu, cu[1:]):
        n = b - a
        see = torch.ones((n, n), dtype=torch.bool, device=DEV).tril()
        kk, vv = (t[a:b].repeat_interleave(G, 1).transpose(0, 1) for t in (k, v))
        s = q[a:b].transpose(0, 1) @ kk.transpose(1, 2) / D ** 0.5
        out.append((s.masked_fill(~see, -torch.inf).softmax(-1) @ vv).transpose(0, 1))
    return torch.cat(out)


def _rel(name, got, want):
    rel = float((got.double() - want).norm() / want.norm())
    print(f"  {name}: relative {rel:.2e}", flush=True)
    assert rel <= REL_FROB, (name, rel)


@pytest.mark.parametrize("lens,Hq,Hkv", [([100, 1, 155], 4, 2), ([384], 8, 1), ([60, 324], 3, 3)])
def test_block_forward_and_backward(lens, Hq, Hkv):
    T, dm = sum(lens), 256
    assert T % 128 == 0                      # the projection's rows
    cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
    pos = torch.cat([torch.arange(n) for n in lens]).to(DEV)
    heads = Hq + 2 * Hkv
    x, dy = _normal((T, dm), 1), _normal((T, dm), 2)
    wqkv, wo = _normal((dm, heads * D), 3, 0.06), _normal((Hq * D, dm), 4, 0.04)
    wq, wk = ((1 + 0.2 * _normal((D,), s).float()) for s in (5, 6))
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)

    qkv = upipe.gemm(x, wqkv).view(T, heads, D)
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    qn, kn = upipe.qk_norm_rope(q, k, wq, wk, pos, BASE, EPS)
    o, lse = upipe.attn_fwd_varlen(qn, kn, v, plan)
    y = upipe.gemm(o.view(T, Hq * D), wo)
    do = upipe.gemm(dy, wo.t().contiguous()).view(T, Hq, D)
    dqkv = torch.empty_like(qkv)             # gradients side by side, as the projection's
    dq, dk, dv = dqkv.split([Hq, Hkv, Hkv], 1)
    upipe.attn_bwd_varlen(qn, kn, v, o, lse, do, plan, out=(dq, dk, dv))
    *_, dwq, dwk = upipe.qk_norm_rope_bwd(q, k, wq, wk, pos, BASE, dq, dk, EPS, out=(dq, dk))
    flat = dqkv.view(T, heads * D)
    dx = upipe.gemm(flat, wqkv.t().contiguous())
    dwqkv = upipe.gemm(x.t().contiguous(), flat)
    dwo = upipe.gemm(o.view(T, Hq * D).t().contiguous(), dy)
    torch.cuda.synchronize()

    leaves = [t.double().requires_grad_() for t in (x, wqkv, wo, wq, wk)]
    x64, wqkv64, wo64, wq64, wk64 = leaves
    q64, k64, v64 = (x64 @ wqkv64).view(T, heads, D).split([Hq, Hkv, Hkv], 1)
    o64 = _attend64(_norm_rope64(q64, wq64, pos), _norm_rope64(k64, wk64, pos), v64, cu)
    y64 = o64.reshape(T, Hq * D) @ wo64
    grads = torch.autograd.grad(y64, leaves, dy.double())
    _rel("y", y, y64.detach())
    for name, a, b in zip(("dx", "dwqkv", "dwo", "dwq", "dwk"), (dx, dwqkv, dwo, dwq, dwk), grads):
        _rel(name, a, b)


def test_prompts_then_tokens():
    """Prompts packed into the caches' first rows, then three tokens each: every token's
    output is the row of a whole pass over the longer sequences."""
    lens, new, Hq, Hkv, cap = [130, 7, 260], 3, 8, 2, 300
    B, total = len(lens), [n + new for n in lens]
    pos = [torch.arange(n, device=DEV) for n in total]
    raw = [_normal((n, Hq + 2 * Hkv, D), 10 + i) for i, n in enumerate(total)]
    wq, wk = ((1 + 0.2 * _normal((D,), s).float()).bfloat16() for s in (5, 6))
    kc = torch.full((B, cap, Hkv, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    vc = kc.clone()
    cu = [sum(lens[:i]) for i in range(B + 1)]
    flat = torch.cat([r[:n] for r, n in zip(raw, lens)])
    q, k, v = flat.split([Hq, Hkv, Hkv], 1)
    at = torch.cat([p[:n] for p, n in zip(pos, lens)])
    qn, kn = upipe.qk_norm_rope(q, k, wq, wk, at, BASE, EPS)
    o, _ = upipe.attn_fwd_varlen(qn, kn, v, upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV))
    for b, n in enumerate(lens):
        kc[b, :n], vc[b, :n] = kn[cu[b]:cu[b + 1]], v[cu[b]:cu[b + 1]]
    outs = [[o[cu[b]:cu[b + 1]]] for b in range(B)]
    which = torch.arange(B, device=DEV)
    for t in range(new):
        tok = torch.stack([raw[b][lens[b] + t] for b in range(B)])
        here = torch.tensor([n + t for n in lens], device=DEV)
        q, k, v = tok.split([Hq, Hkv, Hkv], 1)
        qn, kn = upipe.qk_norm_rope(q, k, wq, wk, here, BASE, EPS)
        kc[which, here], vc[which, here] = kn, v
        o, _ = upipe.attn_decode(qn[:, None], kc, vc, (here + 1).int())
        for b in range(B):
            outs[b].append(o[b])
    torch.cuda.synchronize()
    for b, n in enumerate(total):
        q64, k64, v64 = raw[b].double().split([Hq, Hkv, Hkv], 1)
        want = _attend64(_norm_rope64(q64, wq.double(), pos[b]),
                         _norm_rope64(k64, wk.double(), pos[b]), v64, [0, n])
        _rel(f"sequence {b}", torch.cat(outs[b]), want)
        _rel(f"sequence {b}, new tokens", torch.cat(outs[b][1:]), want[lens[b]:])
