"""The gradients of attention over packed sequences, against their definition in 64
bits (bounds in varlen_ref.py) and against differences, and what the call refuses."""

import pytest
import torch

import varlen_ref as R
from paper_2602_21196_amd import upipe
from test_varlen import CASES, _cu, _layouts, _normal

DEV = "cuda:0"
D = 128


def _step(q, k, v, dout, plan, **kw):
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    return (o, lse, *upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan, **kw))


MORE = [
    ([300, 1200, 64], None, 8, 1, True),            # walks in segments
    ([5000], None, 2, 1, True),
    ([70, 200], [6000, 100], 4, 2, True),
    ([3000, 10], [2000, 4000], 33, 1, False),       # 99 of 128 rows a tile
    ([130, 140], None, 48, 1, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CASES) + len(MORE)))
def test_gradients_match_the_definition(i):
    lq, lk, Hq, Hkv, causal = (CASES + MORE)[i]
    cu_q, cu_k = _cu(lq), _cu(lk or lq)
    print(f"varlen step {lq} {lk} {Hq}/{Hkv} causal={causal}", flush=True)
    q, k, v, dout = (_normal((n, H, D), 100 * i + j) for j, (n, H) in enumerate(
        ((cu_q[-1], Hq), (cu_k[-1], Hkv), (cu_k[-1], Hkv), (cu_q[-1], Hq))))
    plan = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=Hkv, causal=causal, device=DEV)
    o, lse, dq, dk, dv = _step(q, k, v, dout, plan)
    again = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan)
    torch.cuda.synchronize()
    ref = R.Packed(q, k, v, cu_q, cu_k, causal, dout)
    R.check_backward(dq, dk, dv, ref)
    for a, b in zip((dq, dk, dv), again):
        assert torch.equal(a, b)
    if sum(lq) >= 64 and causal and lk is None:     # the bar of the other backward's tests
        for n, a, b in (("dq", dq, ref.dq), ("dk", dk, ref.dk), ("dv", dv, ref.dv)):
            rel = float((a.double() - b).norm() / b.norm())
            print(f"  {n}: relative {rel:.2e}", flush=True)
            assert rel <= 1e-2, (n, rel)


@pytest.mark.gpu
def test_layouts_places_and_rows_behind_the_last():
    lens, Hq, Hkv = [200, 3, 411], 6, 2
    cu, n, pad = _cu(lens), 614, 9
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    want = None
    for name, q, k, v in _layouts(n + pad, Hq, Hkv, 78):
        print("layout", name, flush=True)
        dout = _normal((n + pad, Hq, D), 9)
        for t in (q, k, v, dout):
            t[n:] = float("nan")
        if name == "head-major":
            dout = dout.transpose(0, 1).contiguous().transpose(0, 1)
        o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
        buf = _normal((n + pad, Hq + 2 * Hkv, D), 6)
        keep = buf.clone()
        dq, dk, dv = buf.split([Hq, Hkv, Hkv], 1)
        upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan, out=(dq, dk, dv))
        torch.cuda.synchronize()
        assert torch.equal(buf[n:], keep[n:])
        if want is None:
            want = buf[:n].clone()
            R.check_backward(dq[:n], dk[:n], dv[:n],
                             R.Packed(q[:n], k[:n], v[:n], cu, cu, True, dout[:n]))
        assert torch.equal(buf[:n], want)
        new = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan)
        assert all(bool((t[n:] == 0).all()) for t in new)
        # what the workspace held before does not matter
        ws = upipe.workspace(plan.bwd_workspace, DEV).fill_(255)
        again = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(torch.cat(again, 1)[:n], want)


@pytest.mark.gpu
def test_gradients_match_differences():
    """Central differences of the 64-bit definition (error h^2 ~ 1e-8) along one direction
    of q, k and v each, against the kernel's gradient in that direction, off by its
    elements' bounds."""
    lens, Hq, Hkv, h = [40, 9, 130], 4, 2, 1e-4
    cu = _cu(lens)
    n = cu[-1]
    x = [_normal((n, H, D), j) for j, H in enumerate((Hq, Hkv, Hkv))]
    dout = _normal((n, Hq, D), 7)
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    grads = _step(*x, dout, plan)[2:]
    ref = R.Packed(*x, cu, cu, True, dout)
    g = torch.Generator(device=DEV).manual_seed(3)
    for i, (got, size) in enumerate(zip(grads, (ref.a_dq, ref.a_dk, ref.a_dv))):
        way = torch.empty(x[i].shape, dtype=torch.float64, device=DEV).normal_(generator=g)
        loss = []
        for s in (h, -h):
            at = [t.double() for t in x]
            at[i] = at[i] + s * way
            loss.append(float((R.Packed(*at, cu, cu, True).o * dout.double()).sum()))
        diff = (loss[0] - loss[1]) / (2 * h)
        mine = float((got.double() * way).sum())
        # independent roundings of relative 2^-8 add like their squares; 6 deviations
        off = 6 * 3.2 * R.BF16 * float(((size * way) ** 2).sum().sqrt()) + 1e-6 * abs(diff)
        print(f"  {'qkv'[i]}: {mine:.5f} by differences {diff:.5f}, allowed {off:.5f}", flush=True)
        assert abs(mine - diff) <= off


@pytest.mark.gpu
def test_sequences_do_not_reach_each_other():
    """Whatever the other sequences hold, one keeps its gradients' bits."""
    lens, Hq, Hkv = [100, 333, 17], 4, 1
    cu = _cu(lens)
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    x = [_normal((cu[-1], H, D), j) for j, H in enumerate((Hq, Hkv, Hkv, Hq))]
    want = _step(*x, plan)
    for t in x:
        t[100:433] = float("nan")
    got = _step(*x, plan)
    torch.cuda.synchronize()
    keep = torch.ones(cu[-1], dtype=torch.bool, device=DEV)
    keep[100:433] = False
    for i, (a, b) in enumerate(zip(got, want)):
        if i == 1:
            assert torch.equal(a[:, keep], b[:, keep])
        else:
            assert torch.equal(a[keep], b[keep])


@pytest.mark.gpu
def test_captured_step_and_shared_plan():
    """A captured step replays on new inputs; another stream's step with the same plan has
    its own workspace."""
    lens, Hq, Hkv = [257, 64, 1, 900], 8, 1
    cu = _cu(lens)
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    x = [_normal((cu[-1], H, D), j) for j, H in enumerate((Hq, Hkv, Hkv, Hq))]
    want = _step(*x, plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _step(*x, plan)
    more = _step(*x, plan)
    torch.cuda.synchronize()
    for a, b, c in zip(want, other, more):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _step(*x, plan)
    for n in range(3):
        x[0].mul_(0.7 ** n)
        want = _step(*x, plan)
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)


# ------------------------------------------------------------- no GPU needed

FAKE = 1 << 30


def _heads(p=FAKE, row=4 * D, head=D):
    return upipe.upipe_heads(p, row, head)


def test_refusals():
    plan = upipe.VarlenPlan([0, 700, 800], Hq=4, Hkv=1, device="cpu")

    def bwd(**kw):
        a = dict(q=_heads(), k=_heads(2 * FAKE, D), v=_heads(3 * FAKE, D), o=_heads(4 * FAKE),
                 lse=FAKE, lse_head=800, dout=_heads(5 * FAKE), dq=_heads(6 * FAKE),
                 dk=_heads(7 * FAKE, D), dv=_heads(8 * FAKE, D), plan=plan.host, dev=FAKE, ws=FAKE,
                 n=0, stream=None)
        a.update(kw)
        return upipe.upipe_attn_bwd_varlen(*a.values())
    INV, UNS, WS = -1, -2, -3
    assert bwd() == WS
    for bad in (dict(plan=None), dict(dev=None), dict(lse=None), dict(ws=None), dict(lse_head=799),
                dict(q=_heads(0)), dict(o=_heads(4 * FAKE + 2)), dict(dout=_heads(5 * FAKE, 12)),
                dict(dq=_heads(6 * FAKE, head=0)), dict(dk=_heads(7 * FAKE, 64)), dict(dv=_heads(0)),
                dict(dq=_heads(4 * FAKE)), dict(dq=_heads(2 * FAKE)), dict(dk=_heads(2 * FAKE, D)),
                dict(dv=_heads(FAKE, D)), dict(dk=_heads(6 * FAKE, D)), dict(dv=_heads(7 * FAKE, D)),
                dict(dq=_heads(5 * FAKE + 256)), dict(dq=_heads()), dict(dq=_heads(5 * FAKE))):
        assert bwd(**bad) == INV, bad
    assert bwd(k=_heads(1 << 44, (1 << 22) + 8)) == UNS
    assert bwd(q=_heads(1 << 44, 1 << 23)) == UNS
    assert bwd(dout=_heads(1 << 44, D, 1 << 28)) == UNS
    # columns of one buffer
    row = 6 * D
    assert bwd(dq=_heads(6 * FAKE, row), dk=_heads(6 * FAKE + 1024, row),
               dv=_heads(6 * FAKE + 1280, row)) == WS
    assert upipe.upipe_attn_bwd_varlen_workspace_size(None) == 0
    none = upipe.VarlenPlan([0], Hq=4, Hkv=1, device="cpu")
    assert bwd(plan=none.host, ws=None, lse=None, q=_heads(0)) == 0
