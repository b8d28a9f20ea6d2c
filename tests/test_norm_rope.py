"""The norm of query and key heads with the rotation behind it, and its
gradients, against the formulas in 64 bits.

Tolerances.  A bf16 result is off by half a step, 2^-8 of its value; an fp32 one by
2^-24.  Before that stand fp32 arithmetic and the angle: sines and cosines are good to
2e-5 of the pair's norm (the bound of the rotation's own tests), which also covers
the norm's 128 fp32 products and sums (130 x 2^-24 = 8e-6) by itself, so y gets both,
3e-5.  dx = r (a - n mean(a n)) has the angle in a and in the mean: twice that.  dw sums
N rows in fp32 pieces of at most 2^12 + 8 additions and the pieces in fp64: (3e-5 +
2^-11) of the sum of absolute values."""

import numpy as np
import pytest
import torch

from paper_2602_21196_amd import upipe

DEV = "cuda:0"
D = 128
ARITH = 3e-5


def _inputs(T, Hq, Hkv, seed, w32=False, scale=1.0, big=False):
    g = torch.Generator().manual_seed(seed)
    qkv = (scale * torch.randn((T, Hq + 2 * Hkv, D), generator=g)).bfloat16()
    dy = torch.randn((T, Hq + 2 * Hkv, D), generator=g).bfloat16()
    wt = torch.float32 if w32 else torch.bfloat16
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(wt) for _ in range(2))
    pos = torch.randint(0, (1 << 32) - 1 if big else 5000, (T,), generator=g)
    return qkv, dy, wq, wk, pos


def _turns(pos, base):
    e = np.arange(D // 2)
    a = pos.numpy().astype(np.float64)[:, None] * base ** (-2.0 * e / D)
    return np.cos(a)[:, None], np.sin(a)[:, None]


def _rotate(x, c, s):
    a, b = x[..., :64], x[..., 64:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def _pair(x):
    n = np.sqrt(x[..., :64] ** 2 + x[..., 64:] ** 2)
    return np.concatenate([n, n], -1)


def _f64(t):
    return t.detach().cpu().double().numpy()


def _fwd64(x, w, pos, base, eps):
    x, w = _f64(x), _f64(w)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r * w
    return _rotate(n, *_turns(pos, base)), _pair(n)


def _bwd64(x, w, pos, base, eps, dy):
    """dx, dw and what their arithmetic errors are measured by."""
    x, w, dy = _f64(x), _f64(w), _f64(dy)
    c, s = _turns(pos, base)
    g = _rotate(dy, c, -s)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, a, ga = x * r, g * w, _pair(g)
    dx = r * (a - n * (a * n).mean(-1, keepdims=True))
    dx_size = r * (ga * np.abs(w) + np.abs(n) * (ga * np.abs(w * n)).mean(-1, keepdims=True))
    return dx, (g * n).sum((0, 1)), dx_size, (ga * np.abs(n)).sum((0, 1))


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _check(name, got, ref, size, arith):
    err = np.abs(_f64(got) - ref)
    bound = _half(got.dtype) * np.abs(ref) * (1 + arith) + arith * size + 1e-30
    worst = float((err / bound).max()) if err.size else 0.0
    print(f"  {name}: worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0, (name, worst)


CASES = [  # T, Hq, Hkv, fp32 weights, base, eps, scale, large positions
    (1, 1, 1, False, 1e4, 1e-6, 1.0, False),
    (1, 64, 8, False, 1e6, 1e-6, 1.0, False),
    (7, 3, 5, True, 5e5, 1e-5, 30.0, True),
    (33, 5, 1, False, 1e4, 1e-6, 1e-3, True),
    (1001, 32, 8, True, 1e4, 1e-6, 1.0, False),
    (4099, 8, 2, False, 1e6, 1e-6, 2.0, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,Hq,Hkv,w32,base,eps,scale,big", CASES)
def test_matches_the_formulas(T, Hq, Hkv, w32, base, eps, scale, big):
    print(f"norm T={T} Hq={Hq} Hkv={Hkv} w32={w32} base={base} big={big}", flush=True)
    qkv, dy, wq, wk, pos = _inputs(T, Hq, Hkv, T + Hq, w32, scale, big)
    qd, kd, vd = qkv.to(DEV).split([Hq, Hkv, Hkv], 1)
    dqd, dkd, _ = dy.to(DEV).split([Hq, Hkv, Hkv], 1)
    wqd, wkd, pd = wq.to(DEV), wk.to(DEV), pos.to(DEV)
    before = vd.clone()
    y = upipe.qk_norm_rope(qd, kd, wqd, wkd, pd, base, eps)
    back = upipe.qk_norm_rope_bwd(qd, kd, wqd, wkd, pd, base, dqd, dkd, eps)
    # In place: forward on a copy, backward over the upstream gradients.
    buf, grad = qd._base.clone(), dqd._base.clone()
    bq, bk, bv = buf.split([Hq, Hkv, Hkv], 1)
    gq, gk, gv = grad.split([Hq, Hkv, Hkv], 1)
    upipe.qk_norm_rope(bq, bk, wqd, wkd, pd, base, eps, out=(bq, bk))
    again = upipe.qk_norm_rope_bwd(qd, kd, wqd, wkd, pd, base, gq, gk, eps, out=(gq, gk))
    torch.cuda.synchronize()
    assert torch.equal(bq, y[0]) and torch.equal(bk, y[1]) and torch.equal(bv, before)
    for a, b in zip(again, back):
        assert torch.equal(a, b)
    assert torch.equal(gv, dy.to(DEV)[:, Hq + Hkv:])
    for i, (x, w, d) in enumerate(((qd, wq, dqd), (kd, wk, dkd))):
        ref, size = _fwd64(x, w, pos, base, eps)
        _check("qk"[i] + "'", y[i], ref, size, ARITH)
        dx, dw, dx_size, dw_size = _bwd64(x, w, pos, base, eps, d)
        _check("d" + "qk"[i], back[i], dx, dx_size, 2 * ARITH)
        _check("dw" + "qk"[i], back[2 + i], dw, dw_size, ARITH + 2.0 ** -11)


@pytest.mark.gpu
def test_gradients_match_differences():
    """The formulas' gradients are those of the forward: central differences of the
    64-bit forward (error h^2 ~ 1e-8 of values of order 1) against the kernel, whose bf16
    results are off by 2^-8."""
    T, H, base, eps, h = 3, 2, 1e4, 1e-6, 1e-4
    qkv, dy, wq, wk, pos = _inputs(T, H, H, 5, True)
    q, d = qkv[:, :H], dy[:, :H]
    dev = [t.to(DEV) for t in (qkv, dy, wq, wk, pos)]
    got = upipe.qk_norm_rope_bwd(dev[0][:, :H], dev[0][:, H:2 * H], dev[2], dev[3], dev[4], base,
                                 dev[1][:, :H], dev[1][:, H:2 * H], eps)
    x, w = q.double(), wq.double()

    def loss(x, w):
        return float((_fwd64(x, w, pos, base, eps)[0] * _f64(d)).sum())
    for at in ((0, 0, 0), (1, 1, 63), (2, 0, 64), (0, 1, 127)):
        step = torch.zeros_like(x)
        step[at] = h
        diff = (loss(x + step, w) - loss(x - step, w)) / (2 * h)
        assert abs(float(got[0][at]) - diff) <= 2.0 ** -8 * abs(diff) + 1e-3 * 1.0, at
    for e in (0, 64, 127):
        step = torch.zeros_like(w)
        step[e] = h
        diff = (loss(x, w + step) - loss(x, w - step)) / (2 * h)
        assert abs(float(got[2][e]) - diff) <= 1e-4 * (1 + abs(diff)), e


@pytest.mark.gpu
def test_zero_rows_no_rows_and_other_values():
    qkv, dy, wq, wk, pos = (t.to(DEV) for t in _inputs(4, 2, 1, 9))
    q, k = qkv[:, :2], qkv[:, 2:3]
    q[1] = 0
    q[2, 0, 5] = float("nan")
    y, _ = upipe.qk_norm_rope(q, k, wq, wk, pos, 1e4)
    dq, _, dwq, dwk = upipe.qk_norm_rope_bwd(q, k, wq, wk, pos, 1e4, dy[:, :2], dy[:, 2:3])
    assert bool((y[1] == 0).all())
    # a row that is not a number spoils itself only (and the sum over rows)
    assert bool(y[2, 0].isnan().all()) and not bool(y[[0, 1, 3]].isnan().any())
    assert not bool(y[2, 1].isnan().any()) and not bool(dq[[0, 1, 3]].isnan().any())
    assert not bool(dwk.isnan().any())
    # no rows: nothing to write, weights get zeros
    e = torch.empty((0, 2, D), dtype=torch.bfloat16, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert upipe.qk_norm_rope(e, e, wq, wk, none, 1e4)[0].shape == (0, 2, D)
    back = upipe.qk_norm_rope_bwd(e, e, wq, wk, none, 1e4, e, e)
    assert bool((back[2] == 0).all()) and bool((back[3] == 0).all())


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    qkv, dy, wq, wk, pos = (t.to(DEV) for t in _inputs(517, 4, 2, 11))
    q, k = qkv[:, :4], qkv[:, 4:6]
    gq, gk = dy[:, :4], dy[:, 4:6]
    ws = upipe.workspace(upipe.upipe_qk_norm_rope_bwd_workspace_size(517, 4, 2, D), DEV)

    def both():
        return (*upipe.qk_norm_rope(q, k, wq, wk, pos, 1e4),
                *upipe.qk_norm_rope_bwd(q, k, wq, wk, pos, 1e4, gq, gk, ws=ws))
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for n in range(3):
        qkv.mul_(2 ** n)            # new inputs in place: the graph has to read them
        want_n = both()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want_n):
            assert torch.equal(a, b)
        if n == 0:
            for a, b, c in zip(want, other, want_n):
                assert torch.equal(a, b) and torch.equal(a, c)


FAKE = 1 << 20


def _heads(p=FAKE, row=4 * D, head=D):
    return upipe.upipe_heads(p, row, head)


def _fwd(**kw):
    a = dict(q=_heads(), k=_heads(2 * FAKE, D), wq=FAKE, wk=FAKE, w32=0, pos=FAKE,
             q_out=_heads(3 * FAKE), k_out=_heads(4 * FAKE, D), T=100, Hq=4, Hkv=1, d=D, base=1e4,
             eps=0.0, stream=None)       # eps = 0 is refused: no call here may launch
    a.update(kw)
    return upipe.upipe_qk_norm_rope(*a.values())


def _bwd(**kw):
    a = dict(q=_heads(), k=_heads(2 * FAKE, D), wq=FAKE, wk=FAKE, w32=0, pos=FAKE,
             dq_out=_heads(3 * FAKE), dk_out=_heads(4 * FAKE, D), dq=_heads(5 * FAKE),
             dk=_heads(6 * FAKE, D), dwq=FAKE, dwk=FAKE, T=100, Hq=4, Hkv=1, d=D, base=1e4,
             eps=1e-6, ws=FAKE, ws_bytes=15, stream=None)      # no workspace
    a.update(kw)
    return upipe.upipe_qk_norm_rope_bwd(*a.values())


@pytest.mark.parametrize("fn", [_fwd, _bwd])
def test_refusals(fn):
    INV, UNS, WS = -1, -2, -3
    assert fn() == (INV if fn is _fwd else WS)
    assert fn(T=-1) == INV and fn(Hq=0) == INV and fn(Hkv=0) == INV
    assert fn(d=64) == UNS and fn(Hq=65) == UNS and fn(T=1 << 31) == UNS
    for bad in (dict(w32=2), dict(base=0.0), dict(base=float("inf")), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=1e-60), dict(wq=None), dict(wk=FAKE + 2),
                dict(pos=None), dict(q=_heads(0)), dict(q=_heads(FAKE + 8)), dict(k=_heads(row=12)),
                dict(k=_heads(head=-8)), dict(q=_heads(row=1 << 60))):
        assert fn(**bad) == INV, bad


def test_refusals_of_the_backward():
    for bad in (dict(dwq=None), dict(ws=None), dict(dq=_heads(5 * FAKE, row=0)),
                dict(dk=_heads(5 * FAKE, D)),                  # over dq
                dict(dq=_heads(FAKE + 16)),                    # beside q, not on it
                dict(dk=_heads(3 * FAKE, D)), dict(T=0, w32=3)):
        assert _bwd(**bad) == -1, bad
    # columns of one buffer, or each on its own input
    row = 6 * D
    views = [_heads(FAKE, row), _heads(FAKE + 4 * 256, row)]
    assert _bwd(q=views[0], k=views[1], dq=views[0], dk=views[1]) == -3
    assert _bwd(q=views[0], k=views[1], dq=views[1], dk=views[0]) == -1
    # keys beside values in every head
    pair = [_heads(7 * FAKE, 2 * D, 2 * D), _heads(7 * FAKE + 256, 2 * D, 2 * D)]
    assert _bwd(dq=pair[0], dk=pair[1], Hq=1) == -3
    assert upipe.upipe_qk_norm_rope_bwd_workspace_size(-1, 4, 1, D) == 0
    assert upipe.upipe_qk_norm_rope_bwd_workspace_size(0, 4, 1, D) > 0


def test_binding_refuses_before_the_library_is_called():
    cpu = torch.zeros((4, 2, D), dtype=torch.bfloat16)
    w, pos = torch.ones(D), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        upipe.qk_norm_rope(cpu, cpu, w, w, pos, 1e4)
    with pytest.raises(TypeError):
        upipe.qk_norm_rope(cpu.float(), cpu, w, w, pos, 1e4)
