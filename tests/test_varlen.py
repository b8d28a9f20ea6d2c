"""Attention over packed sequences of different lengths, forward, against its
definition in 64 bits (bounds in varlen_ref.py), and what the calls refuse."""

import ctypes
import random

import pytest
import torch

import varlen_ref as R
from paper_2602_21196_amd import upipe

DEV = "cuda:0"
D = 128


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _normal(shape, seed, dev=DEV):
    g = torch.Generator(device=dev).manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=g)


CASES = [  # query lengths, key lengths (None: the same), Hq, Hkv, causal
    ([1], None, 1, 1, True),
    ([1], [1], 64, 1, True),
    ([5], [3], 4, 2, True),                         # rows that see nothing
    ([0, 7, 0, 0, 130, 1, 0], None, 4, 1, True),
    ([3, 0, 64], [0, 5, 0], 6, 2, True),            # no keys, no queries
    ([9], [0], 2, 1, True),                         # no keys at all
    ([0, 0], [3, 140], 4, 2, False),                # no queries at all
    ([31, 32, 33, 127, 128, 129, 255, 256, 257], None, 8, 2, True),
    ([31, 32, 33, 127, 128, 129, 255, 256, 257], None, 6, 2, False),
    ([700, 1, 411, 128, 257, 551], None, 4, 1, True),
    ([100, 1, 17], [1000, 777, 4000], 10, 2, True),  # behind a cache
    ([100, 1, 17], [1000, 777, 4000], 14, 2, False),
    ([300, 50], [10, 49], 3, 3, True),
    ([1] * 70, [13 * i % 400 for i in range(70)], 40, 8, True),
    ([16], [50000], 8, 1, True),                    # few rows, keys in parts
    ([2, 1, 40], [30000, 9000, 300], 5, 1, True),
    ([4097], None, 2, 2, True),
    ([2500, 1200], None, 24, 8, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_matches_the_definition(i):
    lq, lk, Hq, Hkv, causal = CASES[i]
    cu_q, cu_k = _cu(lq), _cu(lk or lq)
    print(f"varlen {lq} {lk} {Hq}/{Hkv} causal={causal}", flush=True)
    q, k, v = (_normal((n, H, D), 10 * i + j) for j, (n, H) in enumerate(
        ((cu_q[-1], Hq), (cu_k[-1], Hkv), (cu_k[-1], Hkv))))
    plan = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=Hkv, causal=causal, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    again = upipe.attn_fwd_varlen(q, k, v, plan)
    torch.cuda.synchronize()
    R.check_forward(o, lse, R.Packed(q, k, v, cu_q, cu_k, causal))
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def _layouts(n, Hq, Hkv, seed):
    """The same values as columns of one projection, keys beside values in every head,
    and head-major."""
    q, k, v = _normal((n, Hq, D), seed), _normal((n, Hkv, D), seed + 1), _normal((n, Hkv, D), seed + 2)
    yield "dense", q, k, v
    qkv = torch.cat([q, k, v], 1)
    yield "columns", *qkv.split([Hq, Hkv, Hkv], 1)
    kv = torch.stack([k, v], 2)
    yield "pairs", q, kv[:, :, 0], kv[:, :, 1]
    yield "head-major", *(t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))


@pytest.mark.gpu
def test_layouts_and_rows_behind_the_last():
    lens, Hq, Hkv = [200, 3, 411], 6, 2
    cu, n = _cu(lens), 614 + 9
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    want = None
    for name, q, k, v in _layouts(n, Hq, Hkv, 77):
        print("layout", name, flush=True)
        for t in (q, k, v):
            t[614:] = float("nan")           # rows behind the last sequence
        big = _normal((n, 2 * Hq, D), 5)
        o, lse = big[:, Hq:], torch.full((Hq, n), 3.0, device=DEV)
        keep = big.clone()
        upipe.attn_fwd_varlen(q, k, v, plan, out=(o, lse))
        torch.cuda.synchronize()
        assert torch.equal(big[:, :Hq], keep[:, :Hq]) and torch.equal(big[614:], keep[614:])
        assert bool((lse[:, 614:] == 3).all())
        if want is None:
            want = (o[:614].clone(), lse[:, :614].clone())
            R.check_forward(o[:614], lse[:, :614],
                            R.Packed(q[:614], k[:614], v[:614], cu, cu, True))
        assert torch.equal(o[:614], want[0]) and torch.equal(lse[:, :614], want[1])
        new = upipe.attn_fwd_varlen(q, k, v, plan)
        assert bool((new[0][614:] == 0).all()) and bool((new[1][:, 614:] == float("-inf")).all())
        # over its own queries
        qq = q.clone(memory_format=torch.preserve_format)
        upipe.attn_fwd_varlen(qq, k, v, plan, out=(qq, lse))
        assert torch.equal(qq[:614], want[0])


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("lens,Hq", [([300, 40], 4), ([300, 40], 1), ([2000, 9], 16)])
def test_masked_values_do_not_reach_a_row(bad, lens, Hq):
    """Key j is masked for the rows before it and for other sequences: whatever it and its
    value hold, they keep their results (to the same bounds: rows that shared a stage with a
    bad value are formed again, by sums in another order)."""
    cu = _cu(lens)
    q, k, v = _normal((cu[-1], Hq, D), 1), _normal((cu[-1], 1, D), 2), _normal((cu[-1], 1, D), 3)
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=1, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    ref = R.Packed(q, k, v, cu, cu, True)
    for j in (0, 45, 129, 250, lens[0] - 1):
        k2, v2 = k.clone(), v.clone()
        k2[j], v2[j] = bad, bad
        v2[j, 0, ::2] = 1.0
        o2, lse2 = upipe.attn_fwd_varlen(q, k2, v2, plan)
        torch.cuda.synchronize()
        other = torch.ones(cu[-1], dtype=torch.bool, device=DEV)
        other[j:lens[0]] = False
        assert not bool(o2[other].isnan().any()), (j, bad)
        R.check_forward(o2, lse2, ref, other)
        # only the value is bad: the weights are as before, and its good elements
        # spoil nothing
        o3, lse3 = upipe.attn_fwd_varlen(q, k, v2, plan)
        R.check_forward(o3, lse3, ref, other)
        R.check("lse of the others", lse3, ref.lse,
                R.score_error(ref.s_lse) + 4 * R.FP32 * ref.lse.abs() + 8 * R.FP32)
        assert bool(torch.isfinite(o3[:, :, ::2]).all())
        assert not bool(torch.isfinite(o3[j:lens[0], :, 1::2]).any())


@pytest.mark.gpu
def test_extreme_scores():
    """Scores of +-30000: one key takes all the weight, none overflows."""
    n = 200
    q, k, v = _normal((n, 2, D), 1), _normal((n, 1, D), 2), _normal((n, 1, D), 3)
    q *= 170.0
    k *= 170.0
    plan = upipe.VarlenPlan([0, n], Hq=2, Hkv=1, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    R.check_forward(o, lse, R.Packed(q, k, v, [0, n], [0, n], True))


@pytest.mark.gpu
def test_scores_far_below_nought():
    """Every score of a row about -1e36: the weights are what they are between equals."""
    n = 130
    q = torch.full((n, 1, D), 1e17, dtype=torch.bfloat16, device=DEV)
    k = torch.full((n, 1, D), -1e18, dtype=torch.bfloat16, device=DEV)
    v = _normal((n, 1, D), 3)
    plan = upipe.VarlenPlan([0, n], Hq=1, Hkv=1, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    mean = v.double().cumsum(0) / torch.arange(1, n + 1, device=DEV)[:, None, None]
    size = v.double().abs().cumsum(0) / torch.arange(1, n + 1, device=DEV)[:, None, None]
    # equal scores: equal weights, each rounded by half a step of bf16, as is the result
    R.check("o", o, mean, R.BF16 * mean.abs() + 2 * R.BF16 * size)
    score = float((q[0, 0].double() * k[0, 0].double()).sum()) / D ** 0.5
    R.check("lse", lse, torch.full_like(lse, score, dtype=torch.float64),
            torch.full_like(lse, (D + 8) * R.FP32 * abs(score), dtype=torch.float64))


@pytest.mark.gpu
def test_plan_on_another_device_is_refused():
    q = _normal((4, 1, D), 1)
    with pytest.raises(ValueError, match="devices"):
        upipe.attn_fwd_varlen(q, q, q, upipe.VarlenPlan([0, 4], Hq=1, Hkv=1, device="cpu"))


def _random_case(seed):
    r = random.Random(seed)
    n = r.choice([1, 2, 5, 17])
    q = [r.choice([0, 1, 2, 31, 64, 127, 129, 300, 900]) for _ in range(n)]
    k = [max(0, x + r.choice([0, 0, 0, 5, 400, 2000, -3, -x])) for x in q]
    Hkv = r.choice([1, 2, 3, 8])
    G = r.choice([1, 2, 3, 4, 5, 7, 8, 16, 21])
    return q, k, min(Hkv, 64 // G) * G, min(Hkv, 64 // G), r.random() < 0.75


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(8))
def test_random_lengths_and_heads(seed):
    lq, lk, Hq, Hkv, causal = _random_case(seed)
    cu_q, cu_k = _cu(lq), _cu(lk)
    print(f"random {lq} {lk} {Hq}/{Hkv} causal={causal}", flush=True)
    q, dout = _normal((cu_q[-1], Hq, D), seed), _normal((cu_q[-1], Hq, D), seed + 50)
    k, v = _normal((cu_k[-1], Hkv, D), seed + 100), _normal((cu_k[-1], Hkv, D), seed + 150)
    plan = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=Hkv, causal=causal, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    grads = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan)
    torch.cuda.synchronize()
    ref = R.Packed(q, k, v, cu_q, cu_k, causal, dout)
    R.check_forward(o, lse, ref)
    R.check_backward(*grads, ref)


@pytest.mark.gpu
def test_captured_and_on_another_stream():
    lens, Hq, Hkv = [33, 600, 2], 8, 2
    cu = _cu(lens)
    q, k, v = _normal((635, Hq, D), 1), _normal((635, Hkv, D), 2), _normal((635, Hkv, D), 3)
    few_q, few_k = _cu([4]), _cu([20000])
    kf, vf = _normal((20000, Hkv, D), 4), _normal((20000, Hkv, D), 5)
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=Hkv, device=DEV)
    parts = upipe.VarlenPlan(few_q, few_k, Hq=Hq, Hkv=Hkv, device=DEV)
    assert parts.fwd_workspace > 4096          # keys in parts

    def both():
        return (*upipe.attn_fwd_varlen(q, k, v, plan), *upipe.attn_fwd_varlen(q[:4], kf, vf, parts))
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.synchronize()
    for a, b in zip(want, other):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for n in range(3):
        q.mul_(0.5 ** n)
        want = both()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)


# ------------------------------------------------------------- no GPU needed

def _arr(x):
    return (ctypes.c_int64 * len(x))(*x)


def _size(cu_q, cu_k=None, Hq=4, Hkv=1, d=D, causal=1, n=None):
    cu_k = cu_q if cu_k is None else cu_k
    return upipe.upipe_varlen_plan_size(_arr(cu_q), _arr(cu_k), len(cu_q) - 1 if n is None else n, Hq,
                                        Hkv, d, causal)


def test_plan_refusals():
    assert _size([0, 5]) > 0 and _size([0]) > 0
    assert _size([0, 5, 3]) == 0 and _size([1, 5]) == 0 and _size([0, 5], [0, -1]) == 0
    assert _size([0, 5], Hq=4, Hkv=3) == 0 and _size([0, 5], Hq=65) == 0
    assert _size([0, 5], d=64) == 0 and _size([0, 5], causal=2) == 0
    assert _size([0, 1 << 24]) == 0 and _size([0, (1 << 24) - 128]) > 0
    assert _size([0, 5], n=-1) == 0
    assert upipe.upipe_varlen_plan_size(None, _arr([0]), 0, 4, 1, D, 1) == 0
    need = _size([0, 700, 800])
    buf = (ctypes.c_char * need)()
    at = ctypes.addressof(buf)

    def plan(to=at, n=need, cu=(0, 700, 800), **kw):
        a = dict(Hq=4, Hkv=1, d=D, causal=1)
        a.update(kw)
        return upipe.upipe_varlen_plan(_arr(cu), _arr(cu), 2, *a.values(), to, n)
    assert plan() == 0
    assert plan(n=need - 1) == -3 and plan(to=None) == -1 and plan(to=at + 4) == -1
    assert plan(cu=(0, 2, 1)) == -1 and plan(Hkv=3) == -1 and plan(d=64) == -2
    assert upipe.upipe_attn_fwd_varlen_workspace_size(at) > 0
    assert upipe.upipe_attn_fwd_varlen_workspace_size(None) == 0
    other = (ctypes.c_char * need)()
    assert upipe.upipe_attn_fwd_varlen_workspace_size(ctypes.addressof(other)) == 0


FAKE = 1 << 24


def _heads(p=FAKE, row=4 * D, head=D):
    return upipe.upipe_heads(p, row, head)


def test_forward_refusals():
    cu = [0, 700, 800]
    plan = upipe.VarlenPlan(cu, Hq=4, Hkv=1, device="cpu")

    def fwd(**kw):
        a = dict(q=_heads(), k=_heads(2 * FAKE, D), v=_heads(3 * FAKE, D), o=_heads(4 * FAKE),
                 lse=FAKE, lse_head=800, plan=plan.host, dev=FAKE, ws=FAKE, n=0, stream=None)
        a.update(kw)
        return upipe.upipe_attn_fwd_varlen(*a.values())
    INV, UNS, WS = -1, -2, -3
    assert fwd() == WS                       # valid but for the workspace
    for bad in (dict(plan=None), dict(dev=None), dict(dev=FAKE + 8), dict(lse=None), dict(ws=None),
                dict(lse_head=799), dict(q=_heads(FAKE + 2)), dict(q=_heads(row=-8)),
                dict(q=_heads(0)), dict(k=_heads(2 * FAKE, 12)), dict(v=_heads(0, D)),
                dict(o=_heads(4 * FAKE, head=64)), dict(o=_heads(4 * FAKE, row=2 * D)),
                dict(o=_heads(FAKE + 256)), dict(o=_heads(2 * FAKE)), dict(o=_heads(3 * FAKE))):
        assert fwd(**bad) == INV, bad
    assert fwd(k=_heads(1 << 40, (1 << 22) + 8)) == UNS
    assert fwd(o=_heads()) == WS             # over its own queries
    # no rows: nothing to look at
    none = upipe.VarlenPlan([0, 0], Hq=4, Hkv=1, device="cpu")
    assert fwd(plan=none.host, q=_heads(0), o=_heads(0), lse=None) == 0


def test_binding_refuses():
    with pytest.raises(ValueError, match="offsets"):
        upipe.VarlenPlan([0, 4], [0, 4, 8], Hq=4, Hkv=1, device="cpu")
    with pytest.raises(upipe.UpipeError):
        upipe.VarlenPlan([0, 4, 2], Hq=4, Hkv=1, device="cpu")
    plan = upipe.VarlenPlan(torch.tensor([0, 4, 9]), Hq=4, Hkv=1, device="cpu")
    q = torch.zeros((9, 4, D), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        upipe.attn_fwd_varlen(q, q[:, :1], q[:, :1], plan)
