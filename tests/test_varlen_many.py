"""Batches of many short sequences, which go by workgroups of four waves, two a CU: forward
and backward against the definition in 64 bits (bounds in varlen_ref.py)."""

import random
import struct

import pytest
import torch

import varlen_ref as R
from paper_2602_21196_amd import upipe
from test_varlen import _cu, _normal

DEV = "cuda:0"
D = 128


def _half(plan):
    """Bits of the plan: the forward, dQ by half workgroups."""
    return struct.unpack_from("<Q6q12i", bytes(plan._host))[-1]


def _lens(kind):
    r = random.Random(kind)
    return {"even": [256] * 16, "odd": [r.choice([0, 1, 31, 33, 129, 200, 257]) for _ in range(60)],
            "pieces": [r.randint(1, 40) for _ in range(150)]}[kind]


CASES = [  # queries, keys besides them, Hq, Hkv, causal, bits
    ("even", 0, 32, 8, True, 3),
    ("odd", 0, 24, 8, True, 3),            # 3 rows a token: tokens in two waves
    ("odd", 70, 16, 16, True, 3),          # behind what a cache holds
    ("odd", -20, 32, 4, True, 3),          # rows that see nothing
    ("pieces", 0, 40, 8, False, 3),
    ("pieces", 0, 64, 1, True, 3),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_plan_chooses_half_workgroups(i):
    kind, more, Hq, Hkv, causal, bits = CASES[i]
    lq = _lens(kind)
    lk = [max(0, n + more) for n in lq]
    plan = upipe.VarlenPlan(_cu(lq), _cu(lk), Hq=Hq, Hkv=Hkv, causal=causal, device="cpu")
    assert _half(plan) == bits


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CASES)))
def test_matches_the_definition(i):
    kind, more, Hq, Hkv, causal, _ = CASES[i]
    lq = _lens(kind)
    cu_q, cu_k = _cu(lq), _cu([max(0, n + more) for n in lq])
    print(f"{kind} {len(lq)} sequences, {cu_q[-1]} on {cu_k[-1]}, {Hq}/{Hkv}", flush=True)
    q, k, v, dout = (_normal((n, H, D), 700 + 10 * i + j) for j, (n, H) in enumerate(
        ((cu_q[-1], Hq), (cu_k[-1], Hkv), (cu_k[-1], Hkv), (cu_q[-1], Hq))))
    plan = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=Hkv, causal=causal, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    dq, dk, dv = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan)
    into = q.clone()
    upipe.attn_fwd_varlen(into, k, v, plan, out=(into, torch.empty_like(lse)))
    torch.cuda.synchronize()
    ref = R.Packed(q, k, v, cu_q, cu_k, causal, dout)
    R.check_forward(o, lse, ref)
    R.check_backward(dq, dk, dv, ref)
    assert torch.equal(into, o)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_masked_values_stay_out(bad):
    """The last token's value of every sequence: only its own row may have it."""
    lens = [1 + 37 * i % 90 for i in range(80)]
    cu = _cu(lens)
    q, k, v = (_normal((cu[-1], H, D), 5 + H) for H in (32, 8, 8))
    plan = upipe.VarlenPlan(cu, Hq=32, Hkv=8, device=DEV)
    assert _half(plan) & 1
    want, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    last = torch.tensor([c - 1 for c in cu[1:]], device=DEV)
    v[last] = bad
    got, lse2 = upipe.attn_fwd_varlen(q, k, v, plan)
    torch.cuda.synchronize()
    keep = torch.ones(cu[-1], dtype=torch.bool, device=DEV)
    keep[last] = False
    # formed again by plain arithmetic: half a step of the weights and of the result
    assert bool(got[keep].isfinite().all()) and not bool(got[last].isfinite().any())
    err = (got[keep].double() - want[keep].double()).abs()
    assert float(err.max()) <= 4 * R.BF16 * float(v[keep].abs().max())
    assert torch.allclose(lse2[:, keep], lse[:, keep], rtol=0, atol=1e-4)
