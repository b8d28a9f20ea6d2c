"""Values that are infinite or not a number, some visible and some masked, in the forward
over packed sequences and over caches: what they may change and what they may not."""

import pytest
import torch

import varlen_ref as R
from paper_2602_21196_amd import upipe
from test_varlen import _normal

DEV = "cuda:0"
D = 128
pytestmark = pytest.mark.gpu

VALUES = [float("nan"), float("inf")]
BATCHES = [([300, 40], 4), ([300, 40], 1), ([2000, 9], 16)] + [([64 + i % 3 for i in range(70)], 32)]


@pytest.mark.parametrize("bad", VALUES)
@pytest.mark.parametrize("lens,Hq", BATCHES)
def test_log_sum_exps_do_not_depend_on_values(bad, lens, Hq):
    """A whole value row is bad where it is visible, and a later one of its stage where it
    is masked: no element of the rows between them is finite, but their lse is
    that of all their keys, and with it dV, which no value enters."""
    cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
    q, k, v, dout = (_normal((cu[-1], H, D), j) for j, H in enumerate((Hq, 1, 1, Hq)))
    plan = upipe.VarlenPlan(cu, Hq=Hq, Hkv=1, device=DEV)
    ref = R.Packed(q, k, v, cu, cu, True, dout)
    for first, second in ((10, 50), (0, 31), (5, 63)):
        bv = v.clone()
        bv[[first, second]] = bad
        o, lse = upipe.attn_fwd_varlen(q, k, bv, plan)
        _, _, dv = upipe.attn_bwd_varlen(q, k, bv, o, lse, dout, plan)
        torch.cuda.synchronize()
        R.check("lse", lse, ref.lse,
                R.score_error(ref.s_lse) + 4 * R.FP32 * ref.lse.abs() + 8 * R.FP32)
        assert not bool(o[first:lens[0]].isfinite().any())
        clean = torch.cat([o[:first], o[lens[0]:]])
        assert bool(clean.isfinite().all())
        es = float(R.score_error(ref.s_lse.max()))
        c = R.BF16 + (1 + R.BF16) * (3 * es + 16 * R.FP32)
        R.check("dv", dv, ref.dv, R.BF16 * ref.dv.abs() + (1 + R.BF16) * c * ref.a_dv + 1e-30)


def test_opposite_infinities_are_not_a_number():
    """Row i sees +inf at key 10 and, from row 20 on, -inf at key 20; key 50's NaN is
    masked for the rows before it."""
    n = 64
    q, k, v = _normal((n, 2, D), 1), _normal((n, 1, D), 2), _normal((n, 1, D), 3)
    v[10], v[20], v[50] = float("inf"), float("-inf"), float("nan")
    o, lse = upipe.attn_fwd_varlen(q, k, v, upipe.VarlenPlan([0, n], Hq=2, Hkv=1, device=DEV))
    torch.cuda.synchronize()
    assert bool(o[:10].isfinite().all()) and bool((o[10:20] == float("inf")).all())
    assert bool(o[20:].isnan().all()) and bool(lse.isfinite().all())


@pytest.mark.parametrize("bad", VALUES)
def test_large_scores_beside_bad_values(bad):
    """Scores beyond 2^30 and a bad visible value: lse is that of all keys."""
    n = 100
    q = torch.full((n, 1, D), 1e8, dtype=torch.bfloat16, device=DEV)
    k = torch.full((n, 1, D), -1e3, dtype=torch.bfloat16, device=DEV)
    v = _normal((n, 1, D), 3)
    v[[3, 70]] = bad
    o, lse = upipe.attn_fwd_varlen(q, k, v, upipe.VarlenPlan([0, n], Hq=1, Hkv=1, device=DEV))
    score = float((q[0, 0].double() * k[0, 0].double()).sum()) / D ** 0.5
    torch.cuda.synchronize()
    R.check("lse", lse, torch.full_like(lse, score, dtype=torch.float64),
            torch.full_like(lse, (D + 8) * R.FP32 * abs(score), dtype=torch.float64))
    assert bool(o[:3].isfinite().all()) and not bool(o[3:].isfinite().any())


@pytest.mark.parametrize("bad", VALUES)
@pytest.mark.parametrize("at", [0, 700, 4999])
def test_a_visible_value_reaches_the_row_from_every_part(bad, at):
    """Key 5000 has a score 220 above the others', so the weights of parts without it are 0
    in fp32 (e^-220 = 2^-317): a bad value there is visible all the same.  In parts of a
    cache, in parts of a packed sequence, behind a prefix, and whole."""
    n, Hq = 20000, 8
    q = torch.ones((4, Hq, D), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((n, 1, D), dtype=torch.bfloat16, device=DEV)
    v = _normal((n, 1, D), 3)
    k[5000] = 220 / D ** 0.5                    # 128 products over sqrt 128
    v[at, 0, 3] = bad
    score = float(k[5000, 0].double().sum()) / D ** 0.5
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    plan = upipe.VarlenPlan([0, 4], [0, n], Hq=Hq, Hkv=1, device=DEV)
    assert plan.fwd_workspace > 4096            # keys in parts
    runs = {"cache": upipe.attn_decode(q[None], k[None], v[None], lens),
            "prefix": upipe.attn_decode(q[None], k[None, 6000:], v[None, 6000:], lens - 6000,
                                        k[:6000], v[:6000]),
            "packed": upipe.attn_fwd_varlen(q, k, v, plan)}
    torch.cuda.synchronize()
    for name, (o, lse) in runs.items():
        o = o.reshape(4 * Hq, D)
        rest = [e for e in range(D) if e != 3]
        print(f"  {name}: {int((~o[:, 3].isfinite()).sum())} of {4 * Hq} rows", flush=True)
        assert not bool(o[:, 3].isfinite().any()), name
        assert bool(o[:, rest].isfinite().all()), name
        R.check("lse", lse, torch.full_like(lse, score, dtype=torch.float64),
                torch.full_like(lse, (D + 8) * R.FP32 * score, dtype=torch.float64))


REACH = 192          # of a masked pair's bad row in the backward, in keys


@pytest.mark.parametrize("Lq,Lk,G", [(512, 513, 1), (512, 639, 1), (400, 400, 3), (700, 1000, 2),
                                     (300, 290, 5), (256, 256, 16)])
def test_how_far_a_masked_pair_reaches_in_the_backward(Lq, Lk, G):
    """Gradients of rows and keys from 192 on behind a bad row's last visible key keep their
    bits: a tile of 128 rows and a block of 128 keys meet with 127 keys and half a tile between
    a row's last key and a key, a stage of keys and the 32 rows of a wave with less."""
    q, dout = _normal((Lq, G, D), 1), _normal((Lq, G, D), 2)
    k, v = _normal((Lk, 1, D), 3), _normal((Lk, 1, D), 4)
    plan = upipe.VarlenPlan([0, Lq], [0, Lk], Hq=G, Hkv=1, device=DEV)
    o, lse = upipe.attn_fwd_varlen(q, k, v, plan)
    want = upipe.attn_bwd_varlen(q, k, v, o, lse, dout, plan)
    far = 0
    for i in (0, 1, 63, 64, 127, 128, 191, Lq - 1):
        if i >= Lq:
            continue
        last = i + Lk - Lq                  # the bad row's last key
        for bad in VALUES:
            for at in (0, 1):
                x = [q.clone(), dout.clone()]
                x[at][i] = bad
                got = upipe.attn_bwd_varlen(x[0], k, v, o, lse, x[1], plan)
                torch.cuda.synchronize()
                for a, b in zip(got[1:], want[1:]):
                    other = (a != b).any(-1).any(-1).nonzero()
                    far = max(far, int(other.max()) - last if other.numel() else 0)
                keep = torch.arange(Lq, device=DEV) != i
                assert torch.equal(got[0][keep], want[0][keep])
    near = 0
    for j in (0, 5, 127, 128, 255, Lk - 1):
        if j >= Lk:
            continue
        for bad in VALUES:
            bk = k.clone()
            bk[j] = bad
            got = upipe.attn_bwd_varlen(q, bk, v, o, lse, dout, plan)
            torch.cuda.synchronize()
            other = (got[0] != want[0]).any(-1).any(-1).nonzero()
            near = max(near, j - (int(other.min()) + Lk - Lq) if other.numel() else 0)
    print(f"  a row reaches {far} keys behind its last, a key {near} rows before its first",
          flush=True)
    assert far < REACH and near < REACH


@pytest.mark.parametrize("bad", [*VALUES, "mixed"])
@pytest.mark.parametrize("lens,Hq,part", [([9000], 4, False), ([4, 300], 8, True), ([700, 33, 1], 2, False)])
def test_a_bad_column_of_every_value(bad, lens, Hq, part):
    """A column that is bad in every row: bad in every result, the others what they are.  With
    infinities of both signs a row has that of its only key, or no number."""
    lk = [20000, 300] if part else lens
    cu_q, cu_k = ([sum(x[:i]) for i in range(len(x) + 1)] for x in (lens, lk))
    q, k, v = (_normal((n, H, D), j) for j, (n, H) in enumerate(
        ((cu_q[-1], Hq), (cu_k[-1], 1), (cu_k[-1], 1))))
    plan = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=1, device=DEV)
    ref = R.Packed(q, k, v, cu_q, cu_k, True)
    bv = v.clone()
    inf = float("inf")
    for col in (0, 37, 127):
        bv[:, 0, col] = inf if bad == "mixed" else bad
    if bad == "mixed":
        bv[1::2, 0, 37] = -inf
    o, lse = upipe.attn_fwd_varlen(q, k, bv, plan)
    torch.cuda.synchronize()
    R.check("lse", lse, ref.lse,
            R.score_error(ref.s_lse) + 4 * R.FP32 * ref.lse.abs() + 8 * R.FP32)
    if bad == "mixed":
        assert bool((o[:, :, [0, 127]] == inf).all())
        first = torch.zeros(cu_q[-1], dtype=torch.bool, device=DEV)       # rows of one key
        first[[a for a, x, y in zip(cu_q, lens, lk) if x == y]] = True
        assert bool(o[~first][:, :, 37].isnan().all()) and bool(o[first][:, :, 37].isinf().all())
    else:
        want = o.isnan() if bad != bad else o == inf
        assert bool(want[:, :, [0, 37, 127]].all())
    keep = [e for e in range(D) if e not in (0, 37, 127)]
    es = R.score_error(ref.s_lse)
    w = R.BF16 + 2 * es.T[..., None] + 8 * R.FP32
    R.check("others", o[:, :, keep], ref.o[:, :, keep],
            (R.BF16 * ref.o.abs() + (1 + R.BF16) * w * ref.a_o)[:, :, keep] + 1e-30)


@pytest.mark.parametrize("bad", VALUES)
def test_a_bad_column_takes_no_lifetime(bad):
    """One bad column of every value in a long sequence, as a diverged step leaves it: no
    more than 30 times as long as clean ones (formed again key by key it was 62)."""
    n = 16384
    q, k, v = _normal((n, 8, D), 1), _normal((n, 1, D), 2), _normal((n, 1, D), 3)
    plan = upipe.VarlenPlan([0, n], Hq=8, Hkv=1, device=DEV)
    times = []
    for spoil in (False, True):
        if spoil:
            v[:, 0, 5] = bad
        upipe.attn_fwd_varlen(q, k, v, plan)
        torch.cuda.synchronize()
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(3):
            upipe.attn_fwd_varlen(q, k, v, plan)
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) / 3)
    print(f"  clean {times[0]:.3f} ms, with a bad column {times[1]:.3f}", flush=True)
    assert times[1] <= 30 * times[0]
