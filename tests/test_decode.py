"""Attention of new tokens against caches and a shared prefix, against its definition
in 64 bits (bounds in varlen_ref.py), and what the calls refuse."""

import pytest
import torch

import varlen_ref as R
from paper_2602_21196_amd import upipe

DEV = "cuda:0"
D = 128


def _normal(shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


class _Ref:
    """o [tokens, Hq, d] and lse [Hq, tokens] of every sequence's prefix and cache rows."""

    def __init__(self, q, k, v, lens, kp=None, vp=None):
        B, nq, Hq, _ = q.shape
        G = Hq // k.shape[2]
        P = 0 if kp is None else kp.shape[0]
        flat = q.double().reshape(B * nq, Hq, D)
        self.o, self.a_o = torch.zeros_like(flat), torch.zeros_like(flat)
        self.lse = torch.full((Hq, B * nq), -float("inf"), dtype=torch.float64, device=q.device)
        self.s_lse = torch.zeros_like(self.lse)
        for b, n in enumerate(lens):
            n = min(max(n, 0), k.shape[1])
            see = R.visible(nq, n, True, q.device)
            see = torch.cat([torch.ones((nq, P), dtype=torch.bool, device=q.device), see], 1)
            at = slice(b * nq, b * nq + nq)
            for h in range(Hq):
                ks, vs = k[b, :n, h // G].double(), v[b, :n, h // G].double()
                if P:
                    ks = torch.cat([kp[:, h // G].double(), ks])
                    vs = torch.cat([vp[:, h // G].double(), vs])
                o, lse, p, size = R.attend(flat[at, h], ks, vs, see)
                self.o[at, h], self.lse[h, at] = o, lse
                self.a_o[at, h], self.s_lse[h, at] = p @ vs.abs(), size


def _check(o, lse, ref):
    B, nq, Hq, _ = o.shape
    R.check_forward(o.reshape(B * nq, Hq, D), lse.transpose(0, 1).reshape(Hq, B * nq), ref)


CASES = [  # lens, cap, nq, Hq, Hkv, P
    ([1], 1, 1, 1, 1, 0),
    ([1], 16, 1, 64, 1, 0),
    ([5, 0, 16, 99, -3], 16, 1, 4, 2, 0),          # none valid, more than there are
    ([1, 3, 4, 100], 130, 4, 6, 2, 0),             # tokens before the first row see nothing
    ([127, 128, 129, 255, 256, 257, 1], 300, 1, 8, 2, 0),
    ([700, 33], 4000, 7, 14, 2, 0),
    ([1000, 90], 1024, 128, 3, 1, 0),
    ([50000], 50001, 1, 8, 1, 0),                  # a long one, in parts
    ([9, 20000, 300], 20000, 2, 5, 5, 0),
    ([2, 0, 3], 16, 1, 4, 2, 5),
    ([0, 0], 8, 3, 4, 4, 1000),                    # the prefix alone
    ([64, 1, 700], 1000, 2, 40, 8, 129),
    (list(range(1, 65)), 64, 1, 32, 4, 5000),
    ([4, 150, 61], 256, 4, 8, 1, 1000),
]


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(CASES)))
def test_matches_the_definition(i):
    lens, cap, nq, Hq, Hkv, P = CASES[i]
    B = len(lens)
    print(f"decode {lens[:8]} cap={cap} nq={nq} {Hq}/{Hkv} P={P}", flush=True)
    q = _normal((B, nq, Hq, D), 20 * i)
    kv = _normal((B, cap, 2, Hkv, D), 20 * i + 1)           # one buffer of both
    k, v = kv[:, :, 0], kv[:, :, 1]
    for b, n in enumerate(lens):                            # what lies behind is not looked at
        kv[b, max(n, 0):] = float("nan") if b % 2 else float("inf")
    pre = [_normal((P, Hkv, D), 20 * i + 2 + j) for j in range(2)] if P else [None, None]
    ld = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = upipe.attn_decode(q, k, v, ld, *pre)
    torch.cuda.synchronize()
    _check(o, lse, _Ref(q, k, v, lens, *pre))
    # on its own queries, with a workspace of garbage, and once more
    ws = upipe.workspace(upipe.upipe_attn_decode_workspace_size(B, nq, cap, P, Hq, Hkv, D), DEV)
    ws.fill_(255)
    q2, lse2 = q.clone(), torch.empty_like(lse)
    upipe.attn_decode(q2, k, v, ld, *pre, out=(q2, lse2), ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(q2, o) and torch.equal(lse2, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_later_tokens_do_not_reach_earlier_ones(bad):
    nq, Hq, Hkv, n = 4, 8, 2, 300
    q = _normal((1, nq, Hq, D), 1)
    k, v = _normal((1, n, Hkv, D), 2), _normal((1, n, Hkv, D), 3)
    ld = torch.tensor([n], dtype=torch.int32, device=DEV)
    ref = _Ref(q, k, v, [n])
    k[0, n - 2:], v[0, n - 2:] = bad, bad
    o, lse = upipe.attn_decode(q, k, v, ld)
    torch.cuda.synchronize()
    R.check_forward(o.reshape(nq, Hq, D), lse.transpose(0, 1).reshape(Hq, nq), ref, slice(0, 2))
    assert bool(o[0, 2:].isnan().all())


@pytest.mark.gpu
def test_replayed_as_the_caches_grow():
    B, nq, Hq, Hkv, cap, P = 3, 1, 8, 2, 1500, 200
    q = _normal((B, nq, Hq, D), 1)
    k, v = _normal((B, cap, Hkv, D), 2), _normal((B, cap, Hkv, D), 3)
    kp, vp = _normal((P, Hkv, D), 4), _normal((P, Hkv, D), 5)
    lens = torch.tensor([1, 128, 1200], dtype=torch.int32, device=DEV)
    upipe.attn_decode(q, k, v, lens, kp, vp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = upipe.attn_decode(q, k, v, lens, kp, vp)
    for step in (1, 1, 127, 170):
        lens += step
        q.normal_()
        want = upipe.attn_decode(q, k, v, lens, kp, vp)
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        _check(o, lse, _Ref(q, k, v, lens.tolist(), kp, vp))


@pytest.mark.gpu
def test_a_prompt_then_tokens_give_what_one_prompt_gives():
    """Packed prompts, then new tokens one at a time from the caches they filled: the
    same results as prompts that held them from the start, to the bounds of both."""
    lens, new, Hq, Hkv, cap = [130, 7, 513], 3, 8, 2, 640
    total = [n + new for n in lens]
    q, k, v = ([_normal((n, H, D), 10 * s + i) for i, n in enumerate(total)]
               for s, H in ((1, Hq), (2, Hkv), (3, Hkv)))
    caches = [torch.full((3, cap, Hkv, D), float("nan"), dtype=torch.bfloat16, device=DEV)
              for _ in range(2)]
    for b, n in enumerate(total):
        caches[0][b, :n], caches[1][b, :n] = k[b], v[b]
    cu = [0, total[0], total[0] + total[1], sum(total)]
    whole = R.Packed(torch.cat(q), torch.cat(k), torch.cat(v), cu, cu, True)
    for t in range(new):
        ld = torch.tensor([n + t + 1 for n in lens], dtype=torch.int32, device=DEV)
        qt = torch.stack([q[b][lens[b] + t] for b in range(3)])[:, None]
        o, lse = upipe.attn_decode(qt, *caches, ld)
        torch.cuda.synchronize()
        rows = torch.tensor([cu[b] + lens[b] + t for b in range(3)], device=DEV)

        class At:
            o, a_o = whole.o[rows], whole.a_o[rows]
            lse, s_lse = whole.lse[:, rows], whole.s_lse[:, rows]
        _check(o, lse, At)


# ------------------------------------------------------------- no GPU needed

FAKE = 1 << 30


def _heads(p=FAKE, row=4 * D, head=D):
    return upipe.upipe_heads(p, row, head)


def _call(**kw):
    a = dict(q=_heads(), k=_heads(2 * FAKE, D), k_cache=100 * D, v=_heads(3 * FAKE, D),
             v_cache=100 * D, lens=FAKE, kp=_heads(4 * FAKE, D), vp=_heads(5 * FAKE, D),
             o=_heads(6 * FAKE), lse=FAKE, B=8, nq=1, cap=100, P=16, Hq=4, Hkv=1, d=D, ws=FAKE,
             n=0, stream=None)
    a.update(kw)
    return upipe.upipe_attn_decode(*a.values())


def test_refusals():
    INV, UNS, WS = -1, -2, -3
    assert _call() == WS                     # valid but for the workspace
    for bad in (dict(B=0), dict(nq=0), dict(cap=0), dict(P=-1), dict(Hkv=3), dict(Hq=0),
                dict(q=_heads(0)), dict(k=_heads(2 * FAKE + 2, D)), dict(v=_heads(0, D)),
                dict(k_cache=12), dict(v_cache=-8), dict(k_cache=1 << 60), dict(lens=None),
                dict(lens=FAKE + 2), dict(lse=None), dict(ws=None), dict(kp=_heads(0, D)),
                dict(vp=_heads(5 * FAKE, 4)), dict(o=_heads(6 * FAKE, row=D)), dict(o=_heads(FAKE + 256)),
                dict(o=_heads(2 * FAKE)), dict(o=_heads(3 * FAKE + 256 * 100 * 7)),
                dict(o=_heads(5 * FAKE))):
        assert _call(**bad) == INV, bad
    for bad in (dict(d=64), dict(Hq=65), dict(nq=129), dict(cap=1 << 24), dict(P=1 << 24),
                dict(B=65537), dict(B=65536, nq=128, Hq=64, Hkv=1, k_cache=0, v_cache=0),
                dict(k=_heads(2 * FAKE, (1 << 22) + 8))):
        assert _call(**bad) == UNS, bad
    assert _call(o=_heads()) == WS           # over its own queries
    assert _call(P=0, kp=_heads(0), vp=_heads(0)) == WS
    assert upipe.upipe_attn_decode_workspace_size(0, 1, 1, 0, 1, 1, D) == 0
    assert upipe.upipe_attn_decode_workspace_size(8, 1, 100, 0, 4, 1, D) > 0


def test_binding_refuses():
    q = torch.zeros((2, 1, 4, D), dtype=torch.bfloat16)
    c = torch.zeros((2, 8, 1, D), dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        upipe.attn_decode(q, c, c, n)
    with pytest.raises(ValueError, match="neither"):
        upipe.attn_decode(q, c, c, n, k_prefix=c[0])
    with pytest.raises(ValueError, match="lens"):
        upipe.attn_decode(q, c, c, n[:1])
    with pytest.raises(ValueError, match="evenly"):
        upipe.attn_decode(torch.zeros((2, 3, 4, D), dtype=torch.bfloat16)[:, :2], c, c, n)


# A prefix and caches in one launch: tiles of 128 and 64 of the prefix's rows, of 64 packed
# rows of the caches.
BEHIND = [  # B, lens up to, cap, nq, Hq, Hkv, P
    (2, 300, 1000, 40, 8, 2, 700),
    (3, 2000, 2048, 16, 16, 2, 3000),
    (40, 60, 64, 8, 64, 8, 1000),
    (64, 40, 48, 16, 64, 1, 300),
    (96, 30, 32, 4, 64, 8, 600),
    (256, 9, 16, 4, 64, 8, 260),
]


@pytest.mark.gpu
@pytest.mark.parametrize("i", range(len(BEHIND)))
def test_many_tokens_behind_a_prefix(i):
    B, most, cap, nq, Hq, Hkv, P = BEHIND[i]
    print(f"{B} caches of up to {most}/{cap}, nq={nq} {Hq}/{Hkv} P={P}", flush=True)
    lens = [most * (b * b % 7) // 6 for b in range(B)]
    q, kv = _normal((B, nq, Hq, D), 90 * i), _normal((B, cap, 2, Hkv, D), 90 * i + 1)
    k, v = kv[:, :, 0], kv[:, :, 1]
    for b, n in enumerate(lens):
        kv[b, n:] = float("nan")
    kp, vp = _normal((P, Hkv, D), 90 * i + 2), _normal((P, Hkv, D), 90 * i + 3)
    o, lse = upipe.attn_decode(q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), kp, vp)
    torch.cuda.synchronize()
    _check(o, lse, _Ref(q, k, v, lens, kp, vp))


def test_no_more_parts_than_the_merge_holds():
    """A row's parts, its cache's and the prefix's, have their weights in LDS: 2048 at most
    (the workspace holds 129 words of every part's rows)."""
    for cap in (1, 511, 513, 100000, 1 << 20, (1 << 24) - 128):
        for P in (0, 1, 5000, (1 << 24) - 128):
            for B, nq, Hq, Hkv in ((1, 1, 1, 1), (1, 1, 64, 8), (7, 3, 16, 2), (1, 128, 64, 1),
                                   (300, 1, 64, 64), (3, 40, 8, 2), (65536, 1, 32, 8)):
                size = upipe.upipe_attn_decode_workspace_size(B, nq, cap, P, Hq, Hkv, D)
                parts, rest = divmod(size - 16, 129 * 4 * B * nq * Hq)
                assert rest == 0 and 1 <= parts <= 2048, (cap, P, B, nq, Hq, Hkv, parts)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,Hq,Hkv", [(1, 32, 8), (9, 20, 4)])
def test_caches_of_very_different_lengths(nq, Hq, Hkv):
    """More workgroups than start at once, caches alike and longest last among them: the
    order in which they are worked on changes nothing else."""
    lens, cap = [0, 3, 40, 40, 1, 2000, 700, 5, 40, 0, 9000, 16000, 333, 8192], 16000
    B = len(lens)
    q, kv = _normal((B, nq, Hq, D), 1), _normal((B, cap, 2, Hkv, D), 2)
    k, v = kv[:, :, 0], kv[:, :, 1]
    for b, n in enumerate(lens):
        kv[b, n:] = float("nan")
    ld = torch.tensor(lens, dtype=torch.int32, device=DEV)
    o, lse = upipe.attn_decode(q, k, v, ld)
    turn = list(range(B))[::-1]
    o2, lse2 = upipe.attn_decode(q[turn], k[turn], v[turn], ld[turn])
    torch.cuda.synchronize()
    _check(o, lse, _Ref(q, k, v, lens))
    assert torch.equal(o2[turn], o) and torch.equal(lse2[turn], lse)


def test_large_calls_are_not_cut():
    """Where whole tiles fill the chip many times a row has one part, or two with the prefix:
    the workspace stays within a few times the rows."""
    for B, nq, cap, P in ((65536, 1, 4096, 0), (4096, 8, 1 << 20, 1 << 20), (2000, 128, 65536, 999)):
        size = upipe.upipe_attn_decode_workspace_size(B, nq, cap, P, 16, 4, D)
        assert size - 16 == (1 + (P > 0)) * 129 * 4 * B * nq * 16, (B, nq, cap, P)
