"""The plan of packed sequences on the host: what its lists name is every piece of work
once, within the tensors and the workspace, longest first."""

import random
import struct

import pytest

from paper_2602_21196_amd import upipe


def _items(host, at, n, form):
    size = struct.calcsize(form)
    return [struct.unpack_from(form, host, at + i * size) for i in range(n)]


def _plan(cu_q, cu_k, Hq, Hkv, causal):
    p = upipe.VarlenPlan(cu_q, cu_k, Hq=Hq, Hkv=Hkv, causal=causal, device="cpu")
    host = bytes(p._host)
    ints = "<Q6q3i2i1i5i"
    head = struct.unpack_from(ints, host)
    at = struct.unpack_from("<5q", host, (struct.calcsize(ints) + 7) // 8 * 8)
    names = ("magic bytes total_q total_k part_rows term_rows slots Hq Hkv causal fwd_ks dq_ks "
             "one_row n_fwd n_merge n_key n_fold n_dq").split()
    h = dict(zip(names, head), **dict(zip("at_fwd at_merge at_key at_fold at_dq".split(), at)))
    assert h["bytes"] == len(host) and (h["Hq"], h["Hkv"], h["causal"]) == (Hq, Hkv, int(causal))
    fwd = _items(host, h["at_fwd"], h["n_fwd"], "<3q6i")
    merge = _items(host, h["at_merge"], h["n_merge"], "<2q4i")
    key = _items(host, h["at_key"], h["n_key"], "<3q6i")
    fold = _items(host, h["at_fold"], h["n_fold"], "<q4i")
    dq = _items(host, h["at_dq"], h["n_dq"], "<3q4i")
    return p, h, fwd, merge, key, fold, dq


def _seen(tok, Lq, Lk, causal):
    return max(0, min(Lk, tok + 1 + Lk - Lq)) if causal else Lk


CASES = [([7, 1, 130, 0, 33], None, 4, 1, True), ([5], [0], 4, 2, True), ([0, 0], [9, 200], 4, 2, False),
         ([16], [50000], 8, 1, True), ([1] * 8, [20000] * 8, 8, 1, True),
         ([3000, 500], [100, 9000], 6, 3, True), ([32768, 12000, 2], None, 8, 1, True),
         ([8192], None, 8, 2, True), ([2500], None, 66 - 2, 64, False)]


def _random(seed):
    r = random.Random(seed)
    q = [r.choice([0, 1, 5, 100, 129, 1000, 5000]) for _ in range(r.randint(1, 12))]
    k = [max(0, n + r.choice([0, 0, 7, 3000, -50])) for n in q]
    Hkv = r.choice([1, 2, 4])
    return q, k, Hkv * r.choice([1, 2, 3, 5, 8, 16]), Hkv, r.random() < 0.7


@pytest.mark.parametrize("case", CASES + [_random(s) for s in range(12)])
def test_every_piece_of_work_once(case):
    lq, lk, Hq, Hkv, causal = case
    lk = lk or lq
    G, tpt = Hq // Hkv, 128 // (Hq // Hkv)
    cu_q = [sum(lq[:i]) for i in range(len(lq) + 1)]
    cu_k = [sum(lk[:i]) for i in range(len(lk) + 1)]
    p, h, fwd, merge, key, fold, dq = _plan(cu_q, cu_k, Hq, Hkv, causal)
    of = {(cu_q[i], cu_k[i], lq[i], lk[i]) for i in range(len(lq))}
    # forward: every tile of every sequence in all of its parts, once; parts apart from
    # each other and within the workspace
    rows = 256 // h["fwd_ks"]
    want = sorted((cu_q[i], cu_k[i], t) for i in range(len(lq)) for t in range(-(-lq[i] * G // rows)))
    parts = {}
    for q0, k0, p0, Lq, Lk, tile, part, n, _ in fwd:
        assert (q0, k0, Lq, Lk) in of and 0 <= part < n
        parts.setdefault((q0, k0, tile), []).append(part)
        if n > 1:
            assert 0 <= p0 and p0 + n * Lq * Hq <= h["part_rows"]
    assert sorted(parts) == sorted(set(want)) and len(want) == len(set(want))
    assert all(sorted(v) == list(range(len(v))) for v in parts.values())
    # merges: the rows of the sequences that are cut
    cut = {(q0, p0, Lq, n) for q0, _, p0, Lq, _, _, _, n, _ in fwd if n > 1}
    per = 1 if h["one_row"] else 16
    assert sorted((m[0], m[1], m[2], m[3], m[4]) for m in merge) == sorted(
        (*c, b) for c in cut for b in range(-(-c[2] * Hq // per)))
    spans = sorted((p0, p0 + n * Lq * Hq) for _, p0, Lq, n in cut)
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    assert p.fwd_workspace >= h["part_rows"] * 129 * 4
    # row terms: sequences apart
    r0 = {}
    at = 0
    for i in range(len(lq)):
        r0[i] = at
        at += -(-lq[i] // tpt) * 128
    assert at == h["term_rows"]
    assert p.bwd_workspace >= (2 * Hkv * at + Hkv * h["slots"] * 2 * 128 * 128) * 4
    rows = 256 // h["dq_ks"]
    assert sorted((d[0], d[1], d[2], d[5]) for d in dq) == sorted(
        (cu_q[i], cu_k[i], r0[i], t) for i in range(len(lq)) for t in range(-(-lq[i] * G // rows)))
    # dK/dV: the tiles that a key block's keys are seen from, each in one segment
    walks, slots = {}, []
    for q0, k0, r, Lq, Lk, kb, first, count, slot in key:
        assert (q0, k0, Lq, Lk) in of
        walks.setdefault((q0, k0, r, kb), []).append((first, count, slot))
        if slot >= 0:
            slots.append(slot)
    assert sorted(slots) == list(range(h["slots"]))
    folds = {(f[0], f[2]): (f[3], f[4]) for f in fold}
    for i in range(len(lq)):
        last = -(-lq[i] // tpt) - 1
        for kb in range(-(-lk[i] // 128)):
            walk = sorted(walks.pop((cu_q[i], cu_k[i], r0[i], kb)), reverse=True)
            tiles = [t for first, count, _ in walk for t in range(first, first - count, -1)]
            need = [t for t in range(last, -1, -1)
                    if _seen(min(lq[i], (t + 1) * tpt) - 1, lq[i], lk[i], causal) > kb * 128]
            assert tiles == need, (i, kb)
            if len(walk) > 1:       # summed in the order of the walk
                assert [s for _, _, s in walk] == list(range(walk[0][2], walk[0][2] + len(walk)))
                assert folds.pop((cu_k[i], kb)) == (walk[0][2], len(walk))
            else:
                assert walk[0][2] == -1
    assert not walks and not folds
    assert [k[7] for k in key] == sorted((k[7] for k in key), reverse=True)
