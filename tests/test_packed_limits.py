"""The largest calls that the header allows, and the first that it does not: a launch counts
its threads in 32 bits."""

import ctypes
import time

from paper_2602_21196_amd import upipe

D = 128


def _plan(n, Hq, Hkv):
    cu = (ctypes.c_int64 * (n + 1))(*range(n + 1))
    return upipe.upipe_varlen_plan_size(cu, cu, n, Hq, Hkv, D, 1)


def _decode(B, nq, Hq, Hkv, P=0):
    return upipe.upipe_attn_decode_workspace_size(B, nq, 16, P, Hq, Hkv, D)


def test_sequences_times_heads():
    """Tiles of rows of one key/value head each: below 2^23."""
    assert _plan((1 << 17) - 1, 64, 64) > 0 and _plan(1 << 17, 64, 64) == 0
    assert _plan(1 << 17, 64, 32) > 0


def test_rows_of_caches():
    """B nq Hq below 2^23, with a prefix below 2^22 - 4096."""
    assert _decode(65535, 2, 64, 8) > 0 and _decode(65536, 2, 64, 8) == 0
    assert _decode(65536, 1, 64, 8) > 0
    assert _decode(65471, 1, 64, 8, P=1) > 0 and _decode(65472, 1, 64, 8, P=1) == 0


def test_lengths_beyond_any_launch_are_refused_at_once():
    """4096 sequences of the longest length, and keys alone: no list of their work is made
    first (of 16 million tiles a sequence, some terabytes)."""
    most = (1 << 24) - 128
    long = [most * i for i in range(4097)]
    none = [0] * 4097
    for cu_q, cu_k, Hq in ((long, long, 64), (none, long, 64), (long, none, 1)):
        q, k = ((ctypes.c_int64 * 4097)(*c) for c in (cu_q, cu_k))
        start = time.process_time()
        assert upipe.upipe_varlen_plan_size(q, k, 4096, Hq, 1, D, 1) == 0
        assert time.process_time() - start < 0.1
