"""Layouts of gradients that share no element, however the rows of two tensors lie between
each other, against a list of all elements; and those that do share some."""

import pytest

from paper_2602_21196_amd import upipe

FAKE, D = 1 << 30, 128
T, H = 5, 3          # of dk and dv; q has 2 H heads


def _at(offset, row, head):
    return upipe.upipe_heads(6 * FAKE + 2 * offset, row, head)


def _rows(offset, row, head):
    return {offset + t * row + h * head for t in range(T) for h in range(H)}


def _bwd(dk, dv):
    plan = upipe.VarlenPlan([0, T], Hq=2 * H, Hkv=H, device="cpu")

    def dense(n, heads):
        return upipe.upipe_heads(n * FAKE, heads * D, D)
    return upipe.upipe_attn_bwd_varlen(
        dense(1, 2 * H), dense(2, H), dense(3, H), dense(4, 2 * H), FAKE, T, dense(5, 2 * H),
        dense(10, 2 * H), dk, dv, plan.host, FAKE, FAKE, 0, None)


LAYOUTS = {  # (offset, row, head) of dk, of dv
    "columns [T, 2H, d]": ((0, 2 * H * D, D), (H * D, 2 * H * D, D)),
    "beside in every head [T, H, 2, d]": ((0, 2 * H * D, 2 * D), (D, 2 * H * D, 2 * D)),
    "head-major [2, H, T, d]": ((0, D, T * D), (H * T * D, D, T * D)),
    "head-major, beside in every row [H, T, 2, d]": ((0, 2 * D, 2 * T * D), (D, 2 * D, 2 * T * D)),
    "head-major, behind in every head [H, 2, T, d]": ((0, D, 2 * T * D), (T * D, D, 2 * T * D)),
    "the second first": ((T * D, D, 2 * T * D), (0, D, 2 * T * D)),
    "three to a row [H, T, 3, d]": ((2 * D, 3 * D, 3 * T * D), (D, 3 * D, 3 * T * D)),
    "rows with a gap": ((0, 1024, 256), (128, 1024, 256)),
}
SHARED = {
    "the same": ((0, H * D, D), (0, H * D, D)),
    "half a row on": ((0, 2 * D, 2 * T * D), (64, 2 * D, 2 * T * D)),
    "one head common": ((0, 2 * H * D, D), ((H - 1) * D, 2 * H * D, D)),
    "the last head in the next row": ((0, 2 * H * D, D), ((H + 1) * D, 2 * H * D, D)),
    "one row common": ((0, D, 2 * T * D), ((T - 1) * D, D, 2 * T * D)),
    "strides of different grids": ((0, 2 * D, 2 * T * D), (D, 3 * D, 3 * T * D)),
}


@pytest.mark.parametrize("name", [*LAYOUTS, *SHARED])
def test_rows_between_each_other(name):
    dk, dv = {**LAYOUTS, **SHARED}[name]
    share = any(abs(a - b) < D for a in _rows(*dk) for b in _rows(*dv))
    assert share == (name in SHARED)
    # -3: valid but for the workspace
    assert _bwd(_at(*dk), _at(*dv)) == (-1 if share else -3)
