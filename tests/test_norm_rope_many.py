"""The gradient of the norm's weights over very many rows: its fp32 sums stay short."""

import pytest
import torch

from paper_2602_21196_amd import upipe

D = 128
CHAIN = 1 << 12          # additions of one fp32 sum, to be added in fp64


def test_partial_sums_are_enough():
    """A workgroup has 32 lane groups, each of which adds up to 4096 rows (pairs of heads) to
    a sum; the workspace holds one row of sums a workgroup, of q and of k."""
    for T in (1, 1001, 65536, 1 << 20, 140_000_000, (1 << 31) - 1):
        for H in (1, 2, 7, 64):
            size = upipe.upipe_qk_norm_rope_bwd_workspace_size(T, H, H, D)
            groups = 32 * ((size - 16) // (4 * D)) // 2
            per_group = -(-T * ((H + 1) // 2) // groups) * min(H, 2)
            assert per_group <= CHAIN, (T, H, per_group)


@pytest.mark.gpu
def test_a_long_sum():
    """70 million rows, all alike, at position 0: dw is their number times one row's.  Off by
    the bounds of the norm's other tests: 3e-5 of arithmetic and 2^12 + 8 additions in fp32."""
    dev, T, eps = "cuda:0", 70_000_000, 1e-6
    g = torch.Generator(device=dev).manual_seed(1)
    x, dy = (torch.randn((2, 1, D), device=dev, generator=g).bfloat16() for _ in range(2))
    wq, wk = (1 + 0.3 * torch.randn((2, D), device=dev, generator=g)).unbind()
    q, k, dyq, dyk = (t[i:i + 1].expand(T, 1, D) for t in (x, dy) for i in range(2))
    pos = torch.zeros(T, dtype=torch.int64, device=dev)
    dq, dk, dwq, dwk = upipe.qk_norm_rope_bwd(q, k, wq, wk, pos, 1e4, dyq, dyk, eps)
    torch.cuda.synchronize()
    for i, (dx, dw) in enumerate(((dq, dwq), (dk, dwk))):
        x64 = x[i, 0].double()
        want = T * dy[i, 0].double() * x64 / (x64.square().mean() + eps).sqrt()
        err = float(((dw.double() - want).abs() / want.abs()).max())
        print(f"  {'qk'[i]}: relative {err:.2e}", flush=True)
        assert err <= 3e-5 + 2.0 ** -11
        assert bool((dx == dx[:1]).all())
