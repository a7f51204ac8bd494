"""Gated feed-forward block in bf16 with widths that are multiples of eight and rows that start off 16 bytes: a weight inside a flat
parameter buffer, a row stride of no multiple of eight."""
import math

import pytest
import torch

from test_gpu_block_attention import BF16, HALF_STEP, U32, close, workspace
from test_gpu_gated import act_and_slope, fast

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


def off(t, by, ld=None):
    """t with its first element `by` elements behind a 16-byte boundary, rows of ld."""
    M, n = t.shape
    ld = ld or n
    raw = torch.full((M * ld + 16,), 7.0, dtype=t.dtype, device="cuda")
    v = raw.as_strided((M, n), (ld, 1), by)
    v.copy_(t)
    return v


# which of X, W, dZ, H lie off, and how
LAYOUTS = [("X", 1, 0), ("W", 1, 0), ("W", 4, 0), ("dZ", 1, 0), ("dZ", 0, 3), ("XWdZH", 1, 0), ("XWdZH", 0, 5)]


@pytest.mark.parametrize("shape", [(4, 64, 72), (9, 512, 264), (33, 64, 72), (300, 200, 264), (1000, 512, 520), (257, 2048, 64)])
@pytest.mark.parametrize("which,by,more", LAYOUTS)
def test_values(dp, shape, which, by, more):
    M, K, F = shape
    g = torch.Generator().manual_seed(M + by)
    X, W = torch.randn((M, K), generator=g).bfloat16(), (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).bfloat16()
    dH = torch.randn((M, F), generator=g).bfloat16()
    lie = lambda t, n: off(t, by, t.shape[1] + more) if n in which else off(t, 0)                 # noqa: E731
    x, w, h, dz = lie(X, "X"), lie(W, "W"), lie(torch.zeros((M, F)).bfloat16(), "H"), lie(torch.zeros((M, 2 * F)).bfloat16(), "dZ")
    Z, dX = torch.empty((M, 2 * F), dtype=BF16, device="cuda"), lie(torch.zeros((M, K)).bfloat16(), "X")
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, 1))
    dp.dpclip_gated_forward(x, w, None, h, Z, dp.DPCLIP_ACT_SILU, ws)
    dp.dpclip_gated_backward(dH.cuda(), Z, w, dz, dX, dp.DPCLIP_ACT_SILU, ws)
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    z, mag = X.double() @ W.double().t(), X.double().abs() @ W.double().abs().t()
    d = 2 * (K + 2) * U32 * mag
    close(Z, z, HALF_STEP[BF16] * z.abs() + d)
    zg, zu = z[:, :F], z[:, F:]
    a, _ = act_and_slope(zg, "silu")
    close(h, a * zu, HALF_STEP[BF16] * (a * zu).abs() * 1.01 + 1.2 * (zu.abs() + d[:, F:]) * d[:, :F] + a.abs() * d[:, F:] + fast(BF16, zg) * (zg * zu).abs())
    zs = Z.double().cpu()
    a, slope = act_and_slope(zs[:, :F], "silu")
    want = torch.cat([dH.double() * zs[:, F:] * slope, dH.double() * a], 1)
    close(dz, want, HALF_STEP[BF16] * 1.01 * want.abs() + torch.cat([fast(BF16, zs[:, :F]) * (dH.double() * zs[:, F:]).abs(),
                                                                   fast(BF16, zs[:, :F]) * (dH.double() * zs[:, :F]).abs()], 1))
    got = dz.double().cpu()
    close(dX, got @ W.double(), HALF_STEP[BF16] * (got @ W.double()).abs() * 1.01 + 2 * (2 * F + 2) * U32 * (got.abs() @ W.double().abs()))


def _time(call):
    for _ in range(3):
        call()
    best = 1e9
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(4):
            call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / 4)
    return best


@pytest.mark.parametrize("which", ["X", "W", "dZ", "XWdZ"])
def test_no_cliff(dp, which):
    """The copies cost what they move; the fp32 ALUs would take more than ten times as long as the aligned call."""
    M, K, F = 16384, 512, 2048
    X, W = torch.randn((M, K), device="cuda").bfloat16(), (torch.randn((2 * F, K), device="cuda") / 32).bfloat16()
    dH, Z = torch.randn((M, F), device="cuda").bfloat16(), torch.randn((M, 2 * F), device="cuda").bfloat16()
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, 1))
    H, dX = torch.empty((M, F), dtype=BF16, device="cuda"), torch.empty((M, K), dtype=BF16, device="cuda")

    def pair(shift):
        x, w, dz = off(X, 1 if shift and "X" in which else 0), off(W, 1 if shift and "W" in which else 0), off(Z, 1 if shift and "dZ" in which else 0)

        def call():
            dp.dpclip_gated_forward(x, w, None, H, None, dp.DPCLIP_ACT_SILU, ws)
            dp.dpclip_gated_backward(dH, Z, w, dz, dX, dp.DPCLIP_ACT_SILU, ws)
        return call

    assert _time(pair(True)) <= 3 * _time(pair(False))
