"""Gated feed-forward block: an infinity or a NaN of an operand gives what the formula gives, whatever form the sizes take."""
import math

import pytest
import torch

from test_gpu_block_attention import BF16, CODE, F32, HALF_STEP, U32, close, guarded, workspace

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


# M, K, F: a few rows, fp32 ALUs, planes of fp32 on the tensor cores in 64 and 128 columns, split contractions
SHAPES = [(5, 64, 40), (40, 72, 48), (600, 520, 500), (2000, 70, 1100), (130, 4100, 300), (9500, 200, 520)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("rounded", [True, False])
def test_products(dp, dtype, shape, rounded):
    """rounded: weights as they come from bf16, whose second and third plane are zero."""
    M, K, F = shape
    g = torch.Generator().manual_seed(M + K)
    X, W = torch.randn((M, K), generator=g).to(dtype), (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).to(dtype)
    if rounded:
        X, W = X.bfloat16().to(dtype), W.bfloat16().to(dtype)
    X[1, 3], X[2, K - 1], X[3, 7], X[4, 0], X[4, 1] = INF, -INF, NAN, INF, -INF
    W[2, 5], W[F + 9, K - 2], W[11, 4], W[12, 3], W[13, 3], W[14, 3], W[15, 3] = INF, -INF, NAN, 0.0, 1e-30, -3e38, INF
    z = X.double() @ W.double().t()
    mag = X.double().abs() @ W.double().abs().t()
    H, check_h = guarded((M, F), dtype)
    Z, check_z = guarded((M, 2 * F), dtype)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    dp.dpclip_gated_forward(X.cuda(), W.cuda(), None, H, Z, dp.DPCLIP_ACT_RELU, ws)
    torch.cuda.synchronize()
    check_h(); check_z()
    assert dp.dpclip_read_status(ws) == 0
    tol = (2 * (K + 2) if dtype == BF16 else 48 + math.ceil(K / 64) + 8 + K) * U32 * mag
    # Column 14: -3e38 times what is above one leaves fp32 and is an infinity, which beside another of the opposite sign (rows 1 to 4) is NaN
    far = z.abs() > 3.3e38
    assert bool(torch.isinf(Z.cpu()[5:][z[5:].abs() > 3.5e38]).all())
    keep = ~far | torch.isinf(z)
    keep[1:5, 14] = False
    close(torch.where(keep, Z.cpu().double(), 0.0), torch.where(keep, z, 0.0), torch.where(keep, tol + HALF_STEP[dtype] * z.abs(), 1.0))
    zg, zu = Z.cpu().double()[:, :F], Z.cpu().double()[:, F:]
    h = torch.where(zg < 0, 0.0, zg) * zu
    odd = ~(torch.isfinite(zg) & torch.isfinite(zu))
    got = H.cpu().double()
    assert torch.equal(got[odd].nan_to_num(nan=7.0), h[odd].nan_to_num(nan=7.0))
    assert bool(torch.isfinite(got[5:, 16:F]).all())                          # rows and columns without one


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dp, dtype, shape):
    M, K, F = shape
    g = torch.Generator().manual_seed(M * 7 + K)
    Z, dH = torch.randn((M, 2 * F), generator=g).to(dtype), torch.randn((M, F), generator=g).to(dtype)
    W = (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).bfloat16().to(dtype)
    Z[1:5, :F] = Z[1:5, :F].abs() + 0.5                                       # relu is the identity there
    dH[1, 3], dH[2, F - 1], dH[3, 7], dH[4, 0], dH[4, 1] = INF, -INF, NAN, INF, -INF
    W[:, 2] = 0.0
    W[6, 3], W[F + 8, 4] = INF, NAN
    dZ, check_z = guarded((M, 2 * F), dtype)
    dX, check_x = guarded((M, K), dtype)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    dp.dpclip_gated_backward(dH.cuda(), Z.cuda(), W.cuda(), dZ, dX, dp.DPCLIP_ACT_RELU, ws)
    torch.cuda.synchronize()
    check_z(); check_x()
    assert dp.dpclip_read_status(ws) == 0
    z, dh = Z.double(), dH.double()
    want = torch.cat([dh * z[:, F:] * (z[:, :F] > 0), dh * torch.where(z[:, :F] > 0, z[:, :F], 0.0)], 1)
    close(dZ, want, 4 * HALF_STEP[dtype] * want.abs().nan_to_num(posinf=0.0))
    got = dZ.double().cpu()
    dx, mag = got @ W.double(), got.abs() @ W.double().abs()
    close(dX, dx, (HALF_STEP[dtype] * dx.abs() + (2 * (2 * F + 2) + 100) * U32 * mag).nan_to_num(posinf=0.0))
