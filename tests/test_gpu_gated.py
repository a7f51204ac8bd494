"""Gated feed-forward block: the kernels against their formulas in 64 bits on the CPU.

Tolerances.  A product of K terms summed in fp32, in any order, is off by at most K units of 2^-24 of the sum of its terms' magnitudes; the
tensor cores cut off what they shift out where the ALUs round, so twice that.  An output rounded to bf16 is off by 2^-8 of its value, to
fp32 by 2^-24.  The activations' slopes are at most 1.2; the fast exponential and division of bf16 calls are off by 2^-22 times the
argument's size, the exact ones of fp32 calls by a few 2^-24; the slope of gelu_tanh multiplies 1 - p by z + 0.13 z^3.
"""
import math

import pytest
import torch

from test_gpu_block_attention import BF16, CODE, F32, HALF_STEP, U32, close, guarded, workspace

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


def code(dp, act):
    return getattr(dp, "DPCLIP_ACT_" + act.upper())


def act_and_slope(z, act):
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p + z * p * (1 - p)
    if act == "relu":
        return torch.where(z > 0, z, 0.0), (z > 0).double()
    if act == "gelu":
        c = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * c, c + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    p = 1 / (1 + torch.exp(-2 * k * (z + 0.044715 * z ** 3)))
    return z * p, p + 2 * k * z * (1 + 3 * 0.044715 * z * z) * p * (1 - p)


def fast(dtype, z):
    """What the activation may be off by, relative to |z| (value) or 1 (slope)."""
    a = z.abs()
    return (4 + 4 * a + 2 * a ** 3) * (2.0 ** -22 if dtype == BF16 else 4 * U32)


def rows(t, layout, dtype):
    """(M, n) on the device: dense, in longer aligned rows, or at odd addresses."""
    M, n = t.shape
    ld = n if layout == "dense" else (n + 23) // 8 * 8 if layout == "aligned" else n + 3
    raw = torch.full((M * ld + 16,), float("nan"), dtype=dtype, device="cuda")
    dev = raw.as_strided((M, n), (ld, 1), 1 if layout == "odd" else 0)
    dev.copy_(t)
    return dev


FWD = [
    # M, K, F
    (1, 1, 1), (1, 64, 64), (3, 100, 37), (8, 520, 200), (9, 64, 8), (33, 72, 130), (40, 17, 19),
    (256, 64, 128), (300, 200, 264), (257, 1000, 72), (1000, 96, 520), (64, 2048, 128), (16, 4096, 64),
    (700, 333, 161), (130, 64, 1000),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", FWD)
@pytest.mark.parametrize("layout,act,with_bias,keep", [("dense", "silu", False, True), ("aligned", "gelu_tanh", True, True), ("odd", "gelu", True, True),
                                                       ("dense", "relu", True, False)])
def test_forward(dp, dtype, shape, layout, act, with_bias, keep):
    M, K, F = shape
    g = torch.Generator().manual_seed(M + K + F)
    X, W = torch.randn((M, K), generator=g).to(dtype), (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).to(dtype)
    bias = 0.5 * torch.randn((2 * F,), generator=g) if with_bias else None
    x, w = X.double(), W.double()
    z = x @ w.t() + (bias.double() if with_bias else 0)
    mag = x.abs() @ w.abs().t() + (bias.double().abs() if with_bias else 0)
    zg, zu = z[:, :F], z[:, F:]
    a, _ = act_and_slope(zg, act)
    ldh = F if layout == "dense" else (F + 15) // 8 * 8 if layout == "aligned" else F + 1
    H, check_h = guarded((M, F), dtype, strides=(ldh, 1), tail=64 if layout != "odd" else 65)
    Z, check_z = guarded((M, 2 * F), dtype, strides=(2 * F + (8 if layout == "aligned" else 0), 1))
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    dev = (rows(X, layout, dtype), rows(W, layout, dtype), None if bias is None else bias.cuda())
    dp.dpclip_gated_forward(*dev, H, Z if keep else None, code(dp, act), ws)
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    check_h(); check_z()
    dz = 2 * (K + 2) * U32 * mag
    if keep:
        close(Z, z, HALF_STEP[dtype] * z.abs() + dz)
    else:
        assert bool((Z == 0.5).all())
    dg, du = dz[:, :F], dz[:, F:]
    close(H, a * zu, HALF_STEP[dtype] * (a * zu).abs() * 1.01 + 1.2 * (zu.abs() + du) * dg + a.abs() * du + fast(dtype, zg) * zg.abs() * zu.abs() + 1e-37)
    first = H.clone()
    dp.dpclip_gated_forward(*dev, H, Z if keep else None, code(dp, act), ws)
    assert torch.equal(first, H)                                   # the same bits again


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", FWD)
@pytest.mark.parametrize("layout,act", [("dense", "silu"), ("aligned", "gelu_tanh"), ("odd", "gelu"), ("dense", "relu")])
def test_backward(dp, dtype, shape, layout, act):
    M, K, F = shape
    g = torch.Generator().manual_seed(M * 3 + K + F)
    Z, dH = (2 * torch.randn((M, 2 * F), generator=g)).to(dtype), torch.randn((M, F), generator=g).to(dtype)
    Z[0, 0] = 0.0                                                  # relu' at 0
    W = (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).to(dtype)
    z, dh = Z.double(), dH.double()
    zg, zu = z[:, :F], z[:, F:]
    a, slope = act_and_slope(zg, act)
    dev = rows(dH, layout, dtype), rows(Z, layout, dtype), rows(W, layout, dtype)
    ldz = 2 * F if layout == "dense" else (2 * F + 15) // 8 * 8 if layout == "aligned" else 2 * F + 1
    ldx = K if layout == "dense" else (K + 15) // 8 * 8 if layout == "aligned" else K + 1
    dZ, check_z = guarded((M, 2 * F), dtype, strides=(ldz, 1), tail=64 if layout != "odd" else 65)
    dX, check_x = guarded((M, K), dtype, strides=(ldx, 1), tail=64 if layout != "odd" else 65)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    dp.dpclip_gated_backward(*dev, dZ, dX, code(dp, act), ws)
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    check_z(); check_x()
    want = torch.cat([dh * zu * slope, dh * a], 1)
    off = torch.cat([fast(dtype, zg) * (dh * zu).abs(), fast(dtype, zg) * (dh * zg).abs()], 1)
    close(dZ, want, HALF_STEP[dtype] * 1.01 * want.abs() + off + 1e-37)
    got, w = dZ.double().cpu(), W.double()
    dx = got @ w                                                   # the product with dZ as stored
    close(dX, dx, HALF_STEP[dtype] * dx.abs() * 1.01 + 2 * (2 * F + 2) * U32 * (got.abs() @ w.abs()))
    first = dX.clone()
    dp.dpclip_gated_backward(dev[0], dev[1], None, dev[1], None, code(dp, act), ws)     # in place of Z, without dX
    assert torch.equal(dev[1], dZ)
    dp.dpclip_gated_backward(dev[0], rows(Z, layout, dtype), dev[2], dZ, dX, code(dp, act), ws)
    assert torch.equal(first, dX)


@pytest.mark.parametrize("act", ACTS)
def test_extreme_preactivations(dp, act):
    """Far out the activations are 0 or z, their slopes 0 or 1, without a NaN on the way."""
    z = torch.tensor([-3e4, -200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 200.0, 3e4])
    for dtype in (BF16, F32):
        M, F = z.numel(), 8
        Z = torch.ones((M, 2 * F)).to(dtype)
        Z[:, :F] = z[:, None].to(dtype)
        dH = torch.ones((M, F)).to(dtype)
        dZ = torch.empty((M, 2 * F), dtype=dtype, device="cuda")
        ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, 8, F, CODE[dtype]))
        dp.dpclip_gated_backward(dH.cuda(), Z.cuda(), None, dZ, None, code(dp, act), ws)
        got = dZ.double().cpu()
        v = Z[:, :F].double()
        a, slope = torch.where(v > 0, v, 0.0), (v > 0).double()
        far = v.abs() >= 20
        # exp(-20) = 2e-9, times 3 z^2 at most
        assert float((got[:, :F] - slope)[far].abs().max()) <= 1e-5 and float((got[:, F:] - a)[far].abs().max()) <= 1e-5


@pytest.mark.parametrize("act", ACTS)
def test_products_that_would_overflow(dp, act):
    """act(zg) zu where zg zu leaves fp32: zero for the activations that vanish there."""
    M, K, F = 300, 64, 64                                          # the tensor-core form
    X = torch.zeros((M, K)); X[:, 0] = 2.0 ** 40
    W = torch.zeros((2 * F, K)); W[:F, 0] = -2.0 ** 30; W[F:, 0] = 2.0 ** 30
    for dtype in (BF16, F32):
        ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
        H = torch.empty((M, F), dtype=dtype, device="cuda")
        dp.dpclip_gated_forward(X.to(dtype).cuda(), W.to(dtype).cuda(), None, H, None, code(dp, act), ws)
        assert bool((H == 0).all())


def test_against_differences(dp):
    """dX against directional differences of the forward pass in fp32; dW of the step against those of W."""
    B, T, K, F = 3, 7, 12, 10
    g = torch.Generator().manual_seed(4)
    X, W = torch.randn((B, T, K), generator=g).cuda(), (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).cuda()
    dH = torch.randn((B, T, F), generator=g).cuda()
    bias = torch.randn((2 * F,), generator=g).cuda()
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(B * T, K, F, 0))
    H, Z, dZ, dX = (torch.empty((B, T, n), device="cuda") for n in (F, 2 * F, 2 * F, K))
    for act in ACTS[:3]:                                           # relu has a kink

        def loss(X, W, bias):
            dp.dpclip_gated_forward(X, W, bias, H, None, code(dp, act), ws)
            return (H.double() * dH.double()).sum((1, 2)).cpu()

        dp.dpclip_gated_forward(X, W, bias, H, Z, code(dp, act), ws)
        dp.dpclip_gated_backward(dH, Z, W, dZ, dX, code(dp, act), ws)
        gW, gb = torch.empty((2 * F, K), device="cuda"), torch.empty(2 * F, device="cuda")
        ws2 = workspace(dp, dp.dpclip_workspace_bytes(B, T, K, 2 * F))
        dp.dpclip_clipped_grad(X, dZ, None, gW, gb, ws2)
        h = 2.0 ** -8
        mag = float(dH.abs().sum()) * 4
        tol = mag * (20 * U32 / h + 20 * h * h)                    # rounding over 2 h; third derivatives of a few units times h^2
        for grad, at in ((dX, 0), (gW, 1), (gb, 2)):
            v = torch.randn(grad.shape, generator=torch.Generator().manual_seed(at)).cuda()
            args = [[X, W, bias], [X, W, bias]]
            args[0][at] = args[0][at] + h * v
            args[1][at] = args[1][at] - h * v
            diff = float((loss(*args[0]) - loss(*args[1])).sum()) / (2 * h)
            assert abs(diff - float((grad.double() * v.double()).sum())) <= tol, (act, at)


@pytest.mark.parametrize("dtype,shape", [(BF16, (4, 96, 64, 128)), (F32, (5, 20, 30, 44))])
def test_block_in_one_step(dp, dtype, shape):
    """Forward, backward and the step over the block's weight as ONE layer of 2F outputs: its norms, factors and clipped sum against
    per-example gradients in 64 bits; then recorded and replayed with other inputs in the same buffers, on a stream of its own."""
    B, T, K, F = shape
    g = torch.Generator().manual_seed(9)
    X = torch.randn((B, T, K), generator=g).to(dtype).cuda()
    W = (torch.randn((2 * F, K), generator=g) / math.sqrt(K)).to(dtype).cuda()
    dH = (0.02 * torch.randn((B, T, F), generator=g)).to(dtype).cuda()
    H, Z, dZ, dX = (torch.empty((B, T, n), dtype=dtype, device="cuda") for n in (F, 2 * F, 2 * F, K))
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(B * T, K, F, CODE[dtype]))
    plan = dp.StepPlan([dp.Layer(X, dZ, True)])

    def step(C):
        dp.dpclip_gated_forward(X, W, None, H, Z, dp.DPCLIP_ACT_SILU, ws)
        dp.dpclip_gated_backward(dH, Z, W, dZ, dX, dp.DPCLIP_ACT_SILU, ws)
        plan.run(C=C, sigma=0.0, seed=1)

    def check(C):
        x, w, dh = X.double().cpu(), W.double().cpu(), dH.double().cpu()
        z = x @ w.t()
        a, slope = act_and_slope(z[..., :F], "silu")
        dz = torch.cat([dh * z[..., F:] * slope, dh * a], -1)
        G, gb = torch.einsum("bto,bti->boi", dz, x), dz.sum(1)
        n = torch.sqrt(G.square().sum((1, 2)) + gb.square().sum(1))
        c = torch.clamp(C / n, max=1.0)
        # bf16: Z and dZ are rounded, 2^-8 each, against the exact ones here; the path's own tolerance is 1e-2
        tol = 2e-5 if dtype == F32 else 1.5e-2
        assert float(((plan.norms.double().cpu() - n) / n).abs().max()) <= tol
        want = torch.einsum("b,boi->oi", c, G)
        assert float((plan.gW[0].double().cpu() - want).norm() / want.norm()) <= tol
        assert float((plan.gb[0].double().cpu() - (c[:, None] * gb).sum(0)).norm() / gb.sum(0).norm()) <= 2 * tol
        return n

    step(1.0)
    torch.cuda.synchronize()
    n = check(1.0)
    C = float(n.median())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(C)
    X.copy_(torch.randn((B, T, K), generator=g).to(dtype))
    graph.replay()
    torch.cuda.synchronize()
    check(C)
    assert dp.dpclip_read_status(ws) == 0


@pytest.mark.parametrize("shape", [(600, 520, 500), (257, 1301, 460), (2000, 70, 1100), (130, 4100, 300), (90, 200, 8500), (5000, 64, 480)])
@pytest.mark.parametrize("layout,with_bias", [("dense", True), ("odd", False), ("aligned", False)])
def test_fp32_products_in_planes(dp, shape, layout, with_bias):
    """Large fp32 calls: products of three bf16 planes each.  A window of 64 columns has 24 additions, each cut off (two units of 2^-24 of
    what the window adds up); the windows are added up with rounding; the products left out are two more units."""
    M, K, F = shape
    g = torch.Generator().manual_seed(M + K)
    X, W = torch.randn((M, K), generator=g), torch.randn((2 * F, K), generator=g) / math.sqrt(K)
    bias = torch.randn((2 * F,), generator=g) if with_bias else None
    x, w = X.double(), W.double()
    z = x @ w.t() + (bias.double() if with_bias else 0)
    mag = x.abs() @ w.abs().t() + (bias.double().abs() if with_bias else 0)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, 0))
    pad = {"dense": 0, "odd": 1, "aligned": 4}[layout]
    H, check_h = guarded((M, F), F32, strides=(F + pad, 1))
    Z, check_z = guarded((M, 2 * F), F32, strides=(2 * F + pad, 1))
    dev = rows(X, layout, F32), rows(W, layout, F32)
    dp.dpclip_gated_forward(*dev, None if bias is None else bias.cuda(), H, Z, dp.DPCLIP_ACT_GELU, ws)
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    check_h(); check_z()
    tol = (48 + math.ceil(K / 64) + 8) * U32 * mag
    close(Z, z, tol + U32 * z.abs())
    a, _ = act_and_slope(z[:, :F], "gelu")
    zu, dg, du = z[:, F:], tol[:, :F], tol[:, F:]
    close(H, a * zu, U32 * 1.01 * (a * zu).abs() + 1.2 * (zu.abs() + du) * dg + a.abs() * du + fast(F32, z[:, :F]) * (z[:, :F] * zu).abs() + 1e-37)
    dH = torch.randn((M, F), generator=g)
    dZ, check_z = guarded((M, 2 * F), F32, strides=(2 * F + pad, 1))
    dX, check_x = guarded((M, K), F32, strides=(K + pad, 1))
    dp.dpclip_gated_backward(rows(dH, layout, F32), Z, dev[1], dZ, dX, dp.DPCLIP_ACT_GELU, ws)
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    check_z(); check_x()
    got = dZ.double().cpu()
    dx = got @ w
    # a split contraction adds up to 32 partial products more
    close(dX, dx, (48 + math.ceil(2 * F / 64) + 40) * U32 * (got.abs() @ w.abs()) + U32 * dx.abs())
    # an infinity or a NaN of an input does not get lost
    X[3, 5] = float("inf"); X[7, 2] = float("nan")
    dp.dpclip_gated_forward(rows(X, layout, F32), dev[1], None, H, Z, dp.DPCLIP_ACT_GELU, ws)
    bad = ~torch.isfinite(Z)
    assert bool(bad[3].all()) and bool(bad[7].all()) and not bool(bad[8].any()) and not bool(bad[2].any())


@pytest.mark.parametrize("M,K,F,act,in_place", [(9473, 1024, 1800, "silu", False), (9728, 1000, 2048, "gelu_tanh", True), (40000, 256, 424, "gelu", False),
                                                (38000, 264, 520, "relu", True)])
def test_backward_large(dp, M, K, F, act, in_place):
    """Many tiles: every row of both outputs, twice, and as a recorded graph on a stream of its own with other inputs in the same
    buffers."""
    g = torch.Generator(device="cuda").manual_seed(M)
    Z = (2 * torch.randn((M, 2 * F), generator=g, device="cuda")).bfloat16()
    dH, W = torch.randn((M, F), generator=g, device="cuda").bfloat16(), (torch.randn((2 * F, K), generator=g, device="cuda") / math.sqrt(K)).bfloat16()
    dZ, check_z = guarded((M, 2 * F), BF16)
    dX, check_x = guarded((M, K), BF16)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, 1))
    run = lambda: dp.dpclip_gated_backward(dH, dZ if in_place else Z, W, dZ, dX, code(dp, act), ws)        # noqa: E731

    def verify():
        check_z(); check_x()
        for r in range(0, M, 4096):                                # in pieces: 64 bits of everything would be several GB
            z, dh = Z[r:r + 4096].double(), dH[r:r + 4096].double()
            zg, zu = z[:, :F], z[:, F:]
            a, slope = act_and_slope(zg, act)
            want = torch.cat([dh * zu * slope, dh * a], 1)
            off = torch.cat([fast(BF16, zg) * (dh * zu).abs(), fast(BF16, zg) * (dh * zg).abs()], 1)
            got = dZ[r:r + 4096].double()
            close(got, want.cpu(), (HALF_STEP[BF16] * 1.01 * want.abs() + off + 1e-37).cpu())
            dx = got @ W.double()
            close(dX[r:r + 4096], dx.cpu(), (HALF_STEP[BF16] * dx.abs() * 1.01 + 2 * (2 * F + 2) * U32 * (got.abs() @ W.double().abs())).cpu())

    if in_place:
        dZ.copy_(Z)
    run()
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    verify()
    first, first_x = dZ.clone(), dX.clone()
    dX.fill_(0.5)
    if in_place:
        dZ.copy_(Z)
    run()
    assert torch.equal(first, dZ) and torch.equal(first_x, dX)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    if in_place:
        dZ.copy_(Z)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        run()
    dH.mul_(-0.5)
    for _ in range(2):
        if in_place:
            dZ.copy_(Z)
        graph.replay()
    torch.cuda.synchronize()
    verify()
    assert torch.equal(dX, first_x * -0.5) and dp.dpclip_read_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_two_streams_at_once(dp, dtype):
    """Calls on two streams, each with outputs and a workspace of its own, interleaved: the bits of the calls one after the other."""
    M, K, F = 2000, 256, 520
    sides = []
    for k in range(2):
        g = torch.Generator(device="cuda").manual_seed(k)
        X, W = torch.randn((M, K), generator=g, device="cuda").to(dtype), (torch.randn((2 * F, K), generator=g, device="cuda") / 16).to(dtype)
        out = [torch.empty((M, n), dtype=dtype, device="cuda") for n in (F, 2 * F, 2 * F, K)]
        sides.append((X, W, out, workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype])), torch.cuda.Stream()))

    def run(X, W, out, ws, stream):
        dp.dpclip_gated_forward(X, W, None, out[0], out[1], dp.DPCLIP_ACT_SILU, ws, stream=stream)
        dp.dpclip_gated_backward(out[0], out[1], W, out[2], out[3], dp.DPCLIP_ACT_SILU, ws, stream=stream)

    want = []
    for s in sides:
        run(*s[:4], None)
        want.append([t.clone() for t in s[2]])
    torch.cuda.synchronize()
    for _ in range(5):
        for s in sides:
            run(*s)
    torch.cuda.synchronize()
    for s, w in zip(sides, want):
        assert all(torch.equal(a, b) for a, b in zip(s[2], w)) and dp.dpclip_read_status(s[3]) == 0


@pytest.mark.parametrize("shape", [(1, 24, 4003), (3, 40, 5008), (5, 16, 1031), (40, 24, 2049)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_backward_few_long_rows(dp, dtype, shape, layout):
    test_backward(dp, dtype, shape, layout, "gelu_tanh")


@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_fp32_silu_over_its_range(dp, layout):
    """silu and its slope from z alone (dh = u = 1), against 64 bits.

    In units of 2^-24: the exponential is off by 4, the addition of 1 and Newton's step by 1 each and the square of the reciprocal's 2^-22 is
    nothing, so p = sigmoid(z) is off by 6 p, z p by 7 |z| p.  The slope p (1 + z (1 - p)): 1 - p is off by 1 + 6 p, so the bracket by
    |z| (1 + 6 p) + 1 + |z|, the product by 7 (1 + |z|) p more: at most 16 (1 + |z|) p together.  Below 2^-126 p is zero: z p is then off by
    88 x 2^-126.
    """
    z = torch.cat([torch.linspace(-120, 120, 60001), torch.linspace(-2, 2, 4000), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e30])]).float()
    M, F = 1, z.numel()
    Z = rows(torch.stack([z, torch.ones_like(z)]).reshape(1, 2 * F), layout, F32)
    dH, dZ = rows(torch.ones((M, F)), layout, F32), rows(torch.zeros((M, 2 * F)), layout, F32)
    dp.dpclip_gated_backward(dH, Z, None, dZ, None, dp.DPCLIP_ACT_SILU, workspace(dp, dp.dpclip_gated_workspace_bytes(M, 8, F, CODE[F32])))
    got = dZ.cpu().double().reshape(2, F)
    z = z.double()
    p = 1 / (1 + torch.exp(-z))
    tiny = 88 * 2.0 ** -126
    assert ((got[1] - z * p).abs() <= 7 * U32 * z.abs() * p + tiny).all()
    slope = p * (1 + z * (1 - p))
    assert ((got[0] - slope).abs() <= 16 * U32 * (1 + z.abs()) * p + tiny).all()
    # a NaN stays one, an infinity gives what the formula gives
    ends = rows(torch.tensor([[float("nan"), float("inf"), -float("inf"), 1.0, 1.0, 1.0]]), layout, F32)
    dZ = rows(torch.zeros((1, 6)), layout, F32)
    dp.dpclip_gated_backward(rows(torch.ones((1, 3)), layout, F32), ends, None, dZ, None, dp.DPCLIP_ACT_SILU, workspace(dp, dp.dpclip_gated_workspace_bytes(1, 8, 3, CODE[F32])))
    value = dZ.cpu()[0, 3:]
    assert value[0].isnan() and value[1] == float("inf") and value[2].isnan()


def test_expanded_workspace_and_flags_without_a_truth_value_are_refused(dp):
    """By the host, before a launch."""
    t = lambda *s: torch.zeros(s, device="cuda")                              # noqa: E731
    ws = torch.zeros((1,), dtype=torch.uint8, device="cuda").expand(1 << 24)
    with pytest.raises(ValueError, match="workspace"):
        dp.dpclip_gated_backward(t(4, 8), t(4, 16), t(16, 8), t(4, 16), t(4, 8), dp.DPCLIP_ACT_SILU, ws)
    with pytest.raises(TypeError, match="truth"):
        dp.dpclip_relbias_forward(t(8, 1), t(1, 4, 4), 64, bidirectional=torch.zeros(2))


@pytest.mark.parametrize("shape", [(300, 1024, 161), (257, 2000, 30), (64, 1030, 1001), (513, 4097, 66)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_split_contractions_with_ragged_ends(dp, dtype, shape, layout):
    M, K, F = shape
    test_forward(dp, dtype, shape, layout, "silu", True, True)
    test_backward(dp, dtype, (M, F, K // 2), layout, "silu")
