"""The forms of the transformer-block kernels that serve long calls: walks of several blocks that wrap, rings of copies, several tiles for every
pair of CTAs; and every call under the switches that change its launches.  References in 64 bits, on the GPU where they are large.  Tolerances
as in test_gpu_block_attention.py and test_gpu_gated.py."""
import math

import pytest
import torch

from test_block_operators_refusals import bucket_of
from test_gpu_block_attention import BF16, CODE, F32, HALF_STEP, U32, close, guarded, qk_reference, workspace
from test_gpu_gated import act_and_slope, code, fast, rows
from test_gpu_gated import test_backward as gated_backward_case
from test_gpu_gated import test_forward as gated_forward_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


# ---------------------------------------------------------------------------------------------------------------
# relative position bias
# ---------------------------------------------------------------------------------------------------------------
def buckets(Tq, Tk, off, nb, D, both):
    """bucket of (q, k) on the GPU, by whole numbers of the distance"""
    first = -(off + Tq - 1)
    line = torch.tensor([bucket_of(max(-D, min(D, r)), nb, D, both) for r in range(first, Tk - off)], device="cuda")
    at = torch.arange(Tk, device="cuda")[None] - (off + torch.arange(Tq, device="cuda")[:, None]) - first
    return line[at]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Tq,Tk,off,both,causal", [(16, 1000, 1000, 0, True, False), (16, 1000, 1008, 8, False, True), (16, 2048, 2048, 0, True, True),
                                                     (5, 3001, 2999, 0, False, False), (40, 1500, 232, 0, True, False)])
@pytest.mark.parametrize("heads_inside", [False, True])
def test_bias_of_long_walks(dp, dtype, H, Tq, Tk, off, both, causal, heads_inside):
    nb, D = 32, 100
    table = torch.randn((nb, H), generator=torch.Generator().manual_seed(7)).cuda()
    out, check = guarded((H, Tq, Tk), dtype, strides=(Tk, H * Tk, 1) if heads_inside else (Tq * Tk, Tk, 1))
    dp.dpclip_relbias_forward(table, out, D, both, causal, off)
    torch.cuda.synchronize()
    check()
    at = buckets(Tq, Tk, off, nb, D, both)
    above = torch.arange(Tk, device="cuda")[None] > torch.arange(Tq, device="cuda")[:, None] + off
    for h in range(H):
        want = table[:, h].to(dtype)[at]                            # one rounding, the same for every place
        assert torch.equal(out[h], torch.where(above, -math.inf, want) if causal else want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,H,Tq,Tk,nb", [(64, 8, 256, 256, 32), (128, 8, 256, 256, 32), (200, 8, 600, 40, 16), (24, 16, 512, 264, 32), (150, 8, 300, 77, 32),
                                          (3, 4, 1000, 2100, 64), (200, 6, 130, 3, 8)])
@pytest.mark.parametrize("padded,causal", [(False, False), (True, False), (False, True), (True, True)])
def test_table_gradient_of_long_walks(dp, dtype, B, H, Tq, Tk, nb, padded, causal):
    g = torch.Generator(device="cuda").manual_seed(B + Tq)
    dS = torch.randn((B, H, Tq, Tk), generator=g, device="cuda", dtype=dtype)
    q, k = torch.arange(Tq, device="cuda")[:, None], torch.arange(Tk, device="cuda")[None]
    off = max(0, Tk - Tq) if causal else 0
    ql = kl = None
    counts = torch.ones((B, Tq, Tk), dtype=torch.bool, device="cuda")
    if padded:
        ql, kl = (torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32) for n in (Tq, Tk))
        ql[0], kl[0], ql[1] = Tq, Tk, 0
        counts &= (q[None] < ql[:, None, None]) & (k[None] < kl[:, None, None])
    if causal:
        counts &= (k <= q + off)[None]
    dS.masked_fill_(~counts[:, None], float("nan"))
    grads, check_g = guarded((B, nb, H), F32)
    sq, check_s = guarded((B,), F32)
    ws = workspace(dp, dp.dpclip_relbias_workspace_bytes(B, H, Tq, Tk, nb, CODE[dtype]))
    how = dict(max_distance=100, bidirectional=True, causal=causal, q_offset=off, q_lens=ql, k_lens=kl)
    dp.dpclip_relbias_sqnorms(dS, grads, sq, ws, **how)
    torch.cuda.synchronize()
    check_g(); check_s()
    one = torch.nn.functional.one_hot(buckets(Tq, Tk, off, nb, 100, True).flatten(), nb).double()
    G, A = torch.empty((B, nb, H), dtype=torch.float64), torch.empty((B, nb, H), dtype=torch.float64)
    for i in range(B):
        x = torch.where(counts[i], dS[i].double(), 0.0).flatten(1)
        G[i], A[i] = (x @ one).t().cpu(), (x.abs() @ one).t().cpu()
    depth = 700 * U32                                               # 256 additions of a walk, the folds behind it fewer than 400
    close(grads, G, depth * A)
    close(sq, G.square().sum((1, 2)), (2 * depth * A * G.abs() + (depth * A) ** 2).sum((1, 2)) + (nb * H + 8) * U32 * G.square().sum((1, 2)))
    first = grads.clone()
    dp.dpclip_relbias_sqnorms(dS, grads, sq, ws, **how)
    assert torch.equal(first, grads)


# ---------------------------------------------------------------------------------------------------------------
# norms of queries and keys
# ---------------------------------------------------------------------------------------------------------------
LONG_QK = [
    # B, T, Hq, Hk, D, rot, interleaved: at least 64 x 148 tokens' blocks of heads in both types, rings of copies
    (6, 900, 17, 3, 32, 32, False), (40, 250, 9, 2, 64, 64, False), (5, 1000, 9, 5, 64, 32, True), (70, 70, 5, 2, 128, 128, True), (3, 1111, 7, 1, 128, 64, False),
    (2, 1000, 5, 3, 256, 256, False), (3, 1600, 3, 0, 160, 96, True), (2, 2500, 2, 1, 512, 512, False), (3, 3300, 8, 1, 16, 16, False), (1, 5000, 4, 2, 96, 0, False),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", LONG_QK)
@pytest.mark.parametrize("positions", ["listed", "from 0", "from 37"])
def test_rings(dp, dtype, case, positions):
    """Positions in a list, with padding anywhere, or pos0 + t, the last five behind the table."""
    B, T, Hq, Hk, D, rot, inter = case
    g = torch.Generator(device="cuda").manual_seed(T)
    pos0 = 37 if positions == "from 37" else 0
    n_pos = T + pos0 - 5
    angle = torch.rand((n_pos, max(rot, 2) // 2), generator=g, device="cuda", dtype=torch.float64) * 7
    table = torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()
    pos = pos0 + torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1)
    if positions == "listed":
        pos = torch.randint(0, n_pos, (B, T), generator=g, device="cuda", dtype=torch.int32)
        pos[torch.rand((B, T), generator=g, device="cuda") < 0.2] = -1
    there = (pos >= 0) & ((pos < n_pos) if rot else True)
    cs = table.double()[pos.long().clamp(0, n_pos - 1)][:, :, None]
    how = dict(interleaved=inter, positions=pos if positions == "listed" else None, pos0=pos0, eps=1e-5)
    x, gain, dy, y, dx, G, sq, checks = {}, {}, {}, {}, {}, {}, {}, []
    for n, H in (("q", Hq), ("k", Hk)):
        if H == 0:
            x[n] = gain[n] = dy[n] = y[n] = dx[n] = G[n] = sq[n] = None
            continue
        # the rows of a joint projection, values behind them
        joint = torch.randn((B, T, (H + 2) * D), generator=g, device="cuda").to(dtype)
        x[n] = joint[..., D:(H + 1) * D].unflatten(-1, (H, D))
        x[n].masked_fill_(~there[..., None, None], float("nan"))
        dy[n] = torch.randn((B, H, T, D), generator=g, device="cuda").to(dtype).transpose(1, 2)
        dy[n].masked_fill_(~there[..., None, None], float("inf"))
        gain[n] = 1 + 0.3 * torch.randn((D,), generator=g, device="cuda")
        for d, shape, dt in ((y, (B, T, H, D), dtype), (dx, (B, T, H, D), dtype), (G, (B, D), F32), (sq, (B,), F32)):
            d[n], c = guarded(shape, dt)
            checks.append(c)
    rotation = table if rot else None
    dp.dpclip_qknorm_forward(x["q"], x["k"], gain["q"], gain["k"], rotation, y["q"], y["k"], **how)
    ws = workspace(dp, dp.dpclip_qknorm_workspace_bytes(B, T, Hq, Hk, D))
    back = lambda: dp.dpclip_qknorm_backward(dy["q"], dy["k"], x["q"], x["k"], gain["q"], gain["k"], rotation, dx["q"], dx["k"], G["q"], G["k"],       # noqa: E731
                                             sq["q"], sq["k"], ws, **how)
    back()
    torch.cuda.synchronize()
    for c in checks:
        c()
    keep = there[..., None, None]
    for n in ("q", "k"):
        if x[n] is None:
            continue
        clean, signal = torch.where(keep, x[n], 0.0), torch.where(keep, dy[n], 0.0)
        want, scale = qk_reference(clean, gain[n], cs[..., 0, :], cs[..., 1, :], rot, inter, 1e-5)
        close(y[n], torch.where(keep, want, 0.5).cpu(), (HALF_STEP[dtype] * want.abs() + 40 * U32 * scale).cpu())
        d, dm, g1, gm = (torch.where(keep, v, 0.0) for v in qk_reference(clean, gain[n], cs[..., 0, :], cs[..., 1, :], rot, inter, 1e-5, signal))
        close(dx[n], d.cpu(), (HALF_STEP[dtype] * d.abs() + 60 * U32 * dm).cpu())
        want, mag = g1.sum((1, 2)), gm.sum((1, 2))
        depth = (40 + T * x[n].shape[2]) * U32
        close(G[n], want.cpu(), (depth * mag).cpu())
        close(sq[n], want.square().sum(1).cpu(), ((2 * depth * mag * want.abs() + (depth * mag) ** 2).sum(1) + (D + 8) * U32 * want.square().sum(1)).cpu())
    first = {n: (dx[n].clone(), G[n].clone()) for n in ("q", "k") if x[n] is not None}
    back()
    for n, (a, b) in first.items():
        assert torch.equal(dx[n], a) and torch.equal(G[n], b)


# ---------------------------------------------------------------------------------------------------------------
# gated block
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,F", [(9473, 512, 1800), (20000, 576, 1170), (40000, 72, 640), (9728, 1000, 2048)])
@pytest.mark.parametrize("act,with_bias,keep,layout", [("silu", False, True, "dense"), ("gelu", True, True, "odd"), ("gelu_tanh", True, False, "dense"),
                                                       ("relu", False, False, "odd")])
def test_gated_forward_of_many_tiles(dp, dtype, M, K, F, act, with_bias, keep, layout):
    """Every row of the outputs, in slabs; outputs by TMA (widths that are multiples of eight) and at odd addresses."""
    g = torch.Generator(device="cuda").manual_seed(M + F)
    X, W = torch.randn((M, K), generator=g, device="cuda").to(dtype), (torch.randn((2 * F, K), generator=g, device="cuda") / math.sqrt(K)).to(dtype)
    bias = 0.5 * torch.randn((2 * F,), generator=g, device="cuda") if with_bias else None
    pad = 1 if layout == "odd" else 0
    H, check_h = guarded((M, F), dtype, strides=(F + pad, 1), tail=64 + pad)
    Z, check_z = guarded((M, 2 * F), dtype, strides=(2 * F + pad, 1), tail=64 + pad)
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    run = lambda: dp.dpclip_gated_forward(X, W, bias, H, Z if keep else None, code(dp, act), ws)           # noqa: E731
    run()
    torch.cuda.synchronize()
    assert dp.dpclip_read_status(ws) == 0
    check_h(); check_z()
    w = W.double()
    for r in range(0, M, 4096):
        x = X[r:r + 4096].double()
        z, mag = x @ w.t(), x.abs() @ w.abs().t()
        if with_bias:
            z, mag = z + bias.double(), mag + bias.double().abs()
        zg, zu = z[:, :F], z[:, F:]
        a, _ = act_and_slope(zg, act)
        d = (2 * (K + 2) if dtype == BF16 else 48 + math.ceil(K / 64) + 8) * U32 * mag
        if keep:
            close(Z[r:r + 4096], z.cpu(), (HALF_STEP[dtype] * z.abs() + d).cpu())
        dg, du = d[:, :F], d[:, F:]
        tol = HALF_STEP[dtype] * (a * zu).abs() * 1.01 + 1.2 * (zu.abs() + du) * dg + a.abs() * du + fast(dtype, zg) * zg.abs() * zu.abs() + 1e-37
        close(H[r:r + 4096], (a * zu).cpu(), tol.cpu())
    if not keep:
        assert bool((Z == 0.5).all())
    first, first_z = H.clone(), Z.clone()
    H.fill_(0.5); Z.fill_(0.5)
    for _ in range(3):
        run()
    assert torch.equal(first, H) and torch.equal(first_z, Z)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(9, 1, 1), (40, 1, 1), (300, 3, 5), (33, 7, 2), (20, 2600, 1), (20000, 1, 9)])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_gated_widths_below_sixteen_bytes(dp, dtype, shape, layout):
    gated_forward_case(dp, dtype, shape, layout, "silu", True, True)
    gated_backward_case(dp, dtype, shape, layout, "silu")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(5, 64, 72), (300, 200, 264), (700, 333, 161), (600, 520, 500)])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_signal_in_place_with_dx(dp, dtype, shape, layout):
    """dZ in place of Z: the bits of the call with a dZ of its own."""
    M, K, F = shape
    g = torch.Generator().manual_seed(M)
    Z, dH, W = torch.randn((M, 2 * F), generator=g).to(dtype), torch.randn((M, F), generator=g).to(dtype), torch.randn((2 * F, K), generator=g).to(dtype)
    z, dh, w, dz = (rows(t, layout, dtype) for t in (Z, dH, W, torch.zeros_like(Z)))
    a, b = torch.empty((M, K), dtype=dtype, device="cuda"), torch.empty((M, K), dtype=dtype, device="cuda")
    ws = workspace(dp, dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]))
    dp.dpclip_gated_backward(dh, z, w, dz, a, dp.DPCLIP_ACT_GELU_TANH, ws)
    dp.dpclip_gated_backward(dh, z, w, z, b, dp.DPCLIP_ACT_GELU_TANH, ws)
    assert torch.equal(z, dz) and torch.equal(a, b) and dp.dpclip_read_status(ws) == 0


# ---------------------------------------------------------------------------------------------------------------
# clipped sums of stored gradients
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,n", [(50, 33), (700, 33), (5000, 40), (600, 5000)])
def test_stored_sums_recorded(dp, B, n):
    """Clusters and launches that start early, recorded: replays with other gradients and factors in the same buffers."""
    g = torch.Generator(device="cuda").manual_seed(B)
    grads, clip = torch.randn((B, n), generator=g, device="cuda"), torch.rand((B,), generator=g, device="cuda")
    out, again, noisy = (torch.empty(n, device="cuda") for _ in range(3))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dp.dpclip_stored_clipped_grad(grads, clip, out)
        dp.dpclip_stored_clipped_grad(out[None], None, again)                 # reads what the launch in front writes
        dp.dpclip_stored_clipped_grad(grads, clip, noisy, sigma=0.5, C=1.0, seed=1, stream_id=2)
    noise = torch.zeros(n, device="cuda")
    dp.dpclip_add_noise(noise, 0.5, 1.0, 1, 2)
    for k in range(3):
        grads.mul_(-0.5)
        clip.copy_(torch.rand((B,), generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        terms = clip.double()[:, None] * grads.double()
        close(out, terms.sum(0).cpu(), ((B / 8 + 40) * U32 * terms.abs().sum(0)).cpu())
        assert torch.equal(again, out)
        close(noisy, (out.double() + noise.double()).cpu(), 3 * U32 * (out.abs() + noise.abs()).double().cpu())


# ---------------------------------------------------------------------------------------------------------------
# switches
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(300, 200, 264), (700, 333, 161), (600, 520, 500)])
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_gated_on_the_fp32_alus(dp, path_switch, dtype, shape, layout):
    path_switch("DPCLIP_FORCE_SIMT", "1")
    gated_forward_case(dp, dtype, shape, layout, "silu", True, True)
    gated_backward_case(dp, dtype, shape, layout, "gelu")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_without_overlap_the_same_bits(dp, path_switch, dtype):
    """Launches that start before the one in front of them has ended, and the same without: nothing is read too early."""
    M, K, F, B, T, H, D, nb = 600, 520, 200, 12, 50, 3, 64, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s, std=1.0: (std * torch.randn(s, generator=g, device="cuda")).to(dtype)                # noqa: E731
    X, W, dH, dS, q, dq = new(M, K), new(2 * F, K, std=0.05), new(M, F), new(B, H, T, T), new(B, T, H, D), new(B, T, H, D)
    clip = torch.rand((B,), generator=g, device="cuda")
    ws = workspace(dp, max(dp.dpclip_gated_workspace_bytes(M, K, F, CODE[dtype]), dp.dpclip_relbias_workspace_bytes(B, H, T, T, nb, CODE[dtype]),
                           dp.dpclip_qknorm_workspace_bytes(B, T, H, 0, D)))

    def run():
        o = [torch.empty(s, dtype=dtype, device="cuda") for s in ((M, F), (M, 2 * F), (M, 2 * F), (M, K), (B, T, H, D))]
        f = [torch.empty(s, device="cuda") for s in ((B, nb, H), (B,), (nb, H), (B, D), (B,), (D,))]
        for _ in range(3):
            dp.dpclip_gated_forward(X, W, None, o[0], o[1], dp.DPCLIP_ACT_SILU, ws)
            dp.dpclip_gated_backward(dH, o[1], W, o[2], o[3], dp.DPCLIP_ACT_SILU, ws)
            dp.dpclip_relbias_sqnorms(dS, f[0], f[1], ws, 40)
            dp.dpclip_stored_clipped_grad(f[0], clip, f[2])
            dp.dpclip_qknorm_backward(dq, None, q, None, None, None, None, o[4], None, f[3], None, f[4], None, ws)
            dp.dpclip_stored_clipped_grad(f[3], clip, f[5], sigma=0.5, C=2.0, seed=3, stream_id=4)
        torch.cuda.synchronize()
        assert dp.dpclip_read_status(ws) == 0
        return o + f

    want = run()
    path_switch("DPCLIP_NO_OVERLAP", "1")
    for a, b in zip(run(), want):
        assert torch.equal(a, b)


