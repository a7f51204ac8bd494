"""Relative position bias, norms of queries and keys with the rotation, clipped sums of stored per-example gradients: the kernels against
their formulas in 64 bits on the CPU.

Tolerances.  An output rounded once to a type with a step of eps is off by eps / 2 of its value (bf16 2^-8, fp32 2^-24).  What is
computed in fp32 before that is off by a few 2^-24 per operation of the longest chain, relative to the sum of the magnitudes added up; tests
compare with that sum of magnitudes, computed beside the reference, so they need no luck with cancellation.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24
CODE = {F32: 0, BF16: 1}
HALF_STEP = {BF16: 2.0 ** -8, F32: U32}


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


def workspace(dp, nbytes):
    ws = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
    dp.dpclip_workspace_init(ws)
    return ws


def guarded(shape, dtype, fill=0.5, strides=None, tail=64):
    """A tensor in the middle of a larger buffer of a known pattern; check() says whether anything around it was written."""
    strides = strides or torch.empty(shape, device="meta").stride()
    n = 1 + sum((s - 1) * k for s, k in zip(shape, strides))
    raw = torch.full((tail + n + tail,), 77.0, device="cuda", dtype=dtype)
    t = raw.as_strided(shape, strides, tail)
    mask = torch.ones_like(raw, dtype=torch.bool)
    mask.as_strided(shape, strides, tail).fill_(False)
    t.fill_(fill)

    def check():
        assert bool((raw[mask] == 77.0).all()), "written outside the output"
    return t, check


def close(got, want, tol):
    """|got - want| <= tol element by element; equal where want is not finite."""
    got = got.detach().double().cpu()
    want = torch.as_tensor(want, dtype=torch.float64)
    tol = torch.as_tensor(tol, dtype=torch.float64).expand_as(want)
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(nan=1e300), want[~fine].nan_to_num(nan=1e300))
    off = (got - want).abs()[fine] - tol[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"off by {float(off.max()):.3g} more than allowed"


# ---------------------------------------------------------------------------------------------------------------
# relative position bias
# ---------------------------------------------------------------------------------------------------------------
def bucket_table(Tq, Tk, off, n_buckets, max_distance, bidirectional):
    """bucket of (q, k), by whole numbers"""
    n = n_buckets // 2 if bidirectional else n_buckets
    e = n // 2
    m = n - e
    known = {}
    out = np.empty((Tq, Tk), dtype=np.int64)
    for q in range(Tq):
        for k in range(Tk):
            rel = k - (off + q)
            rel = max(-max_distance, min(max_distance, rel))
            if rel not in known:
                base, d = ((n if rel > 0 else 0), abs(rel)) if bidirectional else (0, max(-rel, 0))
                if d < e:
                    known[rel] = base + d
                else:
                    j = 0
                    while j < m - 1 and d ** m * e ** (j + 1) >= max_distance ** (j + 1) * e ** m:
                        j += 1
                    known[rel] = base + e + j
            out[q, k] = known[rel]
    return torch.from_numpy(out)


RELBIAS = [
    # H, Tq, Tk, off, n_buckets, max_distance, bidirectional, causal
    (1, 1, 1, 0, 2, 2, False, False),
    (3, 1, 77, 76, 32, 128, False, True),
    (2, 1, 8, 0, 32, 20, True, True),
    (5, 64, 64, 0, 32, 40, True, False),
    (4, 77, 77, 0, 32, 50, False, True),
    (2, 33, 200, 167, 16, 64, True, True),
    (3, 200, 33, 0, 12, 100, True, False),
    (1, 9, 265, 5, 256, 300, False, False),
    (2, 8, 24, 1 << 33, 32, 128, True, False),        # positions beyond 32 bits
    (2, 130, 1032, 0, 64, 1 << 20, True, False),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", RELBIAS)
@pytest.mark.parametrize("layout", ["dense", "padded", "heads_inside", "odd_start"])
def test_relbias_forward(dp, case, dtype, layout):
    H, Tq, Tk, off, nb, D, both, causal = case
    g = torch.Generator().manual_seed(7)
    table = torch.randn((nb, H + 2), generator=g)
    bucket = bucket_table(Tq, Tk, off, nb, D, both)
    want = table.double()[bucket][..., :H].permute(2, 0, 1).clone()
    if causal:
        q, k = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
        want.masked_fill_((k > q + off)[None], -math.inf)
    ld = Tk if layout in ("dense", "odd_start") else (Tk + 15) // 8 * 8
    strides = (Tq * ld, ld, 1) if layout != "heads_inside" else (ld, H * ld, 1)
    out, check = guarded((H, Tq, Tk), dtype, strides=strides, tail=64 if layout != "odd_start" else 65)
    dev = table.cuda()[:, :H]                                    # rows of H + 2
    dp.dpclip_relbias_forward(dev, out, D, both, causal, off)
    torch.cuda.synchronize()
    check()
    close(out, want, HALF_STEP[dtype] * want.abs().nan_to_num(posinf=0, neginf=0) if dtype == BF16 else torch.zeros_like(want))


GRAD = [
    # B, H, Tq, Tk, off, n_buckets, max_distance, bidirectional, causal, padded
    (1, 1, 1, 1, 0, 2, 2, False, False, False),
    (3, 2, 1, 77, 76, 32, 128, False, True, False),
    (4, 3, 64, 64, 0, 32, 40, True, False, False),
    (5, 2, 77, 77, 0, 32, 50, False, True, True),
    (3, 2, 40, 200, 160, 16, 64, True, True, True),
    (2, 3, 200, 33, 0, 12, 100, True, False, True),
    (4, 1, 9, 264, 5, 256, 300, False, False, True),
    (2, 1, 8, 24, 1 << 33, 32, 128, True, False, False),
    (1, 2, 300, 2100, 0, 32, 1 << 20, True, False, False),     # several tiles along the keys
    (1, 1, 1200, 16, 0, 64, 500, True, False, True),           # many more queries than keys: walks that wrap often
    (70, 16, 16, 16, 0, 8, 20, True, True, True),
]


def relbias_reference(dS, bucket, nb, causal, off, ql, kl):
    """G (B, nb, H) and the same of the magnitudes, in 64 bits."""
    B, H, Tq, Tk = dS.shape
    q, k = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
    counts = torch.ones(B, Tq, Tk, dtype=torch.bool)
    if causal:
        counts &= (k <= q + off)[None]
    if ql is not None:
        counts &= (q[None] < ql[:, None, None])
    if kl is not None:
        counts &= (k[None] < kl[:, None, None])
    x = torch.where(counts[:, None], dS.double(), 0.0).reshape(B * H, -1)
    flat = bucket.reshape(-1)
    G = torch.zeros(B * H, nb, dtype=torch.float64).index_add_(1, flat, x)
    A = torch.zeros(B * H, nb, dtype=torch.float64).index_add_(1, flat, x.abs())
    return G.view(B, H, nb).transpose(1, 2), A.view(B, H, nb).transpose(1, 2)


def grad_inputs(case, dtype, seed=3):
    B, H, Tq, Tk, off, nb, D, both, causal, padded = case
    g = torch.Generator().manual_seed(seed)
    dS = torch.randn((B, H, Tq, Tk), generator=g).to(dtype)
    ql = kl = None
    if padded:
        ql = torch.randint(-2, Tq + 3, (B,), generator=g, dtype=torch.int32)        # lengths outside the tensor too
        kl = torch.randint(-2, Tk + 3, (B,), generator=g, dtype=torch.int32)
        ql[0], kl[0] = Tq, Tk
        if B > 1:
            kl[1] = 0                                                                # an example with nothing in it
        q, k = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
        out = (q[None] >= ql[:, None, None]) | (k[None] >= kl[:, None, None])
        dS.masked_fill_(out[:, None].expand_as(dS), float("nan"))
        dS[:, :, :, ::3] = torch.where(out[:, None, :, ::3], torch.tensor(float("inf"), dtype=dtype), dS[:, :, :, ::3])
    if causal:
        q, k = torch.arange(Tq)[:, None], torch.arange(Tk)[None]
        dS.masked_fill_((k > q + off)[None, None].expand_as(dS), torch.finfo(dtype).min)
    return dS, ql, kl


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", GRAD)
@pytest.mark.parametrize("layout", ["dense", "row_padded", "heads_inside"])
def test_relbias_gradient(dp, case, dtype, layout):
    B, H, Tq, Tk, off, nb, D, both, causal, padded = case
    dS, ql, kl = grad_inputs(case, dtype)
    bucket = bucket_table(Tq, Tk, off, nb, D, both)
    want, mag = relbias_reference(dS, bucket, nb, causal, off, ql, kl)
    ld = Tk if layout == "dense" else (Tk + 15) // 8 * 8
    shape = (B, Tq, H, ld) if layout == "heads_inside" else (B, H, Tq, ld)
    store = torch.full(shape, float("nan"), dtype=dtype, device="cuda")
    dev = store.transpose(1, 2)[..., :Tk] if layout == "heads_inside" else store[..., :Tk]
    dev.copy_(dS)
    grads, check_g = guarded((B, nb, H), F32)
    sq, check_s = guarded((B,), F32)
    ws = workspace(dp, dp.dpclip_relbias_workspace_bytes(B, H, Tq, Tk, nb, CODE[dtype]))
    lens = dict(q_lens=None if ql is None else ql.cuda(), k_lens=None if kl is None else kl.cuda())
    how = dict(max_distance=D, bidirectional=both, causal=causal, q_offset=off, **lens)
    dp.dpclip_relbias_sqnorms(dev, grads, sq, ws, **how)
    torch.cuda.synchronize()
    check_g(); check_s()
    # chains: at most 8 * 32 additions in a walk's register, the folds behind it fewer than 400
    depth = 700 * U32
    close(grads, want, depth * mag)
    close(sq, want.square().sum((1, 2)), (2 * depth * mag * want.abs() + (depth * mag) ** 2).sum((1, 2)) + (nb * H + 8) * U32 * want.square().sum((1, 2)))
    first = grads.clone()
    dp.dpclip_relbias_sqnorms(dev, grads, sq, ws, **how)
    assert torch.equal(first, grads)                              # the same bits again
    dp.dpclip_relbias_sqnorms(dev, grads, sq, ws, accumulate=True, **how)
    close(grads, 2 * want, 2 * depth * mag)
    close(sq, 4 * want.square().sum((1, 2)), 4 * ((2 * depth * mag * want.abs() + (depth * mag) ** 2).sum((1, 2)) + (nb * H + 8) * U32 * want.square().sum((1, 2))))


def test_relbias_gradient_against_differences(dp):
    """d/d table of sum(dS * bias(table)) is the sum of the per-example gradients: by central differences of the forward pass (which is
    linear, so the differences have no error of their own)."""
    H, T, nb, D = 2, 24, 16, 30
    table = torch.randn((nb, H), generator=torch.Generator().manual_seed(1)).cuda()
    dS = torch.randn((3, H, T, T), generator=torch.Generator().manual_seed(2)).cuda()
    grads, sq = torch.empty((3, nb, H), device="cuda"), torch.empty(3, device="cuda")
    ws = workspace(dp, dp.dpclip_relbias_workspace_bytes(3, H, T, T, nb, 0))
    dp.dpclip_relbias_sqnorms(dS, grads, sq, ws, D)
    total = torch.empty((nb, H), device="cuda")
    dp.dpclip_stored_clipped_grad(grads, None, total)

    def loss(t):
        bias = torch.empty((H, T, T), device="cuda")
        dp.dpclip_relbias_forward(t, bias, D)
        return float((dS.double() * bias.double()).sum())

    for j, h in ((0, 0), (3, 1), (7, 0), (9, 1), (15, 0), (8, 1)):
        up, down = table.clone(), table.clone()
        up[j, h] += 0.5; down[j, h] -= 0.5
        step = float(up[j, h].double() - down[j, h].double())
        # each bias is exact, the table's change is rounded to fp32: 2^-23 of |dS| in all
        mag = float(dS.abs().sum())
        assert abs((loss(up) - loss(down)) / step - float(total[j, h])) <= 700 * U32 * mag


# ---------------------------------------------------------------------------------------------------------------
# norms of queries and keys
# ---------------------------------------------------------------------------------------------------------------
QK = [
    # B, T, Hq, Hk, D, rot, interleaved
    (1, 1, 1, 1, 2, 2, False),
    (3, 1, 8, 2, 64, 64, False),
    (2, 37, 8, 2, 64, 64, True),
    (2, 20, 6, 6, 50, 32, True),
    (2, 19, 3, 1, 128, 128, False),
    (2, 33, 5, 2, 128, 64, False),
    (3, 21, 2, 2, 96, 96, False),
    (2, 9, 4, 1, 256, 256, True),
    (2, 5, 2, 1, 512, 512, False),
    (1, 7, 3, 2, 33, 6, False),               # an odd width: the last element has no partner
    (2, 11, 2, 2, 80, 16, False),
    (1, 5, 1, 1, 1, 0, False),
    (2, 6, 3, 0, 64, 0, False),               # queries alone, no rotation
    (4, 260, 16, 2, 128, 128, True),
    (1300, 1, 2, 1, 32, 32, False),           # many examples of one token
    (1250, 3, 1, 2, 50, 20, True),
    (2, 700, 20, 3, 80, 80, False),           # rings of copies, head blocks that are not full, idle lanes
    (3, 300, 7, 5, 160, 96, True),
    (40, 64, 9, 0, 32, 32, False),
]


def qk_reference(x, gain, cos, sin, rot, interleaved, eps, dy=None):
    """Forward value, or (dx, G per row) of one tensor, in 64 bits, with the scale of what is added up."""
    x = x.double()
    D = x.shape[-1]
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    gain = torch.ones(D, dtype=torch.float64) if gain is None else gain.double()
    if dy is None:
        y = x * r * gain
        out, mag = y.clone(), y.abs()
        out[..., a] = cos * y[..., a] - sin * y[..., b]
        out[..., b] = sin * y[..., a] + cos * y[..., b]
        scale = mag.clone()
        scale[..., a] = (cos * y[..., a]).abs() + (sin * y[..., b]).abs()
        scale[..., b] = (sin * y[..., a]).abs() + (cos * y[..., b]).abs()
        return out, scale
    dy = dy.double()
    g, gm = dy.clone(), dy.abs()
    g[..., a] = cos * dy[..., a] + sin * dy[..., b]
    g[..., b] = cos * dy[..., b] - sin * dy[..., a]
    gm[..., a] = (cos * dy[..., a]).abs() + (sin * dy[..., b]).abs()
    gm[..., b] = (cos * dy[..., b]).abs() + (sin * dy[..., a]).abs()
    xh = x * r
    w = g * gain
    dx = r * (w - xh * (w * xh).mean(-1, keepdim=True))
    dm = r * (gm * gain.abs() + xh.abs() * (gm * gain.abs() * xh.abs()).mean(-1, keepdim=True))
    return dx, dm, g * xh, gm * xh.abs()


def qk_inputs(case, dtype, layout, padded, seed=5):
    B, T, Hq, Hk, D, rot, inter = case
    g = torch.Generator().manual_seed(seed)
    n_pos = T + 40
    angle = torch.rand((n_pos, rot // 2), generator=g, dtype=torch.float64) * 7
    table = torch.stack([angle.cos(), angle.sin()], 1).float()
    pos = torch.randint(0, n_pos, (B, T), generator=g, dtype=torch.int32)
    if padded:
        pos[torch.rand((B, T), generator=g) < 0.3] = -1
        pos[0, 0] = n_pos                                          # behind the table: padding as well
        if B > 1:
            pos[B - 1] = -1                                        # an example with nothing in it
    out = {"table": table, "pos": pos, "n_pos": n_pos}
    for n, H in (("q", Hq), ("k", Hk)):
        if H == 0:
            out[n] = out["d" + n] = out["gain_" + n] = None
            continue
        out[n] = torch.randn((B, T, H, D), generator=g).to(dtype)
        out["d" + n] = torch.randn((B, T, H, D), generator=g).to(dtype)
        out["gain_" + n] = 1 + 0.3 * torch.randn((D,), generator=g)
        if padded:
            there = (pos >= 0) & (pos < n_pos)
            for m in (n, "d" + n):
                out[m].masked_fill_(~there[..., None, None], float("nan"))
    return out


def place(t, layout, dtype, extra):
    """A device tensor (B, T, H, D) in one of the layouts a program has."""
    B, T, H, D = t.shape
    if layout == "joint":                                          # columns of a joint projection
        row = torch.full((B, T, (H + extra) * D + (8 if D % 8 == 0 else 3)), 9.0, dtype=dtype, device="cuda")
        dev = row[..., extra * D:(H + extra) * D].unflatten(-1, (H, D))
    elif layout == "head_major":
        dev = torch.full((B, H, T, D), 9.0, dtype=dtype, device="cuda").transpose(1, 2)
    else:
        dev = torch.full((B, T, H, D), 9.0, dtype=dtype, device="cuda")
    dev.copy_(t)
    return dev


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", QK)
@pytest.mark.parametrize("layout,padded", [("dense", False), ("joint", True), ("head_major", False)])
def test_qknorm_forward(dp, case, dtype, layout, padded):
    B, T, Hq, Hk, D, rot, inter = case
    s = qk_inputs(case, dtype, layout, padded)
    there = (s["pos"] >= 0) & (s["pos"] < s["n_pos"])
    cs = s["table"].double()[s["pos"].long().clamp(0, s["n_pos"] - 1)][:, :, None]
    eps = 1e-5
    dev = {n: None if s[n] is None else place(s[n], layout, dtype, 1) for n in ("q", "k")}
    outs, checks = {}, []
    for n, H in (("q", Hq), ("k", Hk)):
        outs[n] = None
        if H:
            outs[n], c = guarded((B, T, H, D), dtype)
            checks.append(c)
    rotation = s["table"].cuda() if rot else None
    gains = [None if s["gain_" + n] is None else s["gain_" + n].cuda() for n in ("q", "k")]
    # without a table every position is in range, so the padded tokens keep a negative one
    pos = s["pos"].clone()
    if rot == 0:
        pos[~there] = -1
    args = (dev["q"], dev["k"], *gains, rotation, outs["q"], outs["k"])
    dp.dpclip_qknorm_forward(*args, interleaved=inter, positions=pos.cuda(), eps=eps)
    torch.cuda.synchronize()
    for c in checks:
        c()
    for n in ("q", "k"):
        if outs[n] is None:
            continue
        want, scale = qk_reference(s[n].nan_to_num(), s["gain_" + n], cs[..., 0, :], cs[..., 1, :], rot, inter, eps)
        want = torch.where(there[..., None, None], want, 0.5)                  # a padding row stays as it was
        # the mean: D additions in a tree of at most 5 + 16 levels; the root's reciprocal 2 units; three products and the turn
        close(outs[n], want, HALF_STEP[dtype] * want.abs() + 40 * U32 * scale)
    if layout == "dense":                                                      # in place
        dp.dpclip_qknorm_forward(dev["q"], dev["k"], *gains, rotation, dev["q"], dev["k"], interleaved=inter, positions=pos.cuda(), eps=eps)
        for n in ("q", "k"):
            if outs[n] is not None:
                assert torch.equal(dev[n], outs[n])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", QK)
@pytest.mark.parametrize("layout,padded", [("dense", False), ("joint", True), ("head_major", False)])
def test_qknorm_backward(dp, case, dtype, layout, padded):
    B, T, Hq, Hk, D, rot, inter = case
    s = qk_inputs(case, dtype, layout, padded)
    there = (s["pos"] >= 0) & (s["pos"] < s["n_pos"])
    cs = s["table"].double()[s["pos"].long().clamp(0, s["n_pos"] - 1)][:, :, None]
    eps = 1e-5
    pos = s["pos"].clone()
    if rot == 0:
        pos[~there] = -1
    dev = {n: None if s[n] is None else place(s[n], layout, dtype, 1) for n in ("q", "k", "dq", "dk")}
    gains = [None if s["gain_" + n] is None else s["gain_" + n].cuda() for n in ("q", "k")]
    rotation = s["table"].cuda() if rot else None
    out, checks = {}, []
    for n, H in (("q", Hq), ("k", Hk)):
        for m, shape, dt in ((n, (B, T, H, D), dtype), ("grads_" + n, (B, D), F32), ("sq_" + n, (B,), F32)):
            out[m] = None
            if H:
                out[m], c = guarded(shape, dt)
                checks.append(c)
    ws = workspace(dp, dp.dpclip_qknorm_workspace_bytes(B, T, Hq, Hk, D))
    how = dict(interleaved=inter, positions=pos.cuda(), eps=eps)
    call = lambda dq, dk: dp.dpclip_qknorm_backward(dev["dq"], dev["dk"], dev["q"], dev["k"], *gains, rotation, dq, dk,      # noqa: E731
                                                    out["grads_q"], out["grads_k"], out["sq_q"], out["sq_k"], ws, **how)
    call(out["q"], out["k"])
    torch.cuda.synchronize()
    for c in checks:
        c()
    for n in ("q", "k"):
        if out[n] is None:
            continue
        dx, dm, G, Gm = qk_reference(s[n].nan_to_num(), s["gain_" + n], cs[..., 0, :], cs[..., 1, :], rot, inter, eps, s["d" + n].nan_to_num())
        keep = there[..., None, None]
        dx, dm, G, Gm = (torch.where(keep, v, 0.0) for v in (dx, dm, G, Gm))
        close(out[n], dx, HALF_STEP[dtype] * dx.abs() + 60 * U32 * dm)
        want, mag = G.sum((1, 2)), Gm.sum((1, 2))
        # a term has 30 roundings at most; a thread adds up at most T * H of them, then the groups, warps and chunks
        depth = (40 + T * s[n].shape[2]) * U32
        close(out["grads_" + n], want, depth * mag)
        close(out["sq_" + n], want.square().sum(1), (2 * depth * mag * want.abs() + (depth * mag) ** 2).sum(1) + (D + 8) * U32 * want.square().sum(1))
    first = {n: v.clone() for n, v in out.items() if v is not None}
    call(dev["dq"], dev["dk"])                                     # in place of the signals, and the same bits again
    for n in ("q", "k"):
        if out[n] is not None:
            assert torch.equal(dev["d" + n], first[n]) and torch.equal(out["grads_" + n], first["grads_" + n])


def test_qknorm_backward_against_differences(dp):
    """Directional differences of the forward pass in fp32, for the inputs and for the gains."""
    B, T, H, D = 2, 5, 3, 16
    g = torch.Generator().manual_seed(11)
    x = torch.randn((B, T, H, D), generator=g).cuda()
    dy = torch.randn((B, T, H, D), generator=g).cuda()
    gain = (1 + 0.2 * torch.randn((D,), generator=g)).cuda()
    rotation = torch.empty((T, 2, D // 2), device="cuda")
    dp.dpclip_rotation_table(rotation)

    def loss(x, gain):
        y = torch.empty_like(x)
        dp.dpclip_qknorm_forward(x, None, gain, None, rotation, y, None)
        return (y.double() * dy.double()).sum((1, 2, 3)).cpu()

    dx, G, sq = torch.empty_like(x), torch.empty((B, D), device="cuda"), torch.empty(B, device="cuda")
    ws = workspace(dp, dp.dpclip_qknorm_workspace_bytes(B, T, H, 0, D))
    dp.dpclip_qknorm_backward(dy, None, x, None, gain, None, rotation, dx, None, G, None, sq, None, ws)
    h = 2.0 ** -7
    mag = float(dy.abs().sum()) * 3                                # |y| <= sqrt(D) |gain|: values of at most 3 on average
    for seed in range(3):
        v = torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)).cuda()
        diff = (loss(x + h * v, gain) - loss(x - h * v, gain)).sum() / (2 * h)
        # rounding 10 units of the values over 2 h; the third derivative's term is h^2 of the values
        assert abs(float(diff) - float((dx.double() * v.double()).sum())) <= mag * (10 * U32 / h + 4 * h * h)
        w = torch.randn(gain.shape, generator=torch.Generator().manual_seed(seed + 9)).cuda()
        diff = (loss(x, gain + h * w) - loss(x, gain - h * w)) / (2 * h)
        want = (G.double() * w.double()).sum(1).cpu()
        assert float((diff - want).abs().max()) <= mag * 10 * U32 / h


def test_default_positions_and_far_angles(dp):
    """positions None is pos0 + t; the table's angles are right far out, where fp32 angles would be off by whole turns."""
    n_pos, rot = 4096, 64
    table = torch.empty((n_pos, 2, rot // 2), device="cuda")
    dp.dpclip_rotation_table(table, 10000.0, 0.001)                # scale below one: angles to 4e6
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] / 0.001 * 10000.0 ** (-2 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    # cosine and sine move by at most what the angle does: 64-bit angles are good to 2^-52 of 4e6, the power to a few units
    close(table[:, 0], angle.cos(), U32 + 2.0 ** -48 * 4.1e6)
    close(table[:, 1], angle.sin(), U32 + 2.0 ** -48 * 4.1e6)
    x = torch.randn((2, 6, 3, 64), generator=torch.Generator().manual_seed(0)).cuda()
    a, b = torch.empty_like(x), torch.empty_like(x)
    pos = (torch.arange(6, dtype=torch.int32) + 4000).repeat(2, 1).cuda()
    dp.dpclip_qknorm_forward(x, None, None, None, table, a, None, pos0=4000)
    dp.dpclip_qknorm_forward(x, None, None, None, table, b, None, positions=pos)
    assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------------------------
# clipped sums of stored gradients
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,n", [(1, 1), (7, 33), (128, 512), (257, 100), (5000, 31), (700, 33), (1025, 64), (600, 5000)])
@pytest.mark.parametrize("with_clip", [True, False])
def test_stored_clipped_grad(dp, B, n, with_clip):
    g = torch.Generator().manual_seed(B * n)
    grads, clip = torch.randn((B, n), generator=g), torch.rand((B,), generator=g)
    want = ((clip.double() if with_clip else torch.ones(B, dtype=torch.float64))[:, None] * grads.double())
    out, check = guarded((n,), F32)
    args = (grads.cuda(), clip.cuda() if with_clip else None)
    dp.dpclip_stored_clipped_grad(*args, out)
    torch.cuda.synchronize()
    check()
    tol = (B / 8 + 40) * U32 * want.abs().sum(0)
    close(out, want.sum(0), tol)
    # noise as dpclip_add_noise draws it, added last
    noisy, noise = torch.empty_like(out), torch.zeros(n, device="cuda")
    dp.dpclip_stored_clipped_grad(*args, noisy, sigma=0.7, C=2.0, seed=5, stream_id=9)
    dp.dpclip_add_noise(noise, 0.7, 2.0, 5, 9)
    close(noisy, out.double().cpu() + noise.double().cpu(), 3 * U32 * (out.abs() + noise.abs()).double().cpu())


# ---------------------------------------------------------------------------------------------------------------
# as they are used
# ---------------------------------------------------------------------------------------------------------------
def test_attention_parameters_in_one_step(dp):
    """One step of a model whose parameters are a projection, the gains of queries and keys and the position table: norms over all of
    them, one set of factors, every sum clipped with it; against per-example gradients built one by one in 64 bits.  The same as a recorded
    graph on another stream."""
    B, T, H, D, nb, far = 6, 24, 2, 32, 16, 20
    d = H * D
    g = torch.Generator().manual_seed(21)
    randn = lambda *s, std=1.0: (torch.randn(s, generator=g) * std)                                    # noqa: E731
    A, Z = randn(B, T, d).cuda(), randn(B, T, d, std=0.01).cuda()
    q, k, dq, dk = randn(B, T, H, D).cuda(), randn(B, T, H, D).cuda(), randn(B, T, H, D, std=0.03).cuda(), randn(B, T, H, D, std=0.03).cuda()
    dS = randn(B, H, T, T, std=0.03).cuda()
    gq, gk = (1 + 0.1 * randn(D)).cuda(), (1 + 0.1 * randn(D)).cuda()
    lens = torch.tensor([T, 1, 7, T, 0, 20], dtype=torch.int32)
    pos = torch.where(torch.arange(T)[None] < lens[:, None], torch.arange(T)[None], -1).to(torch.int32).cuda()
    lens = lens.cuda()
    rotation = torch.empty((T, 2, D // 2), device="cuda")
    dp.dpclip_rotation_table(rotation)
    sq = torch.empty((4, B), device="cuda")
    clip, norms = torch.empty(B, device="cuda"), torch.empty(B, device="cuda")
    gW, gb = torch.empty((d, d), device="cuda"), torch.empty(d, device="cuda")
    Gq, Gk, Gt = torch.empty((B, D), device="cuda"), torch.empty((B, D), device="cuda"), torch.empty((B, nb, H), device="cuda")
    sq_gain = [torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]
    s_t = torch.empty((nb, H), device="cuda")
    dxq, dxk = torch.empty_like(q), torch.empty_like(k)
    ws = workspace(dp, max(dp.dpclip_workspace_bytes(B, T, d, d), dp.dpclip_relbias_workspace_bytes(B, H, T, T, nb, 0),
                           dp.dpclip_qknorm_workspace_bytes(B, T, H, H, D)))

    def step(C=1.0):
        dp.dpclip_layer_sqnorms(A, Z, True, sq[0], ws)
        dp.dpclip_qknorm_backward(dq, dk, q, k, gq, gk, rotation, dxq, dxk, Gq, Gk, sq[1], sq[2], ws, positions=pos)
        dp.dpclip_relbias_sqnorms(dS, Gt, sq[3], ws, far, q_lens=lens, k_lens=lens)
        dp.dpclip_factors(sq, C, clip, norms)
        dp.dpclip_clipped_grad(A, Z, clip, gW, gb, ws)
        dp.dpclip_stored_clipped_grad(Gq, clip, sq_gain[0])
        dp.dpclip_stored_clipped_grad(Gk, clip, sq_gain[1])
        dp.dpclip_stored_clipped_grad(Gt, clip, s_t)

    there = (pos.cpu() >= 0)[..., None, None]
    cs = rotation.double().cpu()[pos.cpu().long().clamp(min=0)][:, :, None]
    wq, wk = ((torch.where(there, qk_reference(x.cpu(), gn.cpu(), cs[..., 0, :], cs[..., 1, :], D, False, 1e-6, dy.cpu())[2], 0.0)).sum((1, 2))
              for x, gn, dy in ((q, gq, dq), (k, gk, dk)))
    wt, _ = relbias_reference(dS.cpu(), bucket_table(T, T, 0, nb, far, True), nb, False, 0, lens.cpu(), lens.cpu())
    wW = torch.einsum("bto,bti->boi", Z.double().cpu(), A.double().cpu())
    wb = Z.double().cpu().sum(1)
    n = torch.sqrt(wW.square().sum((1, 2)) + wb.square().sum(1) + wq.square().sum(1) + wk.square().sum(1) + wt.square().sum((1, 2)))
    clipped = []
    for C in (float(n.median()) * 1.0001, 1.0):                    # about half of the examples clipped, then all
        step(C)
        torch.cuda.synchronize()
        c = torch.clamp(C / n, max=1.0)
        clipped.append(int((c < 1).sum()))
        close(norms, n, 1e-5 * n)
        for got, want in ((gW, torch.einsum("b,boi->oi", c, wW)), (gb, (c[:, None] * wb).sum(0)), (sq_gain[0], (c[:, None] * wq).sum(0)),
                          (sq_gain[1], (c[:, None] * wk).sum(0)), (s_t, (c[:, None, None] * wt).sum(0))):
            assert float((got.double().cpu() - want).norm() / want.norm()) <= 1e-5
    assert clipped == [B // 2, B]
    # recorded, with other inputs in the same buffers at replay
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    want = [t.clone() for t in (Gq, Gk, Gt, sq_gain[0], sq_gain[1], s_t, dxq, dxk)]
    for t in (Gq, Gk, Gt, *sq_gain, s_t, dxq, dxk):
        t.fill_(9.0)
    graph.replay()
    torch.cuda.synchronize()
    for t, w in zip((Gq, Gk, Gt, *sq_gain, s_t, dxq, dxk), want):
        assert torch.equal(t, w)
    dS.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Gt, want[2] * 0.5)


def test_offsets_beyond_32_bits(dp):
    """Examples that lie more than 2^31 elements apart in one buffer (a cache, a pool): read and written where they are."""
    far = (1 << 31) + 24
    pool = torch.empty(far + 4096, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(2)
    dS = torch.randn((2, 2, 16, 24), generator=g).bfloat16()
    dev = pool.as_strided((2, 2, 16, 24), (far, 384, 24, 1))
    dev.copy_(dS)
    nb = 16
    grads, sq = torch.empty((2, nb, 2), device="cuda"), torch.empty(2, device="cuda")
    ws = workspace(dp, dp.dpclip_relbias_workspace_bytes(2, 2, 16, 24, nb, 1))
    dp.dpclip_relbias_sqnorms(dev, grads, sq, ws, 30)
    want, mag = relbias_reference(dS, bucket_table(16, 24, 0, nb, 30, True), nb, False, 0, None, None)
    close(grads, want, 700 * U32 * mag)
    x = torch.randn((2, 3, 2, 64), generator=g).bfloat16()
    xd = pool.as_strided((2, 3, 2, 64), (far, 128, 64, 1), 1024)
    xd.copy_(x)
    y = torch.empty((2, 3, 2, 64), dtype=BF16, device="cuda")
    dp.dpclip_qknorm_forward(xd, None, None, None, None, y, None, eps=1e-5)
    v = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-5)
    close(y, v, HALF_STEP[BF16] * v.abs() + 40 * U32 * v.abs())
    dp.dpclip_qknorm_forward(xd, None, None, None, None, xd, None, eps=1e-5)
    assert torch.equal(xd, y)


def test_two_streams_at_once(dp):
    """Calls on two streams, each with outputs and a workspace of its own, interleaved: the bits of the calls one after the other."""
    B, T, H, D, nb = 16, 256, 8, 64, 32
    table = torch.empty((T, 2, D // 2), device="cuda")
    dp.dpclip_rotation_table(table)
    sides = []
    for k in range(2):
        g = torch.Generator(device="cuda").manual_seed(k)
        s = {n: torch.randn((B, T, H, D), generator=g, device="cuda").bfloat16() for n in ("q", "k", "dq", "dk")}
        s["dS"] = torch.randn((B, H, T, T), generator=g, device="cuda").bfloat16()
        s["ws"] = workspace(dp, max(dp.dpclip_relbias_workspace_bytes(B, H, T, T, nb, 1), dp.dpclip_qknorm_workspace_bytes(B, T, H, H, D)))
        s["out"] = [torch.empty_like(s["q"]), torch.empty_like(s["q"]), torch.empty((B, D), device="cuda"), torch.empty((B, D), device="cuda"),
                    torch.empty((B, nb, H), device="cuda"), torch.empty(B, device="cuda"), torch.empty((nb, H), device="cuda")]
        s["stream"] = torch.cuda.Stream()
        sides.append(s)

    def run(s, stream):
        o = s["out"]
        dp.dpclip_qknorm_backward(s["dq"], s["dk"], s["q"], s["k"], None, None, table, o[0], o[1], o[2], o[3], None, None, s["ws"], stream=stream)
        dp.dpclip_relbias_sqnorms(s["dS"], o[4], o[5], s["ws"], 128, stream=stream)
        dp.dpclip_stored_clipped_grad(o[4], None, o[6], stream=stream)

    want = []
    for s in sides:
        run(s, None)
        want.append([t.clone() for t in s["out"]])
    torch.cuda.synchronize()
    for _ in range(5):
        for s in sides:
            run(s, s["stream"])
    torch.cuda.synchronize()
    for s, w in zip(sides, want):
        assert all(torch.equal(a, b) for a, b in zip(s["out"], w))
