"""Cases for the operators of a transformer block: the learned relative position bias, the norms of queries and keys with
the rotation, and the gated feed-forward block, each with its backward pass as per-example clipping needs it.

  relbias_forward   the bias [H][Tq][Tk] from the bucket table
  relbias_grad      from dL/dS of every example: the per-example gradients of the table, their squared norms, the clipped sum
  qknorm_forward    queries and keys, each head divided by its root mean square, times the gain, rotated by position
  qknorm_grad       dL/dq and dL/dk of the inputs, the per-example gradients of both gains, their squared norms, clipped sums
  gated_forward     act(X Wg^T + bg) (.) (X Wu^T + bu), and both projections' outputs where the backward pass wants them
  gated_grad        the signals dL/dZ of both projections (what the clipping step reads) and dL/dX

`prepare` draws on the GPU; `run` is one pass; the plain forms are written with elementary torch operations in fp32.
"""
import math

import torch

own = False
MASKED = float("nan")                   # what padded places of a batch may hold


# ---------------------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decoded token of a sequence: one row of the bias, all latency
        dict(name="relbias_token", kind="relbias_forward", dtype="bf16", H=8, Tq=1, Tk=777, q_offset=776, n_buckets=32,
             max_distance=128, bidirectional=False, causal=True),
        # the bias of a long sequence, made once a step for all layers
        dict(name="relbias_long_bf16", kind="relbias_forward", dtype="bf16", H=16, Tq=2048, Tk=2048, q_offset=0, n_buckets=32,
             max_distance=128, bidirectional=True, causal=False),
        # the gradient of the table in the sequence model: batch 128, 256 positions, eight heads of 64
        dict(name="relbias_grad_bf16", kind="relbias_grad", dtype="bf16", B=128, H=8, Tq=256, Tk=256, q_offset=0, n_buckets=32,
             max_distance=128, bidirectional=True, causal=False, padded=False),
        # the text model's sentences, padded to 77 words, causal, in fp32
        dict(name="relbias_grad_ragged_f32", kind="relbias_grad", dtype="f32", B=50, H=6, Tq=77, Tk=77, q_offset=0, n_buckets=32,
             max_distance=50, bidirectional=False, causal=True, padded=True),
        # one token of each of 32 sequences
        dict(name="qknorm_tokens_bf16", kind="qknorm_forward", dtype="bf16", B=32, T=1, Hq=8, Hk=2, D=64, rot=64,
             interleaved=False, padded=False),
        # queries and keys of the sequence model
        dict(name="qknorm_bf16", kind="qknorm_forward", dtype="bf16", B=128, T=256, Hq=8, Hk=8, D=64, rot=64,
             interleaved=False, padded=False),
        # grouped heads of 128 in training
        dict(name="qknorm_grad_bf16", kind="qknorm_grad", dtype="bf16", B=128, T=256, Hq=16, Hk=2, D=128, rot=128,
             interleaved=False, padded=False),
        # the text model: 300 columns in six heads of 50, padded sentences, pairs side by side, a part of the head rotated
        dict(name="qknorm_grad_ragged_f32", kind="qknorm_grad", dtype="f32", B=50, T=77, Hq=6, Hk=6, D=50, rot=32,
             interleaved=True, padded=True),
        # a few tokens through the block: weights are all there is to read
        dict(name="gated_tokens_bf16", kind="gated_forward", dtype="bf16", M=4, K=1024, F=4096, act="silu", bias=False, keep=False),
        # the feed-forward layers of the sequence model, in training
        dict(name="gated_bf16", kind="gated_forward", dtype="bf16", M=32768, K=512, F=2048, act="gelu_tanh", bias=False, keep=True),
        # the largest: the backward pass of a wide block
        dict(name="gated_grad_bf16", kind="gated_grad", dtype="bf16", M=32768, K=1024, F=4096, act="silu", bias=False),
        # the text model in fp32: 50 sentences of 77 words, widths that fit no tile
        dict(name="gated_ragged_f32", kind="gated_forward", dtype="f32", M=3850, K=300, F=1100, act="gelu", bias=True, keep=True),
    ]


def _size(rng, lo, hi):
    """Spread over the logarithm of the range, odd sizes among them."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["relbias_forward", "relbias_grad", "qknorm_forward", "qknorm_grad", "gated_forward", "gated_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("relbias"):
        both = rng.random() < 0.5
        n_buckets = 2 * rng.randint(2, 64)
        c = dict(kind=kind, dtype=dtype, n_buckets=n_buckets, max_distance=n_buckets + _size(rng, 1, 4000), bidirectional=both,
                 causal=rng.random() < 0.4)
        limit = (64 if kind == "relbias_forward" else 67) * 10 ** 6 // (1 if dtype == "bf16" else 2)
        H = rng.randint(1, 24)
        Tk = _size(rng, 1, 3000)
        Tq = Tk if rng.random() < 0.5 else _size(rng, 1, 3000)
        if rng.random() < 0.4:                                          # rows that are 16-byte multiples
            Tk = -(-Tk // 8) * 8
        if c["causal"] and not both and Tq > Tk:
            Tq = Tk
        if kind == "relbias_forward":
            while H * Tq * Tk > limit:
                H, Tq = max(1, H // 2), max(1, Tq // 2)
            return dict(c, H=H, Tq=Tq, Tk=Tk, q_offset=max(0, Tk - Tq) if c["causal"] else 0)
        while H * Tq * Tk > limit // 2:
            H, Tq = max(1, H // 2), max(1, Tq // 2)
        B = _size(rng, 1, max(1, min(512, limit // (H * Tq * Tk))))
        return dict(c, B=B, H=H, Tq=Tq, Tk=Tk, q_offset=max(0, Tk - Tq) if c["causal"] else 0, padded=rng.random() < 0.4)
    if kind.startswith("qknorm"):
        D = rng.choice([32, 48, 50, 64, 64, 80, 96, 100, 128, 128, 160, 256])
        rot = D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2)
        Hk = rng.choice([1, 2, 4, 6, 8])
        Hq = Hk * rng.choice([1, 2, 4])
        limit = 75 * 10 ** 6 // (1 if dtype == "bf16" else 2)
        tokens = _size(rng, 1, max(1, min(40000, limit // ((Hq + 2 * Hk) * D))))
        T = 1 if rng.random() < 0.15 else _size(rng, 1, min(tokens, 2048))
        return dict(kind=kind, dtype=dtype, B=max(1, tokens // T), T=T, Hq=Hq, Hk=Hk, D=D, rot=rot,
                    interleaved=rng.random() < 0.5, padded=T > 1 and rng.random() < 0.4)
    aligned = rng.random() < 0.6
    K, F = _size(rng, 64, 2000), _size(rng, 64, 5000)
    if aligned:
        K, F = -(-K // 8) * 8, -(-F // 8) * 8
    limit = 1.2e11 if dtype == "bf16" and aligned else 6e9
    M = _size(rng, 1, max(1, min(32768, int(limit / (K * F)))))
    c = dict(kind=kind, dtype=dtype, M=M, K=K, F=F, act=rng.choice(["silu", "gelu", "gelu_tanh", "relu"]), bias=rng.random() < 0.4)
    return dict(c, keep=rng.random() < 0.6) if kind == "gated_forward" else c


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lens(g, B, T):
    """Lengths of a padded batch: one full example, one of length zero where there are more than two."""
    n = torch.randint(1, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[0] = T
    if B > 2:
        n[B - 1] = 0
    return n


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, kind = _type(case), case["kind"]
    normal = lambda *shape, std=1.0: torch.randn(shape, generator=g, device="cuda") * std                # noqa: E731
    s = {"case": case, "buf": {}}
    if kind == "relbias_forward":
        s["table"] = normal(case["n_buckets"], case["H"])
    elif kind == "relbias_grad":
        B, H, Tq, Tk = case["B"], case["H"], case["Tq"], case["Tk"]
        # dL/dS of a softmax: small against the probabilities' mean, and rows that sum to about zero
        dS = torch.randn((B, H, Tq, Tk), generator=g, device="cuda", dtype=dt) * (1.0 / Tk)
        s["q_lens"] = s["k_lens"] = None
        if case["padded"]:
            s["k_lens"] = _lens(g, B, Tk)
            s["q_lens"] = s["k_lens"].clamp(max=Tq) if Tq != Tk else s["k_lens"]
            pad = torch.arange(Tk, device="cuda")[None, :] >= s["k_lens"][:, None]
            dS.masked_fill_(pad[:, None, None, :], MASKED)
        s["dS"] = dS
        s["clip"] = torch.rand((B,), generator=g, device="cuda") * 0.9 + 0.1
    elif kind.startswith("qknorm"):
        B, T, Hq, Hk, D, rot = (case[k] for k in ("B", "T", "Hq", "Hk", "D", "rot"))
        # queries and keys lie in the rows of one projection, the values behind them
        qkv = normal(B, T, (Hq + 2 * Hk) * D).to(dt)
        s["q"] = qkv[..., :Hq * D].unflatten(-1, (Hq, D))
        s["k"] = qkv[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D))
        s["gain_q"], s["gain_k"] = 1 + 0.2 * normal(D), 1 + 0.2 * normal(D)
        # a single token stands at the end of its sequence
        s["n_pos"] = n_pos = max(T, 1) if T > 1 else 4096
        angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / rot)[None, :]
        s["rotation"] = torch.stack([angle.cos(), angle.sin()], 1).float()                              # (n_pos, 2, rot / 2)
        if T > 1:
            pos = torch.arange(T, device="cuda", dtype=torch.int32).repeat(B, 1)
            if case["padded"]:
                pos = torch.where(pos < _lens(g, B, T)[:, None], pos, -1)
        else:
            pos = torch.randint(0, n_pos, (B, 1), generator=g, device="cuda", dtype=torch.int32)
        s["positions"] = pos.contiguous()
        if kind == "qknorm_forward":
            s["q_out"] = torch.full((B, T, Hq, D), 0.5, device="cuda", dtype=dt)
            s["k_out"] = torch.full((B, T, Hk, D), 0.5, device="cuda", dtype=dt)
        else:
            s["dq_out"], s["dk_out"] = normal(B, T, Hq, D, std=0.05).to(dt), normal(B, T, Hk, D, std=0.05).to(dt)
            s["clip"] = torch.rand((B,), generator=g, device="cuda") * 0.9 + 0.1
    else:
        M, K, F = case["M"], case["K"], case["F"]
        s["W"] = normal(2 * F, K, std=1 / math.sqrt(K)).to(dt)                                          # gate rows, then up rows
        s["bias"] = 0.5 * normal(2 * F) if case["bias"] else None
        if kind == "gated_forward":
            s["X"] = torch.randn((M, K), generator=g, device="cuda", dtype=dt)
        else:
            s["Z"] = torch.randn((M, 2 * F), generator=g, device="cuda", dtype=dt)
            s["dH"] = torch.randn((M, F), generator=g, device="cuda", dtype=dt) * 0.05
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _buckets(case):
    """Bucket of every distance key position - query position, and the smallest distance: near distances one bucket each,
    far ones on a logarithmic scale up to max_distance.  In 64 bits, and whole numbers of the logarithm as such."""
    lo = -(case["q_offset"] + case["Tq"] - 1)
    rel = torch.arange(lo, case["Tk"] - case["q_offset"], device="cuda")
    n = case["n_buckets"]
    base = torch.zeros_like(rel)
    if case["bidirectional"]:
        n //= 2
        base, dist = (rel > 0) * n, rel.abs()
    else:
        dist = (-rel).clamp(min=0)
    exact_n = n // 2
    v = torch.log(dist.clamp(min=1).double() / exact_n) / math.log(case["max_distance"] / exact_n) * (n - exact_n)
    v = torch.where((v - v.round()).abs() < 1e-9, v.round(), v.floor())
    far = (exact_n + v.long()).clamp(max=n - 1)
    return base + torch.where(dist < exact_n, dist, far), lo


def _seen(case, s):
    """Which (example, query, key) count: [B or 1][1][Tq][Tk], or None for all."""
    q = torch.arange(case["Tq"], device="cuda")[:, None]
    k = torch.arange(case["Tk"], device="cuda")[None, :]
    seen = None
    if case["causal"]:
        seen = (k <= q + case["q_offset"])[None, None]
    if s.get("k_lens") is not None:
        inside = (k[None] < s["k_lens"][:, None, None]) & (q[None] < s["q_lens"][:, None, None])
        seen = inside[:, None] if seen is None else seen & inside[:, None]
    return seen


def _rotate(x, cos, sin, rot, interleaved, back=False):
    sin = -sin if back else sin
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., rot:]], -1)


EPS = 1e-6


def _act(z, act):
    """The activation and its derivative."""
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p))
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * c, c + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    t = torch.tanh(u)
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def _plain_relbias_forward(s):
    case = s["case"]
    bucket, lo = _buckets(case)
    line = s["table"][bucket]                                             # (distances, H)
    q = torch.arange(case["Tq"], device="cuda")[:, None] + case["q_offset"]
    k = torch.arange(case["Tk"], device="cuda")[None, :]
    out = line.t()[:, (k - q) - lo]
    if case["causal"]:
        out = torch.where(k <= q, out, float("-inf"))
    return {"bias": out.to(_type(case))}


def _plain_relbias_grad(s):
    case = s["case"]
    B, H, Tq, Tk = case["B"], case["H"], case["Tq"], case["Tk"]
    x = s["dS"].float()
    seen = _seen(case, s)
    if seen is not None:
        x = torch.where(seen, x, 0.0)
    # the sum along every diagonal: the rows are shifted against one another by padding them to one element more
    x = torch.nn.functional.pad(x.flip(2), (0, Tq)).flatten(2)[:, :, :Tq * (Tq + Tk - 1)]
    line = x.unflatten(2, (Tq, Tq + Tk - 1)).sum(2)
    bucket, _ = _buckets(case)
    one = (bucket[:, None] == torch.arange(case["n_buckets"], device="cuda")[None, :]).double()
    G = (line.double() @ one).transpose(1, 2)                             # (B, n_buckets, H)
    return {"grads": G.float(), "sq": G.square().sum((1, 2)).float(), "sum": torch.einsum("b,bnh->nh", s["clip"].double(), G).float()}


def _plain_qknorm_forward(s):
    case = s["case"]
    pos = s["positions"].long()
    cs = s["rotation"][pos.clamp(min=0)][:, :, None]                      # (B, T, 1, 2, rot / 2)
    out = {}
    for n in ("q", "k"):
        x = s[n].float()
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s["gain_" + n]
        y = _rotate(y, cs[..., 0, :], cs[..., 1, :], case["rot"], case["interleaved"]).to(_type(case))
        out[n] = torch.where((pos >= 0)[..., None, None], y, s[n + "_out"])
    return out


def _plain_qknorm_grad(s):
    case = s["case"]
    pos = s["positions"].long()
    cs = s["rotation"][pos.clamp(min=0)][:, :, None]
    there = (pos >= 0)[..., None, None]
    out = {}
    for n in ("q", "k"):
        x = s[n].float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        xh = x * r
        g = _rotate(s["d%s_out" % n].float(), cs[..., 0, :], cs[..., 1, :], case["rot"], case["interleaved"], back=True)
        g = torch.where(there, g, 0.0)
        w = g * s["gain_" + n]
        dx = r * (w - xh * (w * xh).mean(-1, keepdim=True))
        G = (g * xh).sum((1, 2))
        out["d" + n] = torch.where(there, dx, 0.0).to(_type(case))
        out["grads_" + n], out["sq_" + n], out["sum_" + n] = G, G.square().sum(1), (s["clip"][:, None] * G).sum(0)
    return out


def _plain_gated_forward(s):
    case = s["case"]
    z = s["X"].float() @ s["W"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"]
    F = case["F"]
    h = _act(z[:, :F], case["act"])[0] * z[:, F:]
    return {"H": h.to(_type(case)), "Z": z.to(_type(case))} if case["keep"] else {"H": h.to(_type(case))}


def _plain_gated_grad(s):
    case = s["case"]
    F = case["F"]
    z, dh = s["Z"].float(), s["dH"].float()
    a, da = _act(z[:, :F], case["act"])
    dz = torch.cat([dh * z[:, F:] * da, dh * a], 1)
    return {"dZ": dz.to(_type(case)), "dX": (dz @ s["W"].float()).to(_type(case))}


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _buffers(s, **shapes):
    """Outputs that a program keeps from step to step."""
    for n, (shape, dt) in shapes.items():
        if n not in s["buf"]:
            s["buf"][n] = torch.empty(shape, device="cuda", dtype=dt)
    return s["buf"]


def _workspace(s, dp, nbytes):
    if "ws" not in s["buf"]:
        s["buf"]["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
        dp.dpclip_workspace_init(s["buf"]["ws"])
    return s["buf"]["ws"]


def _own(s):
    import paper_2009_03106_b200 as dp
    case, dt, f32 = s["case"], _type(s["case"]), torch.float32
    kind = case["kind"]
    if kind.startswith("relbias"):
        nb, H, Tq, Tk = case["n_buckets"], case["H"], case["Tq"], case["Tk"]
        how = dict(max_distance=case["max_distance"], bidirectional=case["bidirectional"], causal=case["causal"],
                   q_offset=case["q_offset"])
        if kind == "relbias_forward":
            b = _buffers(s, bias=((H, Tq, Tk), dt))
            dp.dpclip_relbias_forward(s["table"], b["bias"], **how)
            return {"bias": b["bias"]}
        B = case["B"]
        b = _buffers(s, grads=((B, nb, H), f32), sq=((B,), f32), sum=((nb, H), f32))
        ws = s["buf"].get("ws")
        if ws is None:
            ws = _workspace(s, dp, dp.dpclip_relbias_workspace_bytes(B, H, Tq, Tk, nb, dp.DPCLIP_F32 if dt == f32 else dp.DPCLIP_BF16))
        dp.dpclip_relbias_sqnorms(s["dS"], b["grads"], b["sq"], ws, q_lens=s["q_lens"], k_lens=s["k_lens"], **how)
        dp.dpclip_stored_clipped_grad(b["grads"], s["clip"], b["sum"])
        return {n: b[n] for n in ("grads", "sq", "sum")}
    if kind.startswith("qknorm"):
        how = dict(rot_dim=case["rot"], interleaved=case["interleaved"], positions=s["positions"], eps=EPS)
        if kind == "qknorm_forward":
            dp.dpclip_qknorm_forward(s["q"], s["k"], s["gain_q"], s["gain_k"], s["rotation"], s["q_out"], s["k_out"], **how)
            return {"q": s["q_out"], "k": s["k_out"]}
        B, T, Hq, Hk, D = (case[k] for k in ("B", "T", "Hq", "Hk", "D"))
        b = _buffers(s, dq=((B, T, Hq, D), dt), dk=((B, T, Hk, D), dt), grads_q=((B, D), f32), grads_k=((B, D), f32),
                     sq_q=((B,), f32), sq_k=((B,), f32), sum_q=((D,), f32), sum_k=((D,), f32))
        ws = s["buf"].get("ws")
        if ws is None:
            ws = _workspace(s, dp, dp.dpclip_qknorm_workspace_bytes(B, T, Hq, Hk, D))
        dp.dpclip_qknorm_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["gain_q"], s["gain_k"], s["rotation"], b["dq"], b["dk"],
                                  b["grads_q"], b["grads_k"], b["sq_q"], b["sq_k"], ws, **how)
        dp.dpclip_stored_clipped_grad(b["grads_q"], s["clip"], b["sum_q"])
        dp.dpclip_stored_clipped_grad(b["grads_k"], s["clip"], b["sum_k"])
        return {n: b[n] for n in ("dq", "dk", "grads_q", "grads_k", "sq_q", "sq_k", "sum_q", "sum_k")}
    M, K, F = case["M"], case["K"], case["F"]
    act = {"silu": dp.DPCLIP_ACT_SILU, "gelu": dp.DPCLIP_ACT_GELU, "gelu_tanh": dp.DPCLIP_ACT_GELU_TANH, "relu": dp.DPCLIP_ACT_RELU}[case["act"]]
    ws = s["buf"].get("ws")
    if ws is None:
        ws = _workspace(s, dp, dp.dpclip_gated_workspace_bytes(M, K, F, dp.DPCLIP_F32 if dt == f32 else dp.DPCLIP_BF16))
    if kind == "gated_forward":
        b = _buffers(s, H=((M, F), dt), **({"Z": ((M, 2 * F), dt)} if case["keep"] else {}))
        dp.dpclip_gated_forward(s["X"], s["W"], s["bias"], b["H"], b.get("Z"), act, ws)
        return {n: b[n] for n in ("H", "Z") if n in b}
    b = _buffers(s, dZ=((M, 2 * F), dt), dX=((M, K), dt))
    dp.dpclip_gated_backward(s["dH"], s["Z"], s["W"], b["dZ"], b["dX"], act, ws)
    return {"dZ": b["dZ"], "dX": b["dX"]}


PLAIN = dict(relbias_forward=_plain_relbias_forward, relbias_grad=_plain_relbias_grad, qknorm_forward=_plain_qknorm_forward,
             qknorm_grad=_plain_qknorm_grad, gated_forward=_plain_gated_forward, gated_grad=_plain_gated_grad)


def run(state):
    return _own(state) if own else PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind.startswith("relbias"):
        pairs = case["Tq"] * case["Tk"]
        table = case["n_buckets"] * case["H"] * 4
        if kind == "relbias_forward":
            return {"bytes": es * case["H"] * pairs + table, "flops": 0}
        B = case["B"]
        read = sum(min(case["Tk"], q + case["q_offset"] + 1) for q in range(case["Tq"])) if case["causal"] else pairs
        read = read // 2 if case["padded"] else read                      # lengths are spread over the whole range
        return {"bytes": es * B * case["H"] * read + (B + 1) * table, "flops": B * case["H"] * read}
    if kind.startswith("qknorm"):
        n = case["B"] * case["T"] * (case["Hq"] + case["Hk"]) * case["D"]
        n = n // 2 if case["padded"] else n
        tables = case["B"] * case["T"] * 4 + min(case["B"] * case["T"], max(case["T"], 1) if case["T"] > 1 else 4096) * case["rot"] * 4
        return {"bytes": n * es * (2 if kind == "qknorm_forward" else 3) + tables, "flops": n * (8 if kind == "qknorm_forward" else 16)}
    M, K, F = case["M"], case["K"], case["F"]
    flops = 4 * M * K * F
    if kind == "gated_forward":
        return {"bytes": es * (M * K + 2 * F * K + M * F + (2 * M * F if case["keep"] else 0)), "flops": flops}
    return {"bytes": es * (5 * M * F + 2 * F * K + M * K), "flops": flops}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _bucket_of(rel, n_buckets, max_distance, bidirectional):
    """Whole numbers only: floor(m log(d / e) / log(D / e)) is the largest k with d^m e^k >= D^k e^m."""
    n, base = n_buckets, 0
    if bidirectional:
        n //= 2
        base, d = (n if rel > 0 else 0), abs(rel)
    else:
        d = max(-rel, 0)
    e = n // 2
    if d < e:
        return base + d
    m, k = n - e, 0
    while k < m - 1 and d ** m * e ** (k + 1) >= max_distance ** (k + 1) * e ** m:
        k += 1
    return base + e + k


def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind.startswith("relbias"):
        Tq, Tk, off, H, nb = case["Tq"], case["Tk"], case["q_offset"], case["H"], case["n_buckets"]
        known = {}
        for rel in range(-(off + Tq - 1), Tk - off):
            far = max(-case["max_distance"], min(case["max_distance"], rel))
            if far not in known:
                known[far] = _bucket_of(far, nb, case["max_distance"], case["bidirectional"])
            known[rel] = known[far]
        first = -(off + Tq - 1)
        of_rel = torch.tensor([known[r] for r in range(first, Tk - off)], device="cuda")
        row = torch.arange(Tq, device="cuda")
        if kind == "relbias_forward":
            out = torch.empty((H, Tq, Tk), dtype=f64, device="cuda")
            for q in range(Tq):
                at = of_rel[Tq - 1 - q:Tq - 1 - q + Tk]
                out[:, q] = s["table"].double()[at].t()
                if case["causal"]:
                    out[:, q, q + off + 1:] = -math.inf
            return {"bias": out}
        G = torch.zeros((case["B"], H, nb), dtype=f64, device="cuda")
        col = torch.arange(Tk, device="cuda")
        for q in range(Tq):
            x = s["dS"][:, :, q].double()
            drop = torch.zeros((case["B"], Tk), dtype=torch.bool, device="cuda")
            if case["causal"]:
                drop |= (col > q + off)[None]
            if s["k_lens"] is not None:
                drop |= (col[None] >= s["k_lens"][:, None]) | (row[q] >= s["q_lens"])[:, None]
            x = x.masked_fill(drop[:, None], 0.0)
            at = of_rel[Tq - 1 - q:Tq - 1 - q + Tk]
            G += x @ torch.nn.functional.one_hot(at, nb).double()
        G = G.transpose(1, 2)
        return {"grads": G, "sq": G.pow(2).sum((1, 2)), "sum": (s["clip"].double()[:, None, None] * G).sum(0)}
    if kind.startswith("qknorm"):
        rot, D = case["rot"], case["D"]
        pos = s["positions"].long()
        there = pos >= 0
        c, sn = (s["rotation"].double()[pos.clamp(min=0), j][:, :, None] for j in (0, 1))
        # the rotation as a product with a matrix of columns: y[first] = c a - s b, y[second] = s a + c b
        i = torch.arange(rot // 2, device="cuda")
        first, second = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
        out = {}
        for n in ("q", "k"):
            x = s[n].double()
            inv = (x.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5)
            gain = s["gain_" + n].double()
            if kind == "qknorm_forward":
                y = x * inv * gain
                turned = y.clone()
                turned[..., first] = c * y[..., first] - sn * y[..., second]
                turned[..., second] = sn * y[..., first] + c * y[..., second]
                turned[~there] = s[n + "_out"][~there].double()
                out[n] = turned
                continue
            dy = s["d%s_out" % n].double()
            g = dy.clone()
            g[..., first] = c * dy[..., first] + sn * dy[..., second]
            g[..., second] = c * dy[..., second] - sn * dy[..., first]
            g[~there] = 0
            # y = gain x inv: dx = inv gain g - x inv^3 sum(gain g x) / D
            dx = inv * gain * g - x * inv.pow(3) * (gain * g * x).sum(-1, keepdim=True) / D
            G = (g * x * inv).sum((1, 2))
            out["d" + n], out["grads_" + n], out["sq_" + n] = dx, G, G.pow(2).sum(1)
            out["sum_" + n] = s["clip"].double() @ G
        return out
    F, act = case["F"], case["act"]
    if case["M"] * case["K"] * F > 2e11:
        return None
    W = s["W"].double()

    def value(z):
        if act == "silu":
            return z / (1 + torch.exp(-z))
        if act == "relu":
            return torch.where(z > 0, z, 0.0)
        if act == "gelu":
            return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))

    if kind == "gated_forward":
        x = s["X"].double()
        zg, zu = x @ W[:F].t(), x @ W[F:].t()
        if s["bias"] is not None:
            zg, zu = zg + s["bias"][:F].double(), zu + s["bias"][F:].double()
        h = value(zg) * zu
        return {"H": h, "Z": torch.cat([zg, zu], 1)} if case["keep"] else {"H": h}
    zg, zu = s["Z"][:, :F].double().requires_grad_(True), s["Z"][:, F:].double()
    a = value(zg)
    slope, = torch.autograd.grad(a.sum(), zg)
    dh = s["dH"].double()
    dg, du = dh * zu * slope, dh * a.detach()
    return {"dZ": torch.cat([dg, du], 1), "dX": dg @ W[:F] + du @ W[F:]}
