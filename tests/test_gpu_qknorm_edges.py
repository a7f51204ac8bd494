"""Norms of queries and keys, backward: settings at which a value that does not count is not finite.  Tolerances as in
test_gpu_block_attention.py."""
import pytest
import torch

from test_gpu_block_attention import BF16, F32, HALF_STEP, U32, close, guarded, qk_inputs, qk_reference, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dp():
    import paper_2009_03106_b200 as pkg
    pkg.load_library()
    return pkg


# Heads that do not fill the heads of a warp, in every form: 16-byte runs, single elements, rings of copies
CASES = [(2, 5, 3, 1, 64, 64, False), (2, 5, 3, 1, 50, 20, True), (2, 7, 5, 2, 128, 64, False), (1, 300, 2, 1, 33, 6, False),
         (2, 2400, 9, 3, 64, 64, False), (3, 2000, 9, 2, 128, 128, True)]


def run(dp, s, case, dtype, pos, eps):
    B, T, Hq, Hk, D, rot, inter = case
    dev = {n: s[n].cuda() for n in ("q", "k", "dq", "dk", "gain_q", "gain_k")}
    out = {}
    for n, H in (("q", Hq), ("k", Hk)):
        for m, shape, dt in ((n, (B, T, H, D), dtype), ("grads_" + n, (B, D), F32), ("sq_" + n, (B,), F32)):
            out[m] = guarded(shape, dt)
    ws = workspace(dp, dp.dpclip_qknorm_workspace_bytes(B, T, Hq, Hk, D))
    dp.dpclip_qknorm_backward(dev["dq"], dev["dk"], dev["q"], dev["k"], dev["gain_q"], dev["gain_k"], s["table"].cuda(),
                              *(out[n][0] for n in ("q", "k", "grads_q", "grads_k", "sq_q", "sq_k")), ws, interleaved=inter, positions=pos.cuda(), eps=eps)
    torch.cuda.synchronize()
    for _, check in out.values():
        check()
    return {n: t for n, (t, _) in out.items()}


def check_gradients(s, case, dtype, out, keep, eps):
    cs = s["table"].double()[s["pos"].long().clamp(0, s["n_pos"] - 1)][:, :, None]
    for n in ("q", "k"):
        _, _, G, Gm = qk_reference(s[n].nan_to_num(), None, cs[..., 0, :], cs[..., 1, :], case[5], case[6], eps, s["d" + n].nan_to_num())
        want, mag = torch.where(keep, G, 0.0).sum((1, 2)), torch.where(keep, Gm, 0.0).sum((1, 2))
        depth = (40 + case[1] * s[n].shape[2]) * U32
        close(out["grads_" + n], want, depth * mag)
        close(out["sq_" + n], want.square().sum(1), (2 * depth * mag * want.abs() + (depth * mag) ** 2).sum(1) + (case[4] + 8) * U32 * want.square().sum(1))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", CASES)
def test_gradients_without_epsilon(dp, case, dtype):
    """eps = 0: the root of nothing is infinite where a warp has no head."""
    s = qk_inputs(case, dtype, "dense", False)
    out = run(dp, s, case, dtype, s["pos"], 0.0)
    check_gradients(s, case, dtype, out, torch.tensor(True), 0.0)
    cs = s["table"].double()[s["pos"].long()][:, :, None]
    for n in ("q", "k"):
        dx, dm, _, _ = qk_reference(s[n], s["gain_" + n], cs[..., 0, :], cs[..., 1, :], case[5], case[6], 0.0, s["d" + n])
        close(out[n], dx, HALF_STEP[dtype] * dx.abs() + 60 * U32 * dm)
