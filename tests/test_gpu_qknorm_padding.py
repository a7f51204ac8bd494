"""Norms of queries and keys, backward: rows of padding come out as zeros whatever stands anywhere else."""
import pytest
import torch

from test_gpu_block_attention import BF16, F32, qk_inputs
from test_gpu_qknorm_edges import CASES, check_gradients, dp, run          # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", CASES)
def test_padding_beside_gains_that_are_not_finite(dp, case, dtype):        # noqa: F811
    """The gain's gradient has no factor of the gain, so it stays what it is; a padding row of dx is zero."""
    s = qk_inputs(case, dtype, "dense", True)
    s["gain_q"][0], s["gain_k"][1] = float("nan"), float("inf")
    out = run(dp, s, case, dtype, s["pos"], 1e-5)
    there = ((s["pos"] >= 0) & (s["pos"] < s["n_pos"]))[..., None, None]
    check_gradients(s, case, dtype, out, there, 1e-5)
    for n in ("q", "k"):
        assert bool((out[n].cpu()[~there.expand_as(out[n])] == 0).all())
