"""Kernels that may start before the one in front of them in their stream has ended: what that one writes is read by ordinary loads, which the
wait orders, and not through the read-only path, which is for data that stays the same for as long as the kernel runs.  No value shows the
difference, so the sources are read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2009_03106_b200", "csrc")


def definition(file, name):
    """Parameters and body of a function."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    start = re.search(r"\b%s\(" % name, text).end()

    def matching(i, opening, closing):
        depth = 1
        while depth:
            depth += {opening: 1, closing: -1}.get(text[i], 0)
            i += 1
        return i

    end = matching(start, "(", ")")
    body = text.index("{", end) + 1
    return text[start:end], text[body:matching(body, "{", "}")]


@pytest.mark.parametrize("file,name", [
    ("kernels_stored.cuh", "stored_grad_kernel"), ("kernels_relbias.cuh", "relbias_finish_kernel"), ("kernels_qknorm.cuh", "qknorm_finish_kernel"),
    ("kernels_gated.cuh", "gated_reduce_kernel"), ("kernels_gated.cuh", "gated_tc_kernel"), ("kernels_gated.cuh", "gated_end"),
    ("kernels_gated_f32.cuh", "gated_tc3_kernel"), ("kernels_stream.cuh", "factors_kernel"), ("kernels_stream.cuh", "factors_rows_kernel"),
    ("kernels_tc_pair.cuh", "row_factor"), ("kernels_group.cuh", "zta_group_kernel")])
def test_results_of_the_launch_in_front_are_read_by_ordinary_loads(file, name):
    parameters, body = definition(file, name)
    assert "__ldg" not in body and "ld.global.nc" not in body
    assert not re.search(r"const\s+\w+\s*\*\s*__restrict__", parameters)
