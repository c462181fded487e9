"""Cross attention whose plan cuts a few long lists among many short ones, forward and backward, against the 64-bit plain form."""
import pytest

import test_gpu_cross as T
from paper_2508_21058_b200.binding import debug_cross_plan

pytestmark = T.pytestmark


@pytest.mark.parametrize("case", [(24, 8, 128, [200] * 40, [15000] + [77] * 39, 3), (16, 16, 64, [300] * 30, [100] * 29 + [9000], 0),
                                  (8, 8, 128, [16] * 100, [128] * 99 + [20000], 1)])
def test_a_long_list_among_short_ones(case):
    run = T.Run(case, seed=21)
    plan = debug_cross_plan(*case[:3], run.q_off, run.k_off, run.k_len)
    assert plan["part_rows"] > 0 and plan["two_tile"] + plan["one_tile"] > 4 * 148
    run.forward().backward().check()
    first = [t.clone() for t in run.outputs()]
    run.forward().backward()
    assert all((a == b).all() for a, b in zip(first, run.outputs()))
