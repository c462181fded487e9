"""Cross attention to no states at all: tensors of no rows, or none that any segment has."""
import pytest
import torch

from paper_2508_21058_b200 import MocCross

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [0, 3])
@pytest.mark.parametrize("H,kv,d,q_len", [(2, 1, 64, [5]), (24, 8, 128, [300, 0, 129]), (1, 1, 128, [1]), (6, 6, 64, [5000])])
def test_no_states_at_all(H, kv, d, q_len, rows):
    n = sum(q_len)
    q_off = [sum(q_len[:i]) for i in range(len(q_len) + 1)]
    op = MocCross(H, kv, d, q_off, [0] * len(q_off))
    ws = op.new_workspace(with_bwd=True)
    q, do, o, dq = (torch.full((H, n, d), x, dtype=torch.bfloat16, device="cuda") for x in (1.0, float("nan"), 7.0, 7.0))
    k, v, dk, dv = (torch.full((kv, rows, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    lse = torch.zeros(H, n, device="cuda")
    op.moc_cross_attend(q, k, v, o, lse, ws)
    op.moc_cross_attend_bwd(q, k, v, o, lse, do, dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert op.moc_cross_get_status(ws) == (0, 0)
    assert bool((o == 0).all()) and bool((lse == -float("inf")).all()) and bool((dq == 0).all())
    assert bool((dk == 7.0).all()) and bool((dv == 7.0).all())
