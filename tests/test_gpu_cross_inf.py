"""Cross attention where scores are minus infinity: such a state has no weight, wherever in its segment it stands (a lane group's first
one, a whole key tile, a whole share), and a row that sees nothing else gets what the formula gives.  On each of the forward's kernels."""
import pytest
import torch

import layer_ref as R
from paper_2508_21058_b200 import MocCross
from paper_2508_21058_b200.binding import debug_cross_plan

pytestmark = pytest.mark.gpu

# the kernel, whether states are in shares, heads, key heads, d, queries and states of every segment
CASES = [
    ("few", False, 2, 1, 64, [1, 2], [70, 33]),
    ("few", True, 6, 2, 128, [1, 1], [3000, 700]),
    ("one_tile", False, 4, 2, 128, [100, 30], [300, 128]),
    ("one_tile", True, 2, 2, 64, [64], [5000]),
    ("one_tile", True, 3, 1, 128, [100, 128, 9], [1000, 129, 128]),
    ("two_tile", False, 16, 4, 128, [1300, 640], [333, 512]),
    ("two_tile", True, 32, 32, 64, [257], [12000]),
]
PLACES = {
    "first": lambda i, n: i == 0,
    "first tile": lambda i, n: i < 128,
    "first half": lambda i, n: i < n // 2,
    "second half": lambda i, n: i >= n // 2,
    "every other": lambda i, n: i % 2 == 0,
    "all but the last": lambda i, n: i < n,
}


def _offsets(n):
    off = [0]
    for x in n:
        off.append(off[-1] + x)
    return off


def _inputs(H, kv, d, q_len, k_len, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    q = torch.randn(H, sum(q_len), d, generator=gen, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(kv, sum(k_len), d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    q[:, :, 5] = q[:, :, 5].abs() + 0.5                     # times minus infinity it is minus infinity
    return q, k, v


def _run(case, q, k, v):
    _, _, H, kv, d, q_len, k_len = case
    q_off, k_off = _offsets(q_len), _offsets(k_len)
    op = MocCross(H, kv, d, q_off, k_off)
    ws = op.new_workspace()
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    op.moc_cross_attend(q, k, v, o, lse, ws)
    torch.cuda.synchronize()
    assert op.moc_cross_get_status(ws) == (0, 0)
    return o, lse


@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("case", CASES)
def test_a_score_of_minus_infinity_has_no_weight(case, place):
    kernel, shares, H, kv, d, q_len, k_len = case
    q_off, k_off = _offsets(q_len), _offsets(k_len)
    plan = debug_cross_plan(H, kv, d, q_off, k_off, n_sm=torch.cuda.get_device_properties(0).multi_processor_count)
    assert plan[kernel] > 0 and (plan["part_rows"] > 0) == shares
    q, k, v = _inputs(H, kv, d, q_len, k_len, 3)
    gone = torch.zeros(sum(k_len), dtype=torch.bool)
    for a, n in zip(k_off, k_len):
        for i in range(n - 1):                              # (the last state stays)
            gone[a + i] = PLACES[place](i, n)
        if place == "second half":
            gone[a + n - 1], gone[a] = n > 1, False
    k[:, gone, 5] = -float("inf")
    o, lse = _run(case, q, k, v)
    # the same without those states
    keep = ~gone
    left = [int(keep[a:a + n].sum()) for a, n in zip(k_off, k_len)]
    ref = R.CrossRef(q.double(), k[:, keep].double(), v[:, keep].double(), q_len, left, _offsets(left)[:-1], d ** -0.5)
    R.check("O", o, ref.o, ref.o_tol)
    R.check("lse", lse, ref.lse, ref.lse_tol)


@pytest.mark.parametrize("case", CASES)
def test_a_row_of_nothing_but_minus_infinity(case):
    """O is 0 / 0 and lse is minus infinity; other segments' rows are numbers."""
    _, _, H, kv, d, q_len, k_len = case
    q, k, v = _inputs(H, kv, d, q_len, k_len, 4)
    k[:, :k_len[0], 5] = -float("inf")
    o, lse = _run(case, q, k, v)
    first = slice(0, q_len[0])
    assert bool(torch.isnan(o[:, first]).all()) and bool((lse[:, first] == -float("inf")).all())
    assert bool(torch.isfinite(o[:, q_len[0]:]).all()) and bool(torch.isfinite(lse[:, q_len[0]:]).all())


@pytest.mark.parametrize("case", CASES)
def test_a_value_without_weight_that_is_not_a_number(case):
    """Its weight is zero, and zero times NaN is NaN, as in the formula; in that channel alone."""
    _, _, H, kv, d, q_len, k_len = case
    q, k, v = _inputs(H, kv, d, q_len, k_len, 5)
    k[:, 0, 5] = -float("inf")
    v[:, 0, 9] = float("nan")
    o, lse = _run(case, q, k, v)
    channels = torch.arange(d, device="cuda") == 9
    assert bool(torch.isnan(o[:, :q_len[0], channels]).all()) and bool(torch.isfinite(o[:, :, ~channels]).all())
    assert bool(torch.isfinite(o[:, q_len[0]:]).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("case", [c for c in CASES if sum(c[5]) < 500])
def test_gradients_of_states_without_weight(case, place):
    """dK and dV of a state that weighs nothing are zero (its dP times zero; the queries that a last tile lacks have no part in it), and
    the others' are as without it.  (dQ is a sum over the states, of which zero times minus infinity is one: NaN by the formula.)"""
    _, _, H, kv, d, q_len, k_len = case
    q_off, k_off = _offsets(q_len), _offsets(k_len)
    q, k, v = _inputs(H, kv, d, q_len, k_len, 6)
    do = torch.randn(q.shape, generator=torch.Generator("cuda").manual_seed(7), device="cuda").to(torch.bfloat16)
    gone = torch.zeros(sum(k_len), dtype=torch.bool)
    for a, n in zip(k_off, k_len):
        for i in range(n - 1):
            gone[a + i] = PLACES[place](i, n)
    k[:, gone, 5] = -float("inf")
    op = MocCross(H, kv, d, q_off, k_off)
    ws = op.new_workspace(with_bwd=True)
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)
    op.moc_cross_attend(q, k, v, o, lse, ws)
    op.moc_cross_attend_bwd(q, k, v, o, lse, do, dq, dk, dv, ws)
    torch.cuda.synchronize()
    assert op.moc_cross_get_status(ws) == (0, 0)
    keep = ~gone
    left = [int(keep[a:a + n].sum()) for a, n in zip(k_off, k_len)]
    ref = R.CrossRef(q.double(), k[:, keep].double(), v[:, keep].double(), q_len, left, _offsets(left)[:-1], d ** -0.5, do.double())
    R.check("dK", dk[:, keep], ref.dk, ref.dk_tol)
    R.check("dV", dv[:, keep], ref.dv, ref.dv_tol)
    assert bool((dk[:, gone] == 0).all()) and bool((dv[:, gone] == 0).all())
