"""What the plan of a cross attention launches (the rules of csrc/moc_cross.cu, through their host-only hook)."""
import random

import pytest

from paper_2508_21058_b200 import MocError
from paper_2508_21058_b200.binding import debug_cross_plan

N_SM = 148


def plan(heads, kv_heads, d, q_len, k_len):
    q_off, k_off = [0], [0]
    for n in q_len:
        q_off.append(q_off[-1] + n)
    for n in k_len:
        k_off.append(k_off[-1] + n)
    return debug_cross_plan(heads, kv_heads, d, q_off, k_off, n_sm=N_SM)


# many segments, one or two of them with far more states than the others
SKEWED = [
    (24, 24, 128, [200] * 61, [77] * 60 + [32760]),
    (24, 8, 128, [200] * 61, [32760] + [77] * 60),
    (12, 12, 64, [700] * 40, [100] * 38 + [30000, 20000]),
    (40, 40, 128, [130] * 30, [500] * 29 + [100000]),
    (8, 8, 128, [16] * 300, [128] * 299 + [50000]),
    (6, 2, 128, [5000] * 8 + [300], [256] * 8 + [60000]),
]


@pytest.mark.parametrize("case", SKEWED)
def test_no_cta_walks_a_long_list_while_the_others_are_done(case):
    """The longest walk of a launch is at most twice the mean and a few tiles: longer lists are cut."""
    p = plan(*case)
    for launch in ("two_tile", "one_tile", "dq"):
        assert p[launch + "_walk"] <= 2 * p[launch + "_mean"] + 6, (launch, p)


def test_even_lists_are_not_cut():
    """Lists of about the same length with items for every CTA: no shares, no launch to put them together."""
    for case in [(24, 24, 128, [33016], [512]), (6, 2, 128, [33016 - 3000 * i for i in range(8)], [512 - 40 * i for i in range(8)]),
                 (16, 16, 64, [1000] * 50, [77] * 50)]:
        assert plan(*case)["part_rows"] == 0


def test_walks_of_any_lists():
    rng = random.Random(1)
    cut = 0
    for _ in range(400):
        kv = rng.choice([1, 2, 8, 24])
        heads = kv * rng.choice([1, 3])
        n = rng.choice([1, 2, 10, 60])
        q = [int(2 ** rng.uniform(0, 12)) for _ in range(n)]
        k = [int(2 ** rng.uniform(0, rng.choice([9, 16]))) for _ in range(n)]
        p = plan(heads, kv, rng.choice([64, 128]), q, k)
        cut += p["part_rows"] > 0
        for launch in ("two_tile", "one_tile", "dq"):
            assert p[launch + "_walk"] <= 2 * p[launch + "_mean"] + 16, (heads, kv, q, k, launch, p)
    assert cut > 50


@pytest.mark.parametrize("case", [
    (1, 1, 64, [5_000_000], [2**30]),                # 512 shares of 5M rows
    (1, 1, 64, [2**23, 2**23], [2**29, 2**29 + 5]),
])
def test_more_than_can_be_counted_is_refused(case):
    """Rows of partial results and work items are 32-bit numbers: a plan with more is refused before anything is allocated for it."""
    with pytest.raises(MocError) as e:
        plan(*case)
    assert e.value.code == -2
    assert plan(*case[:3], [300] * len(case[4]), case[4])["part_rows"] > 0


@pytest.mark.parametrize("case", [
    (64, 1, 64, [3_000_000] + [100] * 500, [1_000_000] + [1_100_000] * 500),
    (8, 8, 128, [20_000_000] + [128] * 200 + [256], [300_000] + [900_000] * 200 + [50_000]),
])
def test_no_warp_waits_through_a_second_of_other_items(case):
    """In items of one query tile the second tile's warps have nothing to do: their wait for the next of two is a bounded one, of two
    seconds, some 600,000 key tiles at the lowest clock."""
    p = plan(*case)
    assert p["two_tile"] > 0 and p["one_tile"] == 0
    assert p["two_tile_wait"] <= 300_000
