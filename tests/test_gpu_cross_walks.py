"""Cross attention where a CTA of the two-tile kernel walks several items: of two query tiles and of one, of no states, with odd last key
tiles; scores of large magnitude in the backward pass; and the kernel of few queries held to fp32 throughout.  Against the
64-bit plain form."""
import pytest
import torch

import layer_ref as R
import test_gpu_cross as T
from paper_2508_21058_b200.binding import debug_cross_plan

pytestmark = pytest.mark.gpu

# heads, key heads, d, queries and states of every segment, padding; items of 256 query rows are two tiles, a segment's last ones may be one
CASES = [
    (24, 8, 128, [2400, 256, 700, 40, 300, 0, 1500], [333, 520, 641, 200, 30, 50, 0], 3),
    (24, 24, 128, [2900, 3000, 2700], [600, 600, 500], 0),
    (24, 8, 128, [2400] * 3 + [100, 70], [333, 520, 400, 500, 390], 1),
    (12, 3, 128, [9000, 40, 600, 120], [300, 650, 500, 140], 0),
    (16, 16, 64, [5000, 2400, 300, 60], [400, 700, 513, 290], 5),
    (40, 40, 64, [5200, 100], [777, 390], 0),
    (24, 24, 128, [5200], [777], 0),
]


def _plan(run):
    return debug_cross_plan(run.H, run.kv, run.d, run.q_off, run.k_off, run.k_len, torch.cuda.get_device_properties(0).multi_processor_count)


@pytest.mark.parametrize("case", CASES)
def test_ctas_walk_items_of_two_tiles_and_of_one(case):
    run = T.Run(case, seed=31)
    plan = _plan(run)
    assert plan["two_tile"] > 2.5 * 148 and plan["one_tile"] == 0
    assert len(case[3]) == 1 or any(0 < n % 256 <= 128 for n in case[3])
    run.forward().backward().check()
    first = [t.clone() for t in run.outputs()]
    run.forward().backward()
    assert all(torch.equal(a, b) for a, b in zip(first, run.outputs()))


@pytest.mark.parametrize("factor", [30, 300])
@pytest.mark.parametrize("case", [(2, 2, 128, [200], [500], 0), (4, 2, 64, [130, 1, 300], [300, 129, 77], 3), (16, 4, 128, [1300, 640], [333, 512], 7),
                                  (2, 1, 128, [64], [2000], 0), (2, 1, 64, [3], [2000], 0)])
def test_scores_of_large_magnitude_there_and_back(case, factor):
    """The backward pass takes P from scores and a log-sum-exp that is rounded to fp32: off by half a step of the lse, and of the score."""
    run = T.Run(case, seed=33)
    run.k[:, :run.Lk] *= torch.linspace(0.1, factor, run.Lk, device="cuda")[None, :, None]
    run.forward().backward().check()


# heads, key heads, d, queries and states of every segment: up to eight rows that share a key head
FEW = [
    (8, 1, 64, [1, 1], [3000, 5]), (1, 1, 128, [2], [20000]), (24, 8, 128, [1] * 9, [1, 300, 129, 128, 127, 64, 250, 31, 77]),
    (2, 2, 128, [2, 4, 8], [700, 129, 40]), (5, 5, 64, [1], [4097]), (7, 1, 128, [1, 1], [33, 640]), (12, 4, 128, [2, 1], [9000, 8000]),
]


@pytest.mark.parametrize("case", FEW)
def test_few_queries_are_fp32_throughout(case):
    """Without a rounding of P to bf16 in the bound; every state's part of O and lse is far above what is left of it where the values of a
    stretch of states are large."""
    H, kv, d, q_len, k_len = case
    run = T.Run((*case, 2), seed=34)
    plan = _plan(run)
    assert plan["few"] > 0 and plan["two_tile"] + plan["one_tile"] == 0
    for a, n in zip(run.k_off, k_len):
        run.v[:, a:a + n:97] *= 16                              # some of every share's values
        run.v[:, a + n - 1] *= 16
    run.forward()
    torch.cuda.synchronize()
    assert run.op.moc_cross_get_status(run.ws) == (0, 0)
    r0 = 0
    for nq, nk, k0 in zip(q_len, k_len, run.k_off):
        # sums: 32 states a stage, two to a lane group; the groups and warps of a block; a warp's shares, eight warps of them
        shares = max(1, plan["part_rows"])
        terms = nk / 16 if plan["part_rows"] == 0 else min(nk, 4096) / 16 + shares
        for h in range(H):
            Q, K, V = (t.double() for t in (run.q[h, r0:r0 + nq], run.k[h // (H // kv), k0:k0 + nk], run.v[h // (H // kv), k0:k0 + nk]))
            s = d ** -0.5 * Q @ K.T
            # the score: the query's scaling, d products summed in fp32; the exponent's difference; exp2 to a few units
            e_s = float((d ** -0.5 * (d + 8) * R.U32 * (Q.abs() @ K.abs().T)).max())
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            e_p = 2 * e_s + 8 * R.U32 * float(s.abs().max() + 1) + (terms + 64) * R.U32
            o = p @ V
            R.check("O", run.o[h, r0:r0 + nq], o, R.U16 * (1 + R.U16) * o.abs() + e_p * (p @ V.abs()) * 1.01)
            R.check("lse", run.lse[h, r0:r0 + nq], lse, e_s + (terms + 64) * R.U32 + 16 * R.U32 * (lse.abs() + 1))
        r0 += nq


def test_one_plan_on_two_streams():
    """At once, with a workspace each."""
    runs = [T.Run(CASES[2], seed=35 + i) for i in range(2)]
    for r in runs:
        r.op = runs[0].op
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for run, s in zip(runs, streams):
            with torch.cuda.stream(s):
                run.forward().backward()
    torch.cuda.synchronize()
    for run in runs:
        run.check()
