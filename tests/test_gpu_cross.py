"""Cross attention to encoder states of another length, forward and backward, through the C ABI against the 64-bit plain form: ragged,
empty and single-token segments, shared key heads, padding that holds NaN, shares of long key lists, layouts, graphs and streams."""
import pytest
import torch

import layer_ref as R
import parity_utils as PU
from paper_2508_21058_b200 import MocCross, MocError

pytestmark = pytest.mark.gpu

# heads, key heads, d, queries and states of every segment, padding behind each segment's states
CASES = [
    (1, 1, 64, [1], [1], 0),
    (1, 1, 128, [1], [16], 0),
    (4, 4, 64, [576], [77], 0),
    (2, 2, 128, [128], [128], 0),
    (2, 1, 128, [129], [129], 0),
    (3, 1, 128, [130, 1, 0, 257], [200, 0, 33, 129], 3),
    (4, 2, 64, [127, 128, 129, 5], [15, 16, 17, 1], 20),
    (2, 1, 128, [64], [2000], 0),                       # shares of the keys, in the forward and in dQ
    (2, 2, 64, [300], [1100], 5),
    (24, 8, 128, [1] * 9, [1, 300, 129, 128, 127, 64, 250, 31, 77], 1),
    (1, 1, 128, [700], [512], 0),
    (6, 2, 128, [513, 0, 31], [40, 50, 0], 0),
    (8, 8, 64, [2000, 3], [512, 512], 0),
    (16, 4, 128, [1300, 640], [333, 512], 7),           # more items than SMs
    # few queries: up to eight rows of the query heads that share a key head, one to four in a block
    (8, 1, 64, [1, 1], [3000, 5], 0),
    (8, 1, 128, [1, 1, 300], [3000, 5, 70], 3),
    (2, 2, 128, [2, 4, 8, 9], [700, 129, 40, 200], 1),
    (4, 2, 64, [3, 0, 1], [1000, 9, 31], 2),
    (5, 5, 128, [1], [4097], 0),
    (7, 1, 128, [1, 1], [33, 640], 0),
    (1, 1, 128, [2], [20000], 0),                       # more shares than a warp puts together
    (1, 1, 64, [130, 3], [9000, 4000], 0),
    # one query tile an item: both softmax groups on it, an odd and an even number of key tiles, shares, beside two-tile items
    (3, 1, 128, [100, 128, 9], [1000, 129, 128], 2),
    (2, 2, 64, [64], [5000], 0),
    (24, 8, 128, [50] * 6, [300, 17, 500, 256, 1, 384], 1),
    (32, 32, 64, [257], [12000], 0),
    (40, 40, 128, [384, 0, 90], [8000, 4, 3000], 1),
]


class Run:
    def __init__(self, case, seed=0, layout="heads", spare=3):
        self.H, self.kv, self.d, self.q_len, self.k_len, pad = case
        gen = torch.Generator("cuda").manual_seed(seed)
        self.k_off, self.q_off = [0], [0]
        for n in self.k_len:
            self.k_off.append(self.k_off[-1] + n + pad)
        for n in self.q_len:
            self.q_off.append(self.q_off[-1] + n)
        Lq, Lk = self.q_off[-1], self.k_off[-1]
        self.Lq, self.Lk = Lq, Lk
        self.guard = PU.Guarded()

        def tensor(heads, rows):
            rows += spare                               # rows behind the last segment's: left as they are
            if layout == "heads":
                return self.guard.empty((heads, rows, self.d), torch.bfloat16)
            return self.guard.empty((rows, heads, self.d), torch.bfloat16).transpose(0, 1)

        self.q, self.do, self.o, self.dq = (tensor(self.H, Lq) for _ in range(4))
        self.k, self.v, self.dk, self.dv = (tensor(self.kv, Lk) for _ in range(4))
        for t in (self.q, self.do, self.k, self.v):
            t.normal_(generator=gen)
        self.live = torch.zeros(Lk + spare, dtype=torch.bool, device="cuda")
        for a, n in zip(self.k_off, self.k_len):
            self.live[a:a + n] = True
        for t in (self.k, self.v):
            t[:, ~self.live] = float("nan")
        for t in (self.q, self.do):
            t[:, Lq:] = float("nan")
        for t in (self.o, self.dq, self.dk, self.dv):
            t.fill_(7.0)
        self.lse = self.guard.empty((self.H, Lq), torch.float32)
        self.op = MocCross(self.H, self.kv, self.d, self.q_off, self.k_off, k_len=self.k_len)
        self.ws = self.guard.empty((self.op.workspace_bytes(True),), torch.uint8)

    def forward(self):
        self.op.moc_cross_attend(self.q, self.k, self.v, self.o, self.lse, self.ws)
        return self

    def backward(self):
        self.op.moc_cross_attend_bwd(self.q, self.k, self.v, self.o, self.lse, self.do, self.dq, self.dk, self.dv, self.ws)
        return self

    def outputs(self):
        return self.o, self.lse, self.dq, self.dk, self.dv

    def check(self, grads=True):
        torch.cuda.synchronize()
        assert self.op.moc_cross_get_status(self.ws) == (0, 0)
        self.guard.check()
        Lq, Lk = self.Lq, self.Lk
        wide = [t.double() for t in (self.q[:, :Lq], self.k[:, :Lk], self.v[:, :Lk], self.do[:, :Lq])]
        ref = R.CrossRef(*wide[:3], self.q_len, self.k_len, self.k_off, self.d ** -0.5, wide[3] if grads else None)
        R.check("O", self.o[:, :Lq], ref.o, ref.o_tol)
        R.check("lse", self.lse, ref.lse, ref.lse_tol)
        assert bool((self.o[:, Lq:] == 7.0).all())
        if grads:
            R.check("dQ", self.dq[:, :Lq], ref.dq, ref.dq_tol)
            R.check("dK", self.dk[:, :Lk], ref.dk, ref.dk_tol)      # (padding and states that nobody reads: zero, and no tolerance)
            R.check("dV", self.dv[:, :Lk], ref.dv, ref.dv_tol)
            assert bool((self.dq[:, Lq:] == 7.0).all()) and bool((self.dk[:, Lk:] == 7.0).all()) and bool((self.dv[:, Lk:] == 7.0).all())


@pytest.mark.parametrize("case", CASES)
def test_forward_against_64_bits(case):
    Run(case).forward().check(grads=False)


@pytest.mark.parametrize("case", CASES)
def test_backward_against_64_bits(case):
    run = Run(case, seed=1)
    run.forward().backward().check()
    first = [t.clone() for t in run.outputs()]
    run.forward().backward()
    assert all(torch.equal(a, b) for a, b in zip(first, run.outputs()))          # bit for bit


@pytest.mark.parametrize("case", [CASES[5], CASES[6], CASES[7]])
def test_token_major_tensors(case):
    Run(case, seed=2, layout="tokens").forward().backward().check()


def test_many_tiles_of_few_keys():
    """Every CTA walks many items and pieces, the rings run on across them."""
    Run((12, 3, 64, [5000, 1, 700], [30, 600, 130], 2), seed=3).forward().backward().check()
    Run((6, 6, 128, [6000], [140], 0), seed=4).forward().backward().check()


def test_scores_of_large_magnitude():
    """Maxima that grow from tile to tile (the rescaling of O), rows that attend to one key alone."""
    run = Run((2, 2, 128, [200], [500], 0), seed=5)
    run.k[:, :500] *= torch.linspace(0.1, 30, 500, device="cuda")[None, :, None]
    run.forward().check(grads=False)


def test_scale_is_the_callers():
    run = Run((2, 2, 64, [50], [70], 0), seed=6)
    run.op = MocCross(2, 2, 64, run.q_off, run.k_off, k_len=run.k_len, softmax_scale=0.03)
    run.forward().backward()
    torch.cuda.synchronize()
    wide = [t.double() for t in (run.q[:, :50], run.k[:, :70], run.v[:, :70], run.do[:, :50])]
    ref = R.CrossRef(*wide[:3], run.q_len, run.k_len, run.k_off, 0.03, wide[3])
    for name, got, n in (("o", run.o, 50), ("dq", run.dq, 50), ("dk", run.dk, 70), ("dv", run.dv, 70)):
        R.check(name, got[:, :n], getattr(ref, name), getattr(ref, name + "_tol"))


@pytest.mark.parametrize("q_len,k_len", [([], []), ([0, 0], [5, 0]), ([4, 2], [0, 0]), ([0], [0])])
def test_nothing_to_attend(q_len, k_len):
    run = Run((2, 1, 64, q_len, k_len, 1), seed=7)
    run.forward().backward()
    torch.cuda.synchronize()
    run.guard.check()
    assert bool((run.o[:, :run.Lq] == 0).all()) and bool((run.lse == -float("inf")).all()) and bool((run.dq[:, :run.Lq] == 0).all())
    assert bool((run.dk[:, :run.Lk] == 0).all()) and bool((run.dv[:, :run.Lk] == 0).all()) and bool((run.dk[:, run.Lk:] == 7.0).all())


@pytest.mark.parametrize("q_len,k_len", [([], []), ([0, 0], [5, 0]), ([4, 2], [0, 0]), ([300, 2], [0, 40])])
def test_nothing_to_attend_in_a_graph(q_len, k_len):
    run = Run((2, 1, 64, q_len, k_len, 1), seed=17)
    run.forward().backward()
    torch.cuda.synchronize()
    want = [t.clone() for t in run.outputs()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.forward().backward()
    for t in run.outputs():
        t.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    for a, b, n in zip(run.outputs(), want, (run.Lq, run.Lq, run.Lq, run.Lk, run.Lk)):
        assert torch.equal(a[:, :n], b[:, :n])


def test_a_bad_value_stays_with_those_who_see_it():
    """An infinite value in one segment's states, NaN in one query and its gradient: other segments' results are as without them."""
    clean = Run((2, 1, 128, [100, 60, 40], [90, 50, 300], 0), seed=8).forward().backward()
    run = Run((2, 1, 128, [100, 60, 40], [90, 50, 300], 0), seed=8)
    run.k[:, 95], run.v[:, 100], run.q[:, 130], run.do[:, 131] = (float(x) for x in ("inf", "inf", "nan", "nan"))
    run.forward().backward()
    torch.cuda.synchronize()
    q, k = [*range(100), *range(160, 200)], [*range(90), *range(140, 440)]
    for a, b, rows in ((clean.o, run.o, q), (clean.dq, run.dq, q), (clean.dk, run.dk, k), (clean.dv, run.dv, k), (clean.lse, run.lse, q)):
        assert torch.equal(a[:, rows], b[:, rows])


def test_graph_replay_with_other_inputs_and_another_stream():
    run = Run(CASES[5], seed=9)
    run.forward().backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run.forward().backward()
    for t in (run.q, run.do):
        t[:, :run.Lq] = torch.randn_like(t[:, :run.Lq])
    graph.replay()
    run.check()
    got = [t.clone() for t in run.outputs()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run.forward().backward()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, run.outputs()))


def test_two_calls_at_once_with_a_workspace_each():
    runs = [Run((4, 2, 128, [900, 30], [700, 100], 3), seed=10 + i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(5):
        for run, s in zip(runs, streams):
            with torch.cuda.stream(s):
                run.forward().backward()
    torch.cuda.synchronize()
    for run in runs:
        run.check()


def test_rows_far_apart():
    """Offsets beyond 32 bits: the heads of Q and O more than 2^31 values apart."""
    run = Run((2, 2, 64, [150], [40], 0), seed=12, spare=0)
    gap = 2**31 + 64

    def apart(t):
        n = t.shape[1] * 64
        b = torch.empty(gap + n, dtype=torch.bfloat16, device="cuda").as_strided((2, t.shape[1], 64), (gap, 64, 1))
        b.copy_(t)
        return b

    run.q, run.o, run.do, run.dq = (apart(t) for t in (run.q, run.o, run.do, run.dq))
    run.forward().backward().check()


def test_refusals_before_a_launch():
    run = Run((2, 1, 64, [20], [30], 0), seed=13)
    a = [run.q, run.k, run.v, run.o, run.lse, run.ws]
    for i, bad, code in [(0, run.q.float(), -2), (0, run.q[:, :-4], -2), (0, run.q[:1], -2), (1, run.q, -2), (1, run.k[:, :29], -2),
                         (0, run.q[:1].expand(2, -1, -1), -2), (4, run.lse.double(), -2), (4, run.lse[:, :-1], -2), (5, run.ws[:run.op.workspace_bytes() - 256], -5),
                         (5, None, -5), (0, run.q.cpu(), -6), (3, run.o[:, :, 1:], -2),
                         (0, torch.empty(2, 20, 72, dtype=torch.bfloat16, device="cuda")[:, :, 4:68], -4),
                         (0, torch.empty(2, 20, 68, dtype=torch.bfloat16, device="cuda")[:, :, :64], -4)]:
        args = list(a)
        args[i] = bad
        with pytest.raises(MocError) as e:
            run.op.moc_cross_attend(*args)
        assert e.value.code == code, (i, code)
    with pytest.raises(MocError) as e:
        run.op.moc_cross_attend(*a[:5], torch.empty(run.op.workspace_bytes() + 256, dtype=torch.uint8, device="cuda")[16:])
    assert e.value.code == -4
