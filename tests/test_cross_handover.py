"""The hand-overs between the warps of the cross attention's kernels, as models of their mbarriers that are run under many schedules
on the CPU: whoever reads a buffer or a tensor-memory tile must find the tile it means, and every warp must come to its end.  Waits are
by parity, as in the kernels: one that is looked at a phase too late waits for ever."""
import random

import pytest


class Barrier:
    def __init__(self, need):
        self.need, self.got, self.phase = need, 0, 0

    def arrive(self):
        self.got += 1
        if self.got == self.need:
            self.got, self.phase = 0, self.phase + 1

    def done(self, parity):
        return (self.phase & 1) != (parity & 1)


class WrongTile(Exception):
    pass


class Model:
    """Warps are generators that yield a condition to wait for; MMAs and commits run in the order of their issuer, copies in any order."""

    def __init__(self, seed, slow):
        self.rng, self.slow = random.Random(seed), slow
        self.mem, self.pipes, self.copies, self.warps = {}, {}, [], {}

    def want(self, where, what):
        if self.mem.get(where) != what:
            raise WrongTile(f"{where} holds {self.mem.get(where)}, not {what}")

    def mma(self, who, reads, write=None, commits=()):
        def go():
            for r in reads:
                self.want(*r)
            if write:
                self.mem[write[0]] = write[1]
        self.pipes.setdefault(who, []).append(go)
        for b in commits:
            self.pipes[who].append(b.arrive)

    def copy(self, where, what, bar):
        self.mem[where] = "in flight"

        def land():
            self.mem[where] = what
            bar.arrive()
        self.copies.append(land)

    def run(self):
        state = {name: [g, next(g, "end")] for name, g in self.warps.items()}
        for _ in range(200000):
            ready = [n for n, (g, c) in state.items() if c != "end" and (c is None or c())]
            moves = ready + [("pipe", w) for w, q in self.pipes.items() if q] + [("copy", i) for i in range(len(self.copies))]
            if not moves:
                return all(c == "end" for _, c in state.values())
            fast = [x for x in moves if x != self.slow and (not isinstance(x, tuple) or x[0] != self.slow)]
            m = self.rng.choice(fast if fast and self.rng.random() < 0.98 else moves)
            if isinstance(m, tuple) and m[0] == "pipe":
                self.pipes[m[1]].pop(0)()
            elif isinstance(m, tuple):
                self.copies.pop(m[1])()
            else:
                state[m][1] = next(state[m][0], "end")
        return False


def dq(items, seed, slow, look_before_lse=True):
    """cross_dq_tc_kernel: items of so many key tiles."""
    m = Model(seed, slow)
    KS, VS, NW = 3, 2, 2                                   # stages; warps that form delta (four in the kernel)
    b = {"X_FULL": Barrier(3 + NW), "X_EMPTY": Barrier(3), "T1_FULL": Barrier(1), "T1_READ": Barrier(1),
         "ACC_FULL": Barrier(1), "ACC_FREE": Barrier(1)}
    for i in range(3):
        for n in ("K_FULL", "K_EMPTY", "V_FULL", "V_EMPTY", "T2_FULL", "DS_DONE"):
            b[n, i] = Barrier(1)

    def states():
        g = 0
        for n, tiles in enumerate(items):
            for j in range(tiles):
                yield lambda: b["K_EMPTY", g % KS].done((g // KS & 1) ^ 1)
                m.copy(("K", g % KS), g, b["K_FULL", g % KS])
                yield lambda: b["V_EMPTY", g % VS].done((g // VS & 1) ^ 1)
                m.copy(("V", g % VS), g, b["V_FULL", g % VS])
                g += 1

    def rows():
        for n in range(len(items)):
            if n:
                yield lambda: b["X_EMPTY"].done(n - 1)
            m.copy("Q", n, b["X_FULL"])
            m.copy("dO", n, b["X_FULL"])
            m.mem["lse", n & 1] = n
            b["X_FULL"].arrive()
            yield None

    def delta(w):
        for n in range(len(items)):
            if n and look_before_lse:
                yield lambda: b["X_EMPTY"].done(n - 1)
            m.mem["delta", n & 1, w] = n
            b["X_FULL"].arrive()
            yield None

    def lanes():
        g = 0
        for n in range(len(items) + 1):
            if n < len(items):
                yield lambda: b["X_FULL"].done(n)
                yield None
                m.want(("lse", n & 1), n)
                for w in range(NW):
                    m.want(("delta", n & 1, w), n)
                b["X_EMPTY"].arrive()
            for j in range(items[n] if n < len(items) else 1):
                if n < len(items):
                    yield lambda: b["T1_FULL"].done(g)
                    m.want("T1", g)
                    b["T1_READ"].arrive()
                    yield lambda: b["T2_FULL", g & 1].done(g >> 1)
                    m.want(("T2", g & 1), g)
                    m.mem["T2", g & 1] = ("dS", g)
                    b["DS_DONE", g & 1].arrive()
                    yield None
                    g += 1
                if j == 0 and n:
                    yield lambda: b["ACC_FULL"].done(n - 1)
                    m.want("ACC", (n - 1, items[n - 1] - 1))
                    b["ACC_FREE"].arrive()
                    yield None

    def issuer1():
        g = 0
        for n, tiles in enumerate(items):
            yield lambda: b["X_FULL"].done(n)
            for j in range(tiles):
                yield lambda: b["K_FULL", g % KS].done(g // KS)
                if g:
                    yield lambda: b["T1_READ"].done(g - 1)
                m.mma("t1", [("Q", n), (("K", g % KS), g)], ("T1", g), [b["T1_FULL"]] + ([b["X_EMPTY"]] if j + 1 == tiles else []))
                g += 1

    def issuer2():
        g = 0

        def t2(t, n, last):
            yield lambda: b["V_FULL", t % VS].done(t // VS)
            m.mma("t2", [("dO", n), (("V", t % VS), t)], (("T2", t & 1), t), [b["T2_FULL", t & 1], b["V_EMPTY", t % VS]] + ([b["X_EMPTY"]] if last else []))

        for n, tiles in enumerate(items):
            yield lambda: b["X_FULL"].done(n)
            yield from t2(g, n, tiles == 1)
            if tiles > 1:
                yield from t2(g + 1, n, tiles == 2)
            for j in range(tiles):
                yield lambda: b["DS_DONE", g & 1].done(g >> 1)
                if j == 0 and n:
                    yield lambda: b["ACC_FREE"].done(n - 1)
                m.mma("t2", [(("T2", g & 1), ("dS", g)), (("K", g % KS), g)] + ([("ACC", (n, j - 1))] if j else []), ("ACC", (n, j)), [b["K_EMPTY", g % KS]])
                g += 1
                if j + 2 < tiles:
                    yield from t2(g + 1, n, j + 3 == tiles)
            m.pipes["t2"].append(b["ACC_FULL"].arrive)

    m.warps = {"states": states(), "rows": rows(), "lanes": lanes(), "t1": issuer1(), "t2": issuer2()}
    m.warps.update({f"delta{w}": delta(w) for w in range(NW)})
    return m.run()


def solo(items, seed, slow, look_before_ml=True):
    """cross_solo_tc_kernel: items of so many key tiles, the two groups on every other one."""
    m = Model(seed, slow)
    b = {"ML": Barrier(1)}
    for i in range(3):
        b["Q_FULL", i], b["Q_EMPTY", i] = Barrier(1), Barrier(2)
        for n in ("K_FULL", "K_EMPTY", "V_FULL", "V_EMPTY", "S_FULL", "P_FULL", "O_FULL", "O_FREE"):
            b[n, i] = Barrier(1)

    def q_and_k():
        used = [0, 0]
        for n, tiles in enumerate(items):
            yield lambda: b["Q_EMPTY", n % 3].done((n // 3 & 1) ^ 1)
            m.copy(("Q", n % 3), n, b["Q_FULL", n % 3])
            for j in range(tiles):
                yield lambda: b["K_EMPTY", j & 1].done((used[j & 1] & 1) ^ 1)
                used[j & 1] += 1
                m.copy(("K", j & 1), (n, j), b["K_FULL", j & 1])

    def v():
        used = [0, 0]
        for n, tiles in enumerate(items):
            for j in range(tiles):
                yield lambda: b["V_EMPTY", j & 1].done((used[j & 1] & 1) ^ 1)
                used[j & 1] += 1
                m.copy(("V", j & 1), (n, j), b["V_FULL", j & 1])

    def issuer(g):
        own = t = 0
        for n, tiles in enumerate(items):
            yield lambda: b["Q_FULL", n % 3].done(n // 3)
            mine = list(range(g, tiles, 2))
            if not mine:
                b["Q_EMPTY", n % 3].arrive()
                yield None
                continue
            who = f"mma{g}"

            def qk(j, after=()):
                m.mma(who, [(("Q", n % 3), n), (("K", g), (n, j))], (("S", g), (n, j)),
                      [b["S_FULL", g], *after, b["K_EMPTY", g]] + ([b["Q_EMPTY", n % 3]] if j == mine[-1] else []))

            yield lambda: b["K_FULL", g].done(t)
            qk(mine[0])
            for i, j in enumerate(mine):
                yield lambda: b["V_FULL", g].done(t)
                if i == 0 and own:
                    yield lambda: b["O_FREE", g].done(own - 1)
                more = i + 1 < len(mine)
                if more:
                    yield lambda: b["K_FULL", g].done(t + 1)
                yield lambda: b["P_FULL", g].done(t)
                m.mma(who, [(("S", g), ("P", n, j)), (("V", g), (n, j))] + ([(("O", g), (n, mine[i - 1]))] if i else []), (("O", g), (n, j)))
                if more:
                    qk(mine[i + 1], [b["V_EMPTY", g]])
                else:
                    m.pipes[who] += [b["V_EMPTY", g].arrive, b["O_FULL", g].arrive]
                t += 1
            own += 1

    def softmax(g):
        t = ml = own = 0
        for n, tiles in enumerate(items):
            for j in range(g, tiles, 2):
                yield lambda: b["S_FULL", g].done(t)
                m.want(("S", g), (n, j))
                m.mem["S", g] = ("P", n, j)
                b["P_FULL", g].arrive()
                yield None
                t += 1
            two = tiles > 1
            if g == 1:
                if two:
                    if ml and look_before_ml:
                        yield lambda: b["O_FREE", 1].done(ml - 1)
                    m.mem["ml"] = n
                    b["ML"].arrive()
                    yield None
                    ml += 1
                continue
            if two:
                yield lambda: b["ML"].done(ml)
                yield None
                m.want("ml", n)
            yield lambda: b["O_FULL", 0].done(own)
            if two:
                yield lambda: b["O_FULL", 1].done(ml)
                m.want(("O", 1), (n, (tiles - 2) // 2 * 2 + 1))
            m.want(("O", 0), (n, (tiles - 1) // 2 * 2))
            own += 1
            ml += two
            b["O_FREE", 0].arrive()
            if two:
                b["O_FREE", 1].arrive()
            yield None

    m.warps = {"qk": q_and_k(), "v": v(), "mma0": issuer(0), "mma1": issuer(1), "soft0": softmax(0), "soft1": softmax(1)}
    return m.run()


def dkv(pieces, seed, slow, look_before_lse=True):
    """cross_dkv_tc_kernel: pieces of so many query tiles, the rings run on across them."""
    m = Model(seed, slow)
    Y1, Y2 = 3, 2
    b = {"X_FULL": Barrier(1), "P_HALF": Barrier(1), "P_DONE": Barrier(1), "ACC_FULL": Barrier(2)}
    for i in range(3):
        for n in ("Y1_FULL", "Y1_EMPTY", "Y2_FULL", "T1_FULL", "T2_FULL", "DS_DONE", "T1_ISSUED"):
            b[n, i] = Barrier(1)
        b["Y2_EMPTY", i] = Barrier(2)
    total = sum(pieces)

    def keys():
        for n in range(len(pieces)):
            if n:
                yield lambda: b["ACC_FULL"].done(n - 1)
            m.copy("X", n, b["X_FULL"])
            yield None

    def rows(ring, stages):
        for j in range(total):
            yield lambda: b[ring + "_EMPTY", j % stages].done((j // stages & 1) ^ 1)
            if ring == "Y1":
                if j >= 2 and look_before_lse:
                    yield lambda: b["DS_DONE", j & 1].done((j - 2) >> 1)
                m.mem["ld", j & 1] = j
            m.copy((ring, j % stages), j, b[ring + "_FULL", j % stages])

    def lanes():
        j = 0
        for n, tiles in enumerate(pieces):
            for _ in range(tiles):
                yield lambda: b["T1_FULL", j & 1].done(j >> 1)
                yield lambda: b["Y1_FULL", j % Y1].done(j // Y1)
                m.want("T1", j)
                m.want(("ld", j & 1), j)
                m.mem["T1 half"] = j
                b["P_HALF"].arrive()
                yield None
                m.want("T1", j)
                m.mem["T1"] = ("P", j)
                b["P_DONE"].arrive()
                yield lambda: b["T2_FULL", j & 1].done(j >> 1)
                m.want("T2", j)
                m.want(("ld", j & 1), j)
                m.mem["T2"] = ("dS", j)
                b["DS_DONE", j & 1].arrive()
                yield None
                j += 1
            yield lambda: b["ACC_FULL"].done(n)
            yield None
            m.want("ACC1", (n, j - 1))
            m.want("ACC2", (n, j - 1))

    def side1():
        j = turn = 0
        for n, tiles in enumerate(pieces):
            end = j + tiles
            yield lambda: b["X_FULL"].done(n)
            yield lambda: b["Y1_FULL", j % Y1].done(j // Y1)
            m.mma("s1", [("X", n), (("Y1", j % Y1), j)], ("T1", j), [b["T1_FULL", j & 1]])
            first = j
            while j < end:
                more = j + 1 < end
                yield lambda: b["Y2_FULL", j % Y2].done(j // Y2)
                yield lambda: b["P_HALF"].done(j)
                m.mma("s1", [("T1 half", j), (("Y2", j % Y2), j)], ("ACC2", "begun" if j == first else m))
                if more:
                    yield lambda: b["Y1_FULL", (j + 1) % Y1].done((j + 1) // Y1)
                yield lambda: b["P_DONE"].done(j)
                m.mma("s1", [("T1", ("P", j)), (("Y2", j % Y2), j)], ("ACC2", (n, j)))
                if more:
                    m.mma("s1", [("X", n), (("Y1", (j + 1) % Y1), j + 1)], ("T1", j + 1), [b["T1_FULL", (j + 1) & 1]])
                m.pipes["s1"].append(b["Y2_EMPTY", j % Y2].arrive)
                if more:
                    b["T1_ISSUED", turn & 1].arrive()
                    turn += 1
                yield None
                j += 1
            m.pipes["s1"].append(b["ACC_FULL"].arrive)

    def side2():
        j = turn = 0
        for n, tiles in enumerate(pieces):
            end, first = j + tiles, j
            yield lambda: b["X_FULL"].done(n)

            def t2(t):
                m.mma("s2", [("X", n), (("Y2", t % Y2), t)], ("T2", t), [b["T2_FULL", t & 1], b["Y2_EMPTY", t % Y2]])

            yield lambda: b["Y2_FULL", j % Y2].done(j // Y2)
            t2(j)
            while j < end:
                more = j + 1 < end
                if more:
                    yield lambda: b["T1_ISSUED", turn & 1].done(turn >> 1)
                    turn += 1
                yield lambda: b["Y1_FULL", j % Y1].done(j // Y1)
                yield lambda: b["DS_DONE", j & 1].done(j >> 1)
                m.mma("s2", [("T2", ("dS", j)), (("Y1", j % Y1), j)] + ([("ACC1", (n, j - 1))] if j > first else []), ("ACC1", (n, j)), [b["Y1_EMPTY", j % Y1]])
                if more:
                    yield lambda: b["Y2_FULL", (j + 1) % Y2].done((j + 1) // Y2)
                    t2(j + 1)
                j += 1
            m.pipes["s2"].append(b["ACC_FULL"].arrive)

    m.warps = {"keys": keys(), "y1": rows("Y1", Y1), "y2": rows("Y2", Y2), "lanes": lanes(), "s1": side1(), "s2": side2()}
    return m.run()


SLOW = {dq: ["lanes", "t1", "t2", "states", "rows", "delta0", "delta1", "copy", "pipe", None],
        solo: ["qk", "v", "mma0", "mma1", "soft0", "soft1", "copy", "pipe", None],
        dkv: ["lanes", "s1", "s2", "keys", "y1", "y2", "copy", "pipe", None]}
SHAPES = [[1] * 9, [4] * 4, [1, 2, 3, 5, 1, 1, 4], [2] * 7, [7, 1, 1, 1, 3]]


@pytest.mark.parametrize("kernel", [dq, solo, dkv])
def test_every_schedule_reads_what_it_means_and_ends(kernel):
    for shape in SHAPES:
        for slow in SLOW[kernel]:
            for seed in range(4):
                assert kernel(shape, seed, slow), (shape, slow, seed)


@pytest.mark.parametrize("broken", [lambda seed, slow: dq([1] * 9, seed, slow, look_before_lse=False),
                                    lambda seed, slow: solo([2] * 7, seed, slow, look_before_ml=False),
                                    lambda seed, slow: dkv([5, 4], seed, slow, look_before_lse=False)])
def test_the_models_find_a_missing_wait(broken):
    """Without the look before lse and delta are written; before the second group's results are."""
    bad = 0
    for slow in ["lanes", "soft0", "soft1", "mma0", "y1", None]:
        for seed in range(60):
            try:
                bad += not broken(seed, slow)
            except WrongTile:
                bad += 1
    assert bad
