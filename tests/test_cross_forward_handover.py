"""The hand-overs of the cross attention's two forward kernels with P in two halves, as models of their mbarriers run under many schedules
on the CPU (see test_cross_handover.py): the two-tile kernel with items of one and of two query tiles and of no states, its turns of the
exponentials and its ring of query tiles; and the one-tile kernel."""
import pytest
from test_cross_handover import Barrier, Model, WrongTile


class Forward(Model):
    """S of a group lies in tensor memory over both halves of P: products of Q and K write all three."""

    def qk(self, who, g, reads, tile, commits):
        def go():
            for r in reads:
                self.want(*r)
            for cell in ("S", "P0", "P1"):
                self.mem[cell, g] = tile
        self.pipes.setdefault(who, []).append(go)
        self.pipes[who] += [b.arrive for b in commits]

    def pv(self, who, g, half, v, tile, before, commits=()):
        """O += P V of a half; `before`: what O holds then, None for whatever it holds (it is overwritten)."""
        def go():
            self.want((f"P{half}", g), ("P", tile))
            self.want(*v)
            if before is not None:
                self.want(("O", g), before)
            self.mem["O", g] = (tile, half)
        self.pipes.setdefault(who, []).append(go)
        self.pipes[who] += [b.arrive for b in commits]

    def softmax(self, g, tile, half_done, done, turn=None):
        """Between two halves of P; the turn is handed over before the last of it."""
        self.want(("S", g), tile)
        self.mem["S", g] = "read"
        yield None
        self.mem["P0", g] = ("P", tile)
        half_done.arrive()
        yield None
        if turn:
            turn.arrive()
        yield None
        self.mem["P1", g] = ("P", tile)
        done.arrive()
        yield None


def two_tile(items, seed, slow, wait_for_buffer=True, release_for_absent=True, turns=True):
    """cross_fwd_tc_kernel; items: (query tiles, key tiles)."""
    m = Forward(seed, slow)
    b = {}
    for g in range(2):
        for i in range(3):
            b["Q_FULL", g, i] = Barrier(1)
        for n in ("S_FULL", "P_HALF", "P_FULL", "O_FULL", "O_FREE", "TURN", "K_FULL", "V_FULL"):
            b[n, g] = Barrier(1)
        b["K_EMPTY", g], b["V_EMPTY", g] = Barrier(2), Barrier(2)
    for i in range(3):
        b["Q_EMPTY", i] = Barrier(1)
    taken = []                                               # whose exponentials had the turn, in order

    def states():
        kv = 0
        for n, (_, tiles) in enumerate(items):
            for j in range(tiles):
                st, ph = kv & 1, kv >> 1 & 1
                yield lambda: b["K_EMPTY", st].done(ph ^ 1)
                m.copy(("K", st), (n, j), b["K_FULL", st])
                yield lambda: b["V_EMPTY", st].done(ph ^ 1)
                m.copy(("V", st), (n, j), b["V_FULL", st])
                kv += 1

    def queries():
        q = 0
        for n, (rows, tiles) in enumerate(items):
            for g in range(rows if tiles else 0):
                if wait_for_buffer:
                    yield lambda: b["Q_EMPTY", q % 3].done((q // 3 & 1) ^ 1)
                yield None
                m.copy(("Q", q % 3), (n, g), b["Q_FULL", g, q % 3])
                q += 1

    def softmax(g):
        s_odd = turn_odd = mine_odd = 0
        turned = False
        for n, (rows, tiles) in enumerate(items):
            two = rows == 2
            if (g == 1 and not two) or tiles == 0:
                continue
            for j in range(tiles):
                yield lambda: b["S_FULL", g].done(s_odd)
                if turns and two and not (g == 0 and not turned):
                    yield lambda: b["TURN", g ^ 1].done(turn_odd ^ (0 if g else 1))
                if two:
                    taken.append((g, n, j))
                yield from m.softmax(g, (n, j), b["P_HALF", g], b["P_FULL", g], b["TURN", g] if two else None)
                s_odd ^= 1
                if two:
                    turn_odd, turned = turn_odd ^ 1, True
            yield lambda: b["O_FULL", g].done(mine_odd)
            mine_odd ^= 1
            m.want(("O", g), ((n, tiles - 1), 1))
            b["O_FREE", g].arrive()
            yield None

    def issuer(g):
        who, mine, kv, p, seq, phase = f"mma{g}", 0, 0, 0, 0, [0, 0, 0]
        for n, (rows, tiles) in enumerate(items):
            if tiles == 0:
                continue
            qb = (seq + g) % 3
            seq += rows
            if g == 1 and rows == 1:
                for j in range(tiles):
                    yield lambda: b["K_FULL", kv & 1].done(kv >> 1)
                    yield lambda: b["V_FULL", kv & 1].done(kv >> 1)
                    if release_for_absent:
                        b["K_EMPTY", kv & 1].arrive()
                        b["V_EMPTY", kv & 1].arrive()
                    yield None
                    kv += 1
                continue

            def qk(j, st, after=()):
                m.qk(who, g, [(("Q", qb), (n, g)), (("K", st), (n, j))], (n, j),
                     [b["S_FULL", g], *after, b["K_EMPTY", st]] + ([b["Q_EMPTY", qb]] if j + 1 == tiles else []))

            yield lambda: b["Q_FULL", g, qb].done(phase[qb])
            phase[qb] ^= 1
            yield lambda: b["K_FULL", kv & 1].done(kv >> 1)
            qk(0, kv & 1)
            for j in range(tiles):
                st, more = kv & 1, j + 1 < tiles
                yield lambda: b["V_FULL", st].done(kv >> 1)
                if more:
                    yield lambda: b["K_FULL", st ^ 1].done((kv + 1) >> 1)
                yield lambda: b["P_HALF", g].done(p)
                if j == 0 and mine:                          # (P_HALF follows the reading of O, in the same threads)
                    yield lambda: b["O_FREE", g].done(mine - 1)
                m.pv(who, g, 0, (("V", st), (n, j)), (n, j), ((n, j - 1), 1) if j else None)
                yield lambda: b["P_FULL", g].done(p)
                m.pv(who, g, 1, (("V", st), (n, j)), (n, j), ((n, j), 0))
                if more:
                    qk(j + 1, st ^ 1, [b["V_EMPTY", st]])
                else:
                    m.pipes[who] += [b["V_EMPTY", st].arrive, b["O_FULL", g].arrive]
                kv += 1
                p += 1
            mine += 1

    m.warps = {"states": states(), "queries": queries(), "soft0": softmax(0), "soft1": softmax(1), "mma0": issuer(0), "mma1": issuer(1)}
    ended = m.run()
    # the groups take turns: the first, then the second, for every key tile of an item of two query tiles
    want = [(g, n, j) for n, (rows, tiles) in enumerate(items) if rows == 2 for j in range(tiles) for g in range(2)]
    if ended and taken != want:
        raise WrongTile(f"turns {taken}")
    return ended


def one_tile(items, seed, slow, look_before_o=True):
    """cross_solo_tc_kernel; items: key tiles, the two groups on every other one."""
    m = Forward(seed, slow)
    b = {"ML": Barrier(1)}
    for i in range(3):
        b["Q_FULL", i], b["Q_EMPTY", i] = Barrier(1), Barrier(2)
    for g in range(2):
        for n in ("K_FULL", "K_EMPTY", "V_FULL", "V_EMPTY", "S_FULL", "P_HALF", "P_FULL", "O_FULL", "O_FREE"):
            b[n, g] = Barrier(1)

    def states(what, with_queries):
        used = [0, 0]
        for n, tiles in enumerate(items):
            if with_queries:
                yield lambda: b["Q_EMPTY", n % 3].done((n // 3 & 1) ^ 1)
                m.copy(("Q", n % 3), n, b["Q_FULL", n % 3])
            for j in range(tiles):
                g = j & 1
                yield lambda: b[what + "_EMPTY", g].done((used[g] & 1) ^ 1)
                used[g] += 1
                m.copy((what, g), (n, j), b[what + "_FULL", g])

    def issuer(g):
        who, own, t = f"mma{g}", 0, 0
        for n, tiles in enumerate(items):
            yield lambda: b["Q_FULL", n % 3].done(n // 3)
            mine = list(range(g, tiles, 2))
            if not mine:
                b["Q_EMPTY", n % 3].arrive()
                yield None
                continue

            def qk(j, after=()):
                m.qk(who, g, [(("Q", n % 3), n), (("K", g), (n, j))], (n, j),
                     [b["S_FULL", g], *after, b["K_EMPTY", g]] + ([b["Q_EMPTY", n % 3]] if j == mine[-1] else []))

            yield lambda: b["K_FULL", g].done(t)
            qk(mine[0])
            for i, j in enumerate(mine):
                more = i + 1 < len(mine)
                yield lambda: b["V_FULL", g].done(t)
                yield lambda: b["P_HALF", g].done(t)
                if i == 0 and own and look_before_o:
                    yield lambda: b["O_FREE", g].done(own - 1)
                m.pv(who, g, 0, (("V", g), (n, j)), (n, j), ((n, mine[i - 1]), 1) if i else None)
                if more:
                    yield lambda: b["K_FULL", g].done(t + 1)
                yield lambda: b["P_FULL", g].done(t)
                m.pv(who, g, 1, (("V", g), (n, j)), (n, j), ((n, j), 0))
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
                yield from m.softmax(g, (n, j), b["P_HALF", g], b["P_FULL", g])
                t += 1
            two = tiles > 1
            if g == 1:
                if two:
                    if ml:
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
                m.want(("O", 1), ((n, (tiles - 2) // 2 * 2 + 1), 1))
            m.want(("O", 0), ((n, (tiles - 1) // 2 * 2), 1))
            own += 1
            ml += two
            b["O_FREE", 0].arrive()
            if two:
                b["O_FREE", 1].arrive()
            yield None

    m.warps = {"qk": states("K", True), "v": states("V", False), "mma0": issuer(0), "mma1": issuer(1), "soft0": softmax(0), "soft1": softmax(1)}
    return m.run()


SLOW = {two_tile: ["states", "queries", "soft0", "soft1", "mma0", "mma1", "copy", "pipe", None],
        one_tile: ["qk", "v", "soft0", "soft1", "mma0", "mma1", "copy", "pipe", None]}
SHAPES = {two_tile: [[(2, 4)] * 4, [(2, 1)] * 7, [(1, 3)] * 4, [(2, 5), (1, 2), (2, 1), (1, 1), (2, 3), (1, 4), (2, 2)],
                     [(1, 1), (2, 1), (2, 0), (1, 0), (1, 2), (2, 2), (1, 1), (1, 1), (2, 1)], [(1, 7), (2, 2)], [(2, 3), (1, 0), (2, 2), (2, 0)]],
          one_tile: [[1] * 9, [4] * 4, [1, 2, 3, 5, 1, 1, 4], [2] * 7, [7, 1, 1, 1, 3]]}


@pytest.mark.parametrize("kernel", [two_tile, one_tile])
def test_every_schedule_reads_what_it_means_and_ends(kernel):
    for shape in SHAPES[kernel]:
        for slow in SLOW[kernel]:
            for seed in range(4):
                assert kernel(shape, seed, slow), (shape, slow, seed)


@pytest.mark.parametrize("broken", [
    lambda seed, slow: two_tile([(2, 1), (1, 1)] * 4, seed, slow, wait_for_buffer=False),
    lambda seed, slow: two_tile([(2, 3), (1, 3), (2, 2)], seed, slow, release_for_absent=False),
    lambda seed, slow: two_tile([(2, 4)] * 2, seed, slow, turns=False),
    lambda seed, slow: one_tile([2] * 7, seed, slow, look_before_o=False),
], ids=["a query buffer in use", "stages of an absent tile kept", "no turns", "O not looked for, one tile"])
def test_the_models_find_a_missing_wait(broken):
    bad = 0
    for slow in ["soft0", "soft1", "mma0", "mma1", None]:
        for seed in range(40):
            try:
                bad += not broken(seed, slow)
            except WrongTile:
                bad += 1
    assert bad
