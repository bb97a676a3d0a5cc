"""The roles of the packed forward on the tensor cores (``csrc/lasad_packed_tc.cu``), simulated on the CPU barrier by barrier.

A CTA's loads, products (a warp for each of two row groups), softmax warps (four a group) and the thread that finds units
wait for one another through barriers of which only the parity of a phase can be seen.  Here every wait, arrival, copy and
product is a step, and steps come in a random order (copies land in any order, a warp's products in theirs).  A run
fails where all wait, where a wait could mistake a phase for one two further on, or where something
is read or overwritten at the wrong time.  Ring sizes, arrival counts and the rule of how far a product warp may look ahead are
read from the kernel's source.
"""
import collections
import os
import random
import re

import pytest

from paper_2507_01652_b200 import build

with open(os.path.join(build.CSRC, "lasad_packed_tc.cu")) as _f:
    SOURCE = _f.read()


def constants():
    c = {}
    for line in re.findall(r"^constexpr int ([^;]*);", SOURCE, re.M):
        for name, value in re.findall(r"(\w+) = ([^,]+)", line):
            try:
                c[name] = eval(value, {}, c)      # (sums and products of the ones before)
            except NameError:
                pass
    return c


C = constants()
COUNT = {name: eval(n, {}, C) for name, n in re.findall(r"mbar_init\(&sm\.(\w+)[^,]*, (\w+)\)", SOURCE)}
AHEAD = eval(re.search(r"owed && \(crossed \|\| n - j > ([^)]*)\)", SOURCE).group(1).replace("/", "//"), {}, C)
STAGES, ROWS, COLS, UNIT = C["kStages"], C["kRows"], C["kCols"], C["kUnit"]


def test_the_source_is_what_is_simulated():
    assert C["kGroups"] == 2 and C["kSoftmaxWarps"] == 8 and UNIT == 2 * ROWS
    assert COUNT == dict(u_full=1, u_free=11, q_full=1, q_free=2, full=1, free=2, s_full=1, p_ready=4, o_done=1, drain=1, answered=1)
    assert "while (ok && live && made - J < 2)" in SOURCE


class Bar:
    def __init__(self, n):
        self.n, self.here, self.done = n, 0, 0

    def arrive(self):
        self.here += 1
        assert self.here <= self.n
        if self.here == self.n:
            self.here, self.done = 0, self.done + 1


class Stuck(Exception):
    pass


def simulate(units, seed, careful=True, o_done_places=2):
    """units: (key tiles of group 0, of group 1).  careful: a product warp does not wait for what comes only after the product
    that it owes.  o_done_places: barriers of a group's products, in turn."""
    rnd = random.Random(seed)
    bars = {}
    for name in ("u_full", "u_free", "q_full", "q_free"):
        bars.update({(name, s): Bar(COUNT[name]) for s in range(2)})
    for name in ("full", "free"):
        bars.update({(name, s): Bar(COUNT[name]) for s in range(STAGES)})
    for name in ("s_full", "p_ready", "o_done"):
        bars.update({(name, g, s): Bar(COUNT[name]) for g in range(2) for s in range(2)})
    ring = [None, None]                           # units
    kv, queries = [None] * STAGES, [None] * 2     # what tile, and what unit's queries, a place holds
    landing, pipe = [], [collections.deque(), collections.deque()]
    read_s, wrote_p, read_o = (collections.Counter() for _ in range(3))          # warps that have, by (group, tile or unit)
    made_s, made_pv = [0, 0], [0, 0]

    def wait(name, phase):
        b = bars[name]
        while True:
            assert b.done in (phase, phase + 1), ("a phase that its parity does not tell", name, phase, b.done)
            if b.done == phase + 1:
                return
            yield True                            # (waits)

    def od(g, J):
        return ("o_done", g, J % o_done_places), J // o_done_places

    def find_units():
        for given, u in enumerate(units + [None]):
            if given >= 2:
                yield from wait(("u_free", given & 1), (given >> 1) - 1)
            ring[given & 1] = u
            bars["u_full", given & 1].arrive()
            yield False

    def next_unit(st):
        s = st["taken"] & 1
        yield from wait(("u_full", s), st["taken"] >> 1)
        st["w"] = ring[s]
        bars["u_free", s].arrive()
        st["taken"] += 1

    def load():
        st = dict(taken=0)
        issued = q = 0
        while True:
            yield from next_unit(st)
            if st["w"] is None:
                return
            n = max(st["w"])
            if n == 0:
                continue
            if q >= 2:
                yield from wait(("q_free", q & 1), (q >> 1) - 1)
            landing.append((queries, q & 1, q, "q_full"))
            q += 1
            for _ in range(n):
                s, r = issued % STAGES, issued // STAGES
                if r > 0:
                    yield from wait(("free", s), r - 1)
                landing.append((kv, s, issued, "full"))
                issued += 1
                yield False

    def products(g):
        st = dict(taken=0)
        q, j, mine, n, tile = -1, 0, 0, 0, 0
        at = None

        def reach(owed):
            nonlocal q, j, mine, n, tile, at
            crossed = False
            while True:
                if j < mine:
                    at = "there"
                    return
                if owed and (crossed or n - j > AHEAD):
                    at = "owed"
                    return
                while j < n:
                    yield from wait(("full", tile % STAGES), tile // STAGES)
                    if mine == 0 and j == 0:
                        yield from wait(("q_full", q & 1), q >> 1)
                    bars["free", tile % STAGES].arrive()
                    if mine == 0 and j == 0:
                        bars["q_free", q & 1].arrive()
                    j, tile = j + 1, tile + 1
                yield from next_unit(st)
                if st["w"] is None:
                    at = "end"
                    return
                j, mine, n = 0, st["w"][g], max(st["w"])
                q += n > 0
                crossed = True

        def scores(J):
            if j == 0:
                yield from wait(("q_full", q & 1), q >> 1)
            yield from wait(("full", tile % STAGES), tile // STAGES)
            t, u, s, last = tile, q, tile % STAGES, j == mine - 1

            def run():
                assert kv[s] == t and queries[u & 1] == u
                assert J < 2 or (read_s[g, J - 2] == 4 and made_pv[g] >= J - 1), "S over scores, or P's place, in use"
                made_s[g] = J + 1
                bars["s_full", g, J & 1].arrive()
                if last:
                    bars["q_free", u & 1].arrive()
            pipe[g].append(run)

        made = J = 0
        live = True
        owed_tiles = []                           # (stage's tile, opens a unit, unit), of the scores ahead
        while True:
            while live and made - J < 2:
                yield from reach(careful and made > J)
                if at == "owed":
                    break
                live = at == "there"
                if not live:
                    break
                owed_tiles.append((tile, j == 0, st["taken"]))
                yield from scores(made)
                made, j, tile = made + 1, j + 1, tile + 1
                yield False
            if made == J:
                return
            yield from wait(("p_ready", g, J & 1), J >> 1)
            t, opens, u = owed_tiles.pop(0)

            def run(J=J, t=t, opens=opens, u=u):
                assert kv[t % STAGES] == t and wrote_p[g, J] == 4 and made_pv[g] == J
                assert not opens or all(read_o[g, w] == 4 for w in range(1, u) if units[w - 1][g]), "O over an O that is not read"
                made_pv[g] = J + 1
                bars[od(g, J)[0]].arrive()
                bars["free", t % STAGES].arrive()
            pipe[g].append(run)
            J += 1
            yield False

    def softmax(g, quad):
        st = dict(taken=0)
        J = tile = 0
        while True:
            yield from next_unit(st)
            if st["w"] is None:
                return
            for j in range(st["w"][g]):
                yield from wait(("s_full", g, J & 1), J >> 1)
                assert made_s[g] in (J + 1, J + 2)
                read_s[g, J] += 1
                if j > 0 and rnd.random() < 0.3:  # (a maximum moves: O is scaled)
                    yield from wait(*od(g, J - 1))
                    assert made_pv[g] == J
                assert kv[(tile + j) % STAGES] == tile + j                       # (values past the end are put to 0 there)
                wrote_p[g, J] += 1
                bars["p_ready", g, J & 1].arrive()
                J += 1
                yield False
            tile += max(st["w"])
            if st["w"][g]:
                yield from wait(*od(g, J - 1))
                assert made_pv[g] == J
                yield False
                assert made_pv[g] == J
                read_o[g, st["taken"]] += 1
            yield False

    roles = [find_units(), load(), products(0), products(1)] + [softmax(g, w) for g in range(2) for w in range(4)]
    weights = [rnd.choice((1, 1, 5, 20)) for _ in range(len(roles) + 3)]         # (some are slow)
    live, idle = set(range(len(roles))), 0
    while live or landing or pipe[0] or pipe[1]:
        steps = sorted(live) + [len(roles) + k for k, some in enumerate((landing, pipe[0], pipe[1])) if some]
        i = rnd.choices(steps, [weights[s] for s in steps])[0]
        if i == len(roles):
            place, s, what, name = landing.pop(rnd.randrange(len(landing)))
            place[s] = what
            bars[name, s].arrive()
            idle = 0
        elif i > len(roles):
            pipe[i - len(roles) - 1].popleft()()
            idle = 0
        else:
            try:
                idle = idle + 1 if next(roles[i]) else 0
            except StopIteration:
                live.discard(i)
                idle = 0
        # (nothing in flight and every role waiting, many times over)
        if idle > 2000 and not (landing or pipe[0] or pipe[1]):
            raise Stuck((units, seed, {k: b.done for k, b in bars.items()}))
    tiles = [sum(u[g] for u in units) for g in range(2)]
    assert made_pv == tiles and made_s == tiles and all(read_o[g, w + 1] == (4 if u[g] else 0) for g in range(2) for w, u in enumerate(units))


def of_rows(first, rows):
    """The unit that begins at a sequence's row ``first`` and has ``rows`` of them."""
    tiles = lambda last: -(-last // COLS)   # noqa: E731
    return tiles(first + min(rows, ROWS)), tiles(first + rows) if rows > ROWS else 0


def some_units(rnd):
    return [(0, 0) if rnd.random() < 0.15 else of_rows(UNIT * rnd.choice((0, 0, 1, 2, 5)), rnd.choice((1, 1, 60, 64, 65, 128, 129, 200, 256)))
            for _ in range(rnd.randint(1, 12))]


@pytest.mark.parametrize("part", range(4))
def test_random_units(part):
    rnd = random.Random(part)
    for n in range(60):
        simulate(some_units(rnd), 1000 * part + n)


LISTS = [[], [(0, 0)] * 6, [(1, 0)] * 12, [(5, 0)] * 6, [(37, 0)] * 2 + [(2, 4)], [(2, 4)] + [(9, 0)] * 4, [(2, 4), (0, 0), (0, 0), (1, 0), (0, 0), (2, 4)],
         [of_rows(256 * n, 256) for n in (3, 2, 1, 0)], [of_rows(256, 1), of_rows(0, 256)] * 4]


@pytest.mark.parametrize("units", LISTS)
def test_units_that_one_group_has_none_of(units):
    for seed in range(12):
        simulate(units, seed)


def test_it_finds_a_product_warp_that_waits_too_far_ahead():
    with pytest.raises((Stuck, AssertionError)):
        for seed in range(40):
            simulate([(2, 4)] + [(9, 0)] * 4, seed, careful=False)


def test_it_finds_a_phase_that_a_parity_does_not_tell():
    with pytest.raises(AssertionError, match="parity"):
        rnd = random.Random(9)
        for seed in range(200):
            simulate(some_units(rnd), seed, o_done_places=1)
