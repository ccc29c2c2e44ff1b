"""The barriers of the paged attention over caches in 4 bits, in a model run in
random order on the CPU: warps that copy codes, scales and query tiles, four that
convert (a quarter of every key and value tile, and of an item's query tiles, when they
are there, after its first tiles at the latest), one that issues the matrix products, and the two halves' softmax, who
write the output. A barrier is waited for by its phase's parity alone, as on the
device, so a phase that a warp misses, or asks for two phases early, shows as a wrong
tile, an overwritten one or a run that does not end."""

import random

import pytest


CONVERTERS, STAGED = 4, 3


class Barrier:
    def __init__(self, count=1):
        self.phase, self.count, self.arrived = 0, count, 0

    def arrive(self):
        self.arrived += 1
        if self.arrived == self.count:
            self.phase, self.arrived = self.phase + 1, 0

    def done(self, parity):  # the phase that ended last has that parity
        return (self.phase & 1) != parity


def place_k(j):
    return j if j < 2 else 2 * j - 1


def place_v(j, n):
    return min(2 + 2 * j, 2 * n - 1)


def run(seed, stages, units):
    """units: (two query tiles?, key tiles) of a CTA's share, in order."""
    rng = random.Random(seed)
    new = lambda k, count=1: [Barrier(count) for _ in range(k)]  # noqa: E731
    full, empty, q_raw, q_full, q_empty = new(stages, CONVERTERS), new(stages), new(2), new(2, CONVERTERS), new(2)
    staged_full, staged_empty = new(STAGED, 2), new(STAGED, CONVERTERS)
    s_full, p_full, o_full, o_free, stat_full = new(2), new(2), new(2), new(2), new(2)
    # a tile of the ring: what each converting warp wrote to it last
    parts = [[None] * CONVERTERS for _ in range(stages)]
    free, q_tiles = [[True] * CONVERTERS for _ in range(stages)], [None, None]
    outputs = [0, 0]  # items written
    copies, products = [], []  # in flight: copies end in any order, products in theirs

    class Tiles:
        def __getitem__(self, s):
            x = parts[s]
            return x[0] if all(y == x[0] for y in x) else None

    tiles = Tiles()

    def wait(barrier, parity):
        while not barrier.done(parity):
            yield

    def places():
        for u, (_, n) in enumerate(units):
            order = {place_k(j): ("k", j) for j in range(n)} | {place_v(j, n): ("v", j) for j in range(n)}
            assert sorted(order) == list(range(2 * n))
            for place in range(2 * n):
                yield u, place, (u, *order[place])

    staged = [[None, None] for _ in range(STAGED)]
    read = [[True] * CONVERTERS for _ in range(STAGED)]

    def copier(what):  # codes or scales
        for at, (_, _, tile) in enumerate(places()):
            s = at % STAGED
            if at >= STAGED:
                yield from wait(staged_empty[s], at // STAGED - 1 & 1)
            assert all(read[s]) or staged[s][1 - what] == tile, "codes in use are overwritten"
            staged[s][what] = tile
            read[s] = [False] * CONVERTERS
            copies.append(staged_full[s].arrive)
            yield

    def queries():
        nq = 0
        for u, (pair, _) in enumerate(units):
            for t in range(2 if pair else 1):
                if nq > 1:
                    yield from wait(q_empty[nq & 1], nq // 2 - 1 & 1)
                q_tiles[nq & 1] = (u, t)
                copies.append(q_raw[nq & 1].arrive)
                nq += 1
                yield

    def converter(number):
        nq = left = 0
        for at, (u, place, tile) in enumerate(places()):
            s, f = at % stages, at % STAGED
            yield from wait(staged_full[f], at // STAGED & 1)
            assert staged[f] == [tile, tile]
            if at >= stages:
                yield from wait(empty[s], at // stages - 1 & 1)
            assert free[s][number], "a tile in use is overwritten"
            free[s][number], parts[s][number] = False, tile
            read[f][number] = True
            yield
            staged_empty[f].arrive()
            full[s].arrive()
            left = (2 if units[u][0] else 1) if place == 0 else left
            while left:
                last = place == min(stages, 2 * units[u][1]) - 1
                if not last and not q_raw[nq & 1].done(nq // 2 & 1):
                    break
                yield from wait(q_raw[nq & 1], nq // 2 & 1)
                assert q_tiles[nq & 1] == (u, nq - first_tile(u))
                q_full[nq & 1].arrive()  # (converted)
                nq, left = nq + 1, left - 1
                yield

    def first_tile(u):
        return sum(2 if pair else 1 for pair, _ in units[:u])

    def issuer():
        base = nq = 0
        np = [0, 0]

        def wait_full(place):
            yield from wait(full[(base + place) % stages], (base + place) // stages & 1)

        def scores(t, q, place, tile):
            assert tiles[(base + place) % stages] == tile and q_tiles[q & 1] == (tile[0], q - nq)
            products.append(s_full[t].arrive)

        def release(place):
            s = (base + place) % stages

            def end():
                free[s] = [True] * CONVERTERS
                empty[s].arrive()
            products.append(end)

        def weigh(t, place, tile, first):
            if first and tile[0]:
                yield from wait(o_free[t], tile[0] - 1 & 1)
            yield from wait(p_full[t], np[t] & 1)
            np[t] += 1
            assert tiles[(base + place) % stages] == tile

        for u, (pair, n) in enumerate(units):
            yield from wait_full(0)
            yield from wait(q_full[nq & 1], nq // 2 & 1)
            if pair:
                scores(0, nq, 0, (u, "k", 0))
                yield from wait(q_full[nq + 1 & 1], (nq + 1) // 2 & 1)
                scores(1, nq + 1, 0, (u, "k", 0))
                release(0)
            else:
                for j in range(min(n, 2)):
                    if j:
                        yield from wait_full(j)
                    scores(j, nq, j, (u, "k", j))
                    release(j)
            if n <= (1 if pair else 2):
                products.extend(q_empty[nq + t & 1].arrive for t in range(2 if pair else 1))
            if not pair and n == 1 and u:
                yield from wait(o_free[1], u - 1 & 1)
            ahead = 1 if pair else 2  # steps between a tile's product and the next scores in its half
            for j in range(n):
                v, k = place_v(j, n), place_k(j + ahead)
                yield from wait_full(v)
                if j + ahead < n:
                    yield from wait_full(k)
                for t in (0, 1) if pair else (j & 1,):
                    yield from weigh(t, v, (u, "v", j), j < ahead)
                    if not pair or t:
                        release(v)
                    if j + ahead < n:
                        scores(t, nq + (t if pair else 0), k, (u, "k", j + ahead))
                        if not pair or t:
                            release(k)
                    else:
                        products.append(o_full[t].arrive)
                    yield
                if j + ahead + 1 == n and n > ahead:
                    products.extend(q_empty[nq + t & 1].arrive for t in range(2 if pair else 1))
            nq += 2 if pair else 1
            base += 2 * n

    def softmax(t):
        ns = 0
        ends = [0, 0]
        for u, (pair, n) in enumerate(units):
            for _ in range(0 if pair else t, n, 1 if pair else 2):
                yield from wait(s_full[t], ns & 1)
                ns += 1
                yield
                p_full[t].arrive()
            if u:
                yield from wait(o_free[t], u - 1 & 1)
            stat_full[t].arrive()
            yield
            if pair or t == 0:  # the output
                yield from wait(stat_full[t], u & 1)
                if not pair:
                    yield from wait(stat_full[1], u & 1)
                    if n > 1:
                        yield from wait(o_full[1], ends[1] & 1)
                        ends[1] += 1
                yield from wait(o_full[t], ends[t] & 1)
                ends[t] += 1
                assert outputs[t] == u
                outputs[t] += 1
                if not pair:
                    assert outputs[1] == u
                    outputs[1] += 1
                yield
                o_free[t].arrive()
                if not pair:
                    o_free[1].arrive()
            if pair if t == 0 else not pair and n > 1:
                ends[1] += 1

    def hardware(queue, pick):
        while True:
            if queue:
                queue.pop(pick(len(queue)))()
            yield

    warps = {"codes": copier(0), "scales": copier(1), "queries": queries(), **{f"c{i}": converter(i) for i in range(CONVERTERS)},
             "mma": issuer(), "s0": softmax(0), "s1": softmax(1)}
    rest = {"tensor": hardware(products, lambda n: 0), "memory": hardware(copies, rng.randrange)}
    pace = {}
    for step in range(300_000):
        if step % 100 == 0:
            pace = {w: rng.choice([1, 1, 1, 5, 30]) for w in (*warps, *rest)}
        everyone = [*warps, *rest]
        w = rng.choices(everyone, [pace[x] for x in everyone])[0]
        try:
            next(warps[w] if w in warps else rest[w])
        except StopIteration:
            del warps[w]
            if not warps:
                return
    raise AssertionError(f"no end: {sorted(warps)} of {units}")


@pytest.mark.parametrize("stages", [4, 10])
def test_random_shares(stages):
    for seed in range(150):
        rng = random.Random(seed)
        units = [(rng.random() < 0.5, rng.choice([1, 1, 2, 3, 4, 5, 9])) for _ in range(rng.randint(1, 9))]
        run(seed, stages, units)


@pytest.mark.parametrize("stages", [4, 10])
def test_short_units_after_long_ones(stages):
    for seed in range(40):
        run(seed, stages, [(True, 1), (True, 3), (False, 1), (False, 2), (False, 1), (False, 1), (True, 2), (False, 7), (False, 1)])
