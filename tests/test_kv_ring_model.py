"""A model of the barriers between the paged attention kernel's warps, run in
random order on the CPU: a warp that copies query and key tiles, one that copies
values, one that issues the matrix products, the two halves' softmax, and the
warps that write a unit's output. A barrier is waited for by its phase's parity
alone, as on the device, so a phase that a warp misses, or asks for two phases
early, shows as a wrong tile, an overwritten one or a run that does not end."""

import random

import pytest


class Barrier:
    def __init__(self):
        self.phase = 0

    def arrive(self):
        self.phase += 1

    def done(self, parity):  # the phase that ended last has that parity
        return (self.phase & 1) != parity


def place_k(j):
    return j if j < 2 else 2 * j - 1


def place_v(j, n):
    return min(2 + 2 * j, 2 * n - 1)


def run(seed, stages, units):
    """units: (two query tiles?, key tiles) of a CTA's share, in order."""
    rng = random.Random(seed)
    new = lambda k: [Barrier() for _ in range(k)]  # noqa: E731
    full, empty, q_full, q_empty = new(stages), new(stages), new(2), new(2)
    s_full, p_full, o_full, o_free, stat_full = new(2), new(2), new(2), new(2), new(2)
    tiles, free, q_tiles = [None] * stages, [True] * stages, [None, None]
    copies, products = [], []  # in flight: copies end in any order, products in theirs

    def wait(barrier, parity):
        while not barrier.done(parity):
            yield

    def copier(values):
        base = nq = 0
        for u, (pair, n) in enumerate(units):
            for j in range(n):
                at = base + (place_v(j, n) if values else place_k(j))
                s = at % stages
                if at >= stages:
                    yield from wait(empty[s], at // stages - 1 & 1)
                assert free[s], "a tile in use is overwritten"
                free[s], tiles[s] = False, (u, "v" if values else "k", j)
                copies.append(full[s].arrive)
                yield
                if j == 0 and not values:
                    for t in range(2 if pair else 1):
                        if nq > 1:
                            yield from wait(q_empty[nq & 1], nq // 2 - 1 & 1)
                        q_tiles[nq & 1] = (u, t)
                        copies.append(q_full[nq & 1].arrive)
                        nq += 1
                        yield
            base += 2 * n

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
                free[s] = True
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

    def writer():
        ends = [0, 0]
        for u, (pair, n) in enumerate(units):
            for tile in range(2 if pair else 1):
                yield from wait(stat_full[tile], u & 1)
                if not pair:
                    yield from wait(stat_full[1], u & 1)
                    if n > 1:
                        yield from wait(o_full[1], ends[1] & 1)
                        ends[1] += 1
                yield from wait(o_full[tile], ends[tile] & 1)
                ends[tile] += 1
                yield
                o_free[tile].arrive()
                if not pair:
                    o_free[1].arrive()

    def hardware(queue, pick):
        while True:
            if queue:
                queue.pop(pick(len(queue)))()
            yield

    warps = {"k": copier(False), "v": copier(True), "mma": issuer(), "s0": softmax(0), "s1": softmax(1), "out": writer()}
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


@pytest.mark.parametrize("stages", [5, 11])
def test_random_shares(stages):
    for seed in range(150):
        rng = random.Random(seed)
        units = [(rng.random() < 0.5, rng.choice([1, 1, 2, 3, 4, 5, 9])) for _ in range(rng.randint(1, 9))]
        run(seed, stages, units)


@pytest.mark.parametrize("stages", [5, 11])
def test_short_units_after_long_ones(stages):
    for seed in range(40):
        run(seed, stages, [(True, 1), (True, 3), (False, 1), (False, 2), (False, 1), (False, 1), (True, 2), (False, 7), (False, 1)])
