"""CPU: the barriers of the attention kernels over a compacted cache.  Their roles (copies, products, looking through V, softmax) are
stepped in random order as in csrc/attend_tc.cu and csrc/attend_mma.cu; a wait by parity must never pass, or hold, for another
phase than the one meant, and everything must end."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count, self.left, self.phase = count, count, 0

    def arrive(self, n=1):
        self.left -= n
        assert self.left >= 0, "more arrivals than a phase has"
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1


class Machine:
    """Roles are generators that yield (barrier, phase) to wait for; events (a copy, an MMA's commit) happen at random times, those
    of one queue in order."""

    def __init__(self, seed):
        self.rng, self.roles, self.queues = random.Random(seed), [], []

    def run(self):
        waits = {r: None for r in self.roles}
        live = list(self.roles)
        while live or any(self.queues):
            ready = [("role", r) for r in live if waits[r] is None or self.passes(*waits[r])]
            ready += [("event", q) for q in self.queues if q]
            assert ready, "nothing can go on: " + str([(n, b.phase, p) for n, (b, p) in ((r.__name__, waits[r]) for r in live)])
            kind, x = self.rng.choice(ready)
            if kind == "event":
                x.pop(0)()
                continue
            if waits[x] is not None:
                barrier, phase = waits[x]
                assert barrier.phase == phase + 1, "%s passed for phase %d at %d" % (x.__name__, phase, barrier.phase)
            try:
                waits[x] = next(x)
            except StopIteration:
                live.remove(x)

    @staticmethod
    def passes(barrier, phase):
        return barrier.phase & 1 != phase & 1


def segments_of(rng, tiles_of_items, run):
    """(t0, t1, tiles) of a CTA that begins somewhere in the first item."""
    out, first, left = [], True, run
    for tiles in tiles_of_items:
        t0 = rng.randrange(tiles) if first else 0
        t1 = min(tiles, t0 + left)
        out.append((t0, t1, tiles))
        left -= t1 - t0
        first = False
        if left == 0:
            break
    return out


@pytest.mark.parametrize("mt", [1, 2])
@pytest.mark.parametrize("nu", [4, 5, 6, 8])
@pytest.mark.parametrize("positions", [False, True])
def test_tensor_core_kernel(mt, nu, positions):
    for seed in range(60):
        rng = random.Random(seed)
        segs = segments_of(rng, [rng.choice([1, 1, 1, 2, 3, 7]) for _ in range(rng.randint(1, 8))], rng.randint(1, 16))
        n_tail = rng.randint(1, 2)                        # tiles of an item with new tokens
        m = Machine(seed)
        full, empty = [Barrier(1) for _ in range(nu)], [Barrier(1) for _ in range(nu)]
        q_full, q_empty, v_look, v_ready = Barrier(2), Barrier(1), Barrier(1), Barrier(2)
        s_full, p_ready, o_done, o_free = ([Barrier(c) for _ in range(2)] for c in (1, 1, 1, 1))
        copies = [[] for _ in range(nu)]
        mma = []
        m.queues = copies + [mma]

        def producer():
            n = 0
            for t0, t1, _ in segs:
                for _ in range(2 * (t1 - t0)):
                    if n >= nu:
                        yield empty[n % nu], n // nu - 1
                    copies[n % nu].append(full[n % nu].arrive)
                    n += 1

        def products():
            n, tails, done, used = 0, 0, [0, 0], [0, 0]
            for seg, (t0, t1, tiles) in enumerate(segs):
                jobs = (t1 - t0) * mt

                def scores(j):
                    unit = 2 * (n + j // mt)
                    yield full[unit % nu], unit // nu
                    mma.append(s_full[j & 1].arrive)
                    if j % mt == mt - 1:
                        mma.append(empty[unit % nu].arrive)
                    if j == jobs - 1:
                        mma.append(q_empty.arrive)

                yield q_full, seg
                for j in range(min(2, jobs)):
                    yield from scores(j)
                for j in range(jobs):
                    s, t = j & 1, j // mt
                    unit = 2 * (n + t) + 1
                    yield full[unit % nu], unit // nu
                    tail = t0 + t >= tiles - n_tail and j % mt == 0
                    if tail:
                        v_look.arrive()
                    if j < 2:
                        if used[s]:
                            yield o_free[s], used[s] - 1
                        used[s] += 1
                    yield p_ready[s], done[s]
                    if tail:
                        yield v_ready, tails
                        tails += 1
                    mma.append(o_done[s].arrive)
                    if j % mt == mt - 1:
                        mma.append(empty[unit % nu].arrive)
                    done[s] += 1
                    if j + 2 < jobs:
                        yield from scores(j + 2)
                n += t1 - t0

        def helper():
            tails = 0
            for seg, (t0, t1, tiles) in enumerate(segs):
                if seg:
                    yield q_empty, seg - 1
                q_full.arrive()
                for _ in range(max(t0, tiles - n_tail, 0), t1):
                    yield v_look, tails
                    tails += 1
                    v_ready.arrive()

        def softmax(s):
            n, done = 0, 0
            for t0, t1, _ in segs:
                tiles = t1 - t0
                jobs = tiles if mt == 2 else (tiles + 1 - s) // 2
                for k in range(jobs):
                    yield s_full[s], done
                    if positions:
                        unit = 2 * (n + (k if mt == 2 else 2 * k + s)) + 1
                        yield full[unit % nu], unit // nu
                    if k and rng.random() < 0.5:
                        yield o_done[s], done - 1
                    p_ready[s].arrive()
                    done += 1
                if jobs:
                    yield o_done[s], done - 1
                    o_free[s].arrive()
                n += tiles

        m.roles = [producer(), products(), helper(), helper(), softmax(0), softmax(1)]
        m.run()


@pytest.mark.parametrize("stages,groups", [(4, 4), (8, 4), (4, 2), (6, 2), (8, 2)])
def test_ring_of_the_kernels_with_groups(stages, groups):
    for seed in range(60):
        m = Machine(seed)
        run = random.Random(seed).randint(1, 40)
        full, empty = [Barrier(1) for _ in range(stages)], [Barrier(4) for _ in range(stages)]
        m.queues = copies = [[] for _ in range(stages)]

        def producer():
            for n in range(run):
                if n >= stages:
                    yield empty[n % stages], n // stages - 1
                copies[n % stages].append(full[n % stages].arrive)

        def warp(group):
            for n in range(group, run, groups):
                yield full[n % stages], n // stages
                empty[n % stages].arrive()

        m.roles = [producer()] + [warp(g) for g in range(groups) for _ in range(4)]
        m.run()
