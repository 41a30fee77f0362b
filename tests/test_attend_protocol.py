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
    nr = nu if mt == 2 else nu // 2                       # places of a ring
    for seed in range(100):
        rng = random.Random(seed)
        segs = segments_of(rng, [rng.choice([1, 1, 1, 2, 3, 7]) for _ in range(rng.randint(1, 8))], rng.randint(1, 16))
        n_tail = rng.randint(1, 2)                        # tiles of an item with new tokens
        m = Machine(seed)
        full, empty = [Barrier(1) for _ in range(nu)], [Barrier(mt) for _ in range(nu)]
        q_full, q_empty = Barrier(2), Barrier(2)
        s_full, p_half, p_ready, o_done, o_free, v_look, v_ready = ([Barrier(1) for _ in range(2)] for _ in range(7))
        turn = [Barrier(1), Barrier(1)]
        copies, mma = [[] for _ in range(nu)], [[], []]
        m.queues = copies + mma

        def place(s, unit):
            return (0 if mt == 2 else s * nr) + unit % nr

        def jobs_of(s, tiles):
            return tiles if mt == 2 else (tiles + 1 - s) // 2

        def producer():
            made = [0, 0]
            for t0, t1, _ in segs:
                for t in range(t1 - t0):
                    s = 0 if mt == 2 else t & 1
                    for _ in range(2):
                        unit = made[s]
                        if unit >= nr:
                            yield empty[place(s, unit)], unit // nr - 1
                        copies[place(s, unit)].append(full[place(s, unit)].arrive)
                        made[s] += 1

        def products(s):
            n, tails, done, used = 0, 0, 0, 0
            for seg, (t0, t1, tiles) in enumerate(segs):
                jobs = jobs_of(s, t1 - t0)

                def scores(k):
                    unit = 2 * (n + k)
                    yield full[place(s, unit)], unit // nr
                    mma[s] += [s_full[s].arrive, empty[place(s, unit)].arrive]

                yield q_full, seg
                if jobs:
                    yield from scores(0)
                for k in range(jobs):
                    t, unit = k if mt == 2 else 2 * k + s, 2 * (n + k) + 1
                    yield full[place(s, unit)], unit // nr
                    tail = t0 + t >= tiles - n_tail
                    if tail:
                        v_look[s].arrive()
                    if k == 0:
                        if used:
                            yield o_free[s], used - 1
                        used += 1
                    if tail:
                        yield v_ready[s], tails
                        tails += 1
                    yield p_half[s], done
                    yield p_ready[s], done
                    mma[s] += [o_done[s].arrive, empty[place(s, unit)].arrive]
                    done += 1
                    if k + 1 < jobs:
                        yield from scores(k + 1)
                n += jobs

        def looks():
            tails = [0, 0]
            for t0, t1, tiles in segs:
                for t in range(max(t0, tiles - n_tail, 0), t1):
                    mine = [0, 1] if mt == 2 else [(t - t0) & 1]
                    for s in mine:
                        yield v_look[s], tails[s]
                        tails[s] += 1
                    for s in mine:
                        v_ready[s].arrive()

        def softmax(s):
            done = 0
            for seg, (t0, t1, _) in enumerate(segs):
                if seg:
                    yield q_empty, seg - 1
                q_full.arrive()
                jobs = jobs_of(s, t1 - t0)
                for k in range(jobs):
                    yield s_full[s], done
                    if positions:
                        yield full[place(s, 2 * done + 1)], (2 * done + 1) // nr
                    if k and rng.random() < 0.5:
                        yield o_done[s], done - 1
                    if mt == 2 and done >= 1 - s:
                        yield turn[s], done - 1 + s
                    p_half[s].arrive()
                    yield None                            # (others may go on)
                    p_ready[s].arrive()
                    if mt == 2:
                        turn[1 - s].arrive()
                    done += 1
                q_empty.arrive()
                if jobs:
                    yield o_done[s], done - 1
                    o_free[s].arrive()

        m.roles = [producer(), products(0), products(1), looks(), softmax(0), softmax(1)]
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
