"""CPU: the barriers of attention over a paged cache on tcgen05.  Its roles (producers, products, softmax) are stepped in random order as in
csrc/attend_pages_tc.cu; a wait by parity must never pass, or hold, for another phase than the one meant, no place is written while it is
read, and everything must end."""
import random

import pytest

from tests.test_attend_protocol import Barrier, Machine

WARPS = 4                                                          # of a stream's softmax, of its producers


class Place:
    """Something that roles write and read in turn: what it holds, and who still reads it."""

    def __init__(self):
        self.holds, self.readers = None, 0

    def write(self, what):
        assert self.readers == 0, "written while it is read"
        self.holds = what

    def read(self, what):
        assert self.holds == what, "holds %s, not %s" % (self.holds, what)


def build(seed, segments, copies):
    """segments: tiles (t0, t1) of each of a CTA's items, one after another."""
    m = Machine(seed)
    rng = m.rng
    full = {(s, v, p): Barrier(WARPS) for s in range(2) for v in range(2) for p in range(2)}
    empty = {k: Barrier(1) for k in full}
    s_full, p_ready, o_done = ({(s, p): Barrier(n) for s in range(2) for p in range(2)} for n in (1, WARPS, 1))
    drained = [Barrier(1), Barrier(1)]
    q_full, q_empty, met, sent = Barrier(2 * WARPS), Barrier(2 * WARPS + 2), Barrier(2 * WARPS), Barrier(2 * WARPS)
    rows, handed, scores = Place(), Place(), {k: Place() for k in s_full}
    operand = {k: [Place() for _ in range(WARPS)] for k in full}    # each producing warp's part
    info = {(s, i): [Place() for _ in range(WARPS)] for s in range(2) for i in range(4)}
    outputs = [Place(), Place()]
    finished = []
    jobs_of = lambda seg, s: (seg[1] - seg[0] + 1 - s) // 2
    queues = [[], []]                                               # a stream's products, in order
    m.queues += queues

    def products(s):
        done = 0
        for n, seg in enumerate(segments):
            jobs = jobs_of(seg, s)
            yield q_full, n
            q_empty.arrive()
            for k in range(-2, jobs):
                job = done + k
                p = job & 1
                if k >= 0:
                    yield full[s, 1, p], job >> 1
                    yield p_ready[s, p], job >> 1
                    for w in range(WARPS):
                        operand[s, 1, p][w].read(job)
                        operand[s, 1, p][w].readers += 1
                    scores[s, p].read(("weights", job))
                    scores[s, p].readers += 1

                    def outputs_made(job=job, p=p, n=n):
                        outputs[s].write((n, job))
                        for w in range(WARPS):
                            operand[s, 1, p][w].readers -= 1
                        scores[s, p].readers -= 1
                        o_done[s, p].arrive()
                        empty[s, 1, p].arrive()
                    queues[s].append(outputs_made)
                if k + 2 < jobs:
                    yield full[s, 0, p], (job + 2) >> 1
                    for w in range(WARPS):
                        operand[s, 0, p][w].read(job + 2)
                        operand[s, 0, p][w].readers += 1
                    rows.read(n)
                    rows.readers += 1

                    def scores_made(job=job + 2, p=p):
                        scores[s, p].write(("scores", job))
                        rows.readers -= 1
                        for w in range(WARPS):
                            operand[s, 0, p][w].readers -= 1
                        s_full[s, p].arrive()
                        empty[s, 0, p].arrive()
                    queues[s].append(scores_made)
            done += jobs
        queues[s].append(lambda: drained[s].arrive())
        yield drained[s], 0

    def producer(s, w):
        for done in range(sum(jobs_of(seg, s) for seg in segments)):
            p = done & 1
            for v in range(2):
                if done > 1:
                    yield empty[s, v, p], (done >> 1) - 1
                operand[s, v, p][w].write(done)
                if v == 0:
                    info[s, done & 3][w].write(done)
                full[s, v, p].arrive()

    def softmax(s, w):
        done = 0
        for n, seg in enumerate(segments):
            if n > 0:
                yield q_empty, n - 1
            rows.write(n)
            handed.write(n)
            q_full.arrive()
            yield q_full, n
            jobs = jobs_of(seg, s)
            for k in range(jobs):
                yield s_full[s, done & 1], done >> 1
                place = scores[s, done & 1]
                assert place.holds in (("scores", done), ("weights", done))
                for x in range(WARPS):
                    info[s, done & 3][x].read(done)
                    info[s, done & 3][x].readers += 1
                if k > 0 and rng.random() < 0.5:                    # the reference grows: outputs are scaled
                    yield o_done[s, (done - 1) & 1], (done - 1) >> 1
                    outputs[s].read((n, done - 1))
                for x in range(WARPS):
                    info[s, done & 3][x].readers -= 1
                place.write(("weights", done))
                p_ready[s, done & 1].arrive()
                done += 1
            if jobs:
                yield o_done[s, (done - 1) & 1], (done - 1) >> 1
            met.arrive()
            yield met, n
            for x in range(2):
                if jobs_of(seg, x):
                    outputs[x].read((n, sum(jobs_of(y, x) for y in segments[:n + 1]) - 1))
                    outputs[x].readers += 1
            assert rows.readers == 0, "rows' place is reused while products read it"
            if copies == 2:
                sent.arrive()
                yield sent, n
            handed.readers += 1                                     # (partial results pass through the rows' place)
            yield met, n
            handed.readers -= 1
            for x in range(2):
                if jobs_of(seg, x):
                    outputs[x].readers -= 1
            finished.append((n, s, w))
            q_empty.arrive()

    for s in range(2):
        m.roles.append(products(s))
        m.roles += [producer(s, w) for w in range(WARPS)] + [softmax(s, w) for w in range(WARPS)]
    return m, finished


@pytest.mark.parametrize("copies", [1, 2])
@pytest.mark.parametrize("seed", range(150))
def test_every_wait_is_for_its_phase(seed, copies):
    rng = random.Random(seed)
    segments = []
    for _ in range(rng.randrange(1, 6)):
        t0 = rng.randrange(4)
        segments.append((t0, t0 + rng.choice([1, 1, 2, 3, rng.randrange(1, 9)])))
    m, finished = build(seed, segments, copies)
    m.run()
    assert len(finished) == len(segments) * 2 * WARPS


def test_a_segment_of_one_tile_after_another():
    m, finished = build(7, [(0, 1)] * 12, 2)                        # the second stream never has a tile
    m.run()
    assert len(finished) == 12 * 2 * WARPS
