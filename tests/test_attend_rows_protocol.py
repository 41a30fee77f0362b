"""CPU: the barrier by which a segment's rows of Q are replaced in csrc/attend_tc.cu, with up to 128 rows (two streams of key tiles,
one of which may have no tile in a segment), and the flags that say that V of a new token was not finite.  The kernel's roles are
stepped in random order, some thousand orders; how many arrivals the barrier waits for, and whose flag is read, is taken from the
source."""
import os
import random
import re

import pytest

from tests.test_attend_protocol import Barrier, Machine, segments_of

SOURCE = os.path.join(os.path.dirname(__file__), "..", "paper_2604_06746_b200", "csrc", "attend_tc.cu")


def arrivals_in_source():
    with open(SOURCE) as f:
        return int(re.search(r"mbar_init\(q_empty, (\d+)\);", f.read()).group(1))


def flags_in_source():
    """"own": a stream answers for the tiles of its own; "first": stream 0 for those of both."""
    with open(SOURCE) as f:
        text = f.read()
    return "own" if re.search(r"const bool odd = odd_v\[s\] && [^|\n]*;", text) else "first"


def step(seed, nu, positions, arrivals, flags="own"):
    """One random order.  ``arrivals``: of q_empty, four for every stream's softmax and, where there are more, one for its products."""
    by_products = {8: False, 10: True}[arrivals]
    nr = nu // 2                                          # places of a ring, a ring a stream
    rng = random.Random(seed)
    segs = segments_of(rng, [rng.choice([1, 1, 1, 2, 3, 7]) for _ in range(rng.randint(1, 8))], rng.randint(1, 16))
    n_tail = rng.randint(1, 2)                            # tiles of an item with new tokens
    m = Machine(seed)
    full, empty = [Barrier(1) for _ in range(nu)], [Barrier(1) for _ in range(nu)]
    q_full, q_empty = Barrier(2), Barrier(arrivals)
    s_full, p_ready, o_done, o_free, v_look, v_ready = ([Barrier(1) for _ in range(2)] for _ in range(6))
    looked = set()                                        # (segment, tile) whose V was looked through
    copies, mma = [[] for _ in range(nu)], [[], []]
    m.queues = copies + mma

    def place(s, unit):
        return s * nr + unit % nr

    def producer():
        made = [0, 0]
        for t0, t1, _ in segs:
            for t in range(t1 - t0):
                s = t & 1
                for _ in range(2):
                    if made[s] >= nr:
                        yield empty[place(s, made[s])], made[s] // nr - 1
                    copies[place(s, made[s])].append(full[place(s, made[s])].arrive)
                    made[s] += 1

    def products(s):
        n, tails, done, used = 0, 0, 0, 0
        for seg, (t0, t1, tiles) in enumerate(segs):
            jobs = (t1 - t0 + 1 - s) // 2

            def scores(k):
                unit = 2 * (n + k)
                yield full[place(s, unit)], unit // nr
                mma[s] += [s_full[s].arrive, empty[place(s, unit)].arrive]

            yield q_full, seg
            if by_products:
                q_empty.arrive()
            if jobs:
                yield from scores(0)
            for k in range(jobs):
                unit = 2 * (n + k) + 1
                yield full[place(s, unit)], unit // nr
                tail = t0 + 2 * k + s >= tiles - n_tail
                if tail:
                    v_look[s].arrive()
                if k == 0:
                    if used:
                        yield o_free[s], used - 1
                    used += 1
                if tail:
                    yield v_ready[s], tails
                    tails += 1
                yield p_ready[s], done
                mma[s] += [o_done[s].arrive, empty[place(s, unit)].arrive]
                done += 1
                if k + 1 < jobs:
                    yield from scores(k + 1)
            n += jobs

    def looks():
        tails = [0, 0]
        for seg, (t0, t1, tiles) in enumerate(segs):
            for t in range(max(t0, tiles - n_tail, 0), t1):
                s = (t - t0) & 1
                yield v_look[s], tails[s]
                tails[s] += 1
                looked.add((seg, t))
                v_ready[s].arrive()

    def softmax(s):
        done = 0
        for seg, (t0, t1, tiles) in enumerate(segs):
            if seg:
                yield q_empty, seg - 1
            q_full.arrive()
            jobs = (t1 - t0 + 1 - s) // 2
            for k in range(jobs):
                yield s_full[s], done
                if positions:
                    yield full[place(s, 2 * done + 1)], (2 * done + 1) // nr
                if k and rng.random() < 0.5:
                    yield o_done[s], done - 1
                p_ready[s].arrive()
                done += 1
            q_empty.arrive(4)
            if jobs:
                yield o_done[s], done - 1
                # the flag is read here: what it stands for has to be there
                for t in range(max(t0, tiles - n_tail, 0), t1):
                    if (t - t0) & 1 == s if flags == "own" else s == 0:
                        assert (seg, t) in looked, "the flag is read before tile %d was looked through" % t
                o_free[s].arrive()

    m.roles = [producer(), products(0), products(1), looks(), softmax(0), softmax(1)]
    m.run()


@pytest.mark.parametrize("nu", [4, 6, 8])
@pytest.mark.parametrize("positions", [False, True])
def test_rows_are_replaced_behind_every_reader(nu, positions):
    for seed in range(4000):
        step(seed, nu, positions, arrivals_in_source(), flags_in_source())


@pytest.mark.parametrize("arrivals,flags", [(8, "own"), (10, "first")])
def test_the_model_sees_what_can_be_lost(arrivals, flags):
    """Without the products' arrivals some orders leave a stream behind; where stream 0 answers for both, some let it read too soon."""
    lost = 0
    for seed in range(4000):
        for nu in (4, 6, 8):
            try:
                step(seed, nu, False, arrivals, flags)
            except AssertionError:
                lost += 1
    assert lost > 0
