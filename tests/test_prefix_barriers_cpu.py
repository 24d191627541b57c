"""The barriers of the tensor-core kernel of the shared-prefix attention (csrc/prefix_attn_tc.cuh), played through in random order.

A wait on an mbarrier names the parity of a phase and so cannot tell a phase from the one before the last. The model has the kernel's
threads (two copy warps, two MMA threads with their queues of products, two softmax groups), its rings and its barriers; copies land in any
order, some of them very late. Every wait that is passed is compared with what it stands for: the tile, queries, mask and segment that the thread
goes on to use have to be there, and nobody may be left waiting."""
import random

import pytest


class Bar:
    def __init__(self, count):
        self.count, self.arrived, self.phase = count, 0, 0

    def arrive(self):
        self.arrived += 1
        if self.arrived == self.count:
            self.arrived, self.phase = 0, self.phase + 1

    def passes(self, parity):
        return (self.phase & 1) != parity


def play(segs, NK, NV, NF, seed, slow, NI=12):
    """segs: (key tiles, two query tiles) of each segment; slow: steps that a softmax group takes a tile. Returns the first thing that goes wrong, or None."""
    r = random.Random(seed)
    full = {k: [Bar(1) for _ in range(NF)] for k in "KV"}
    empty = {"K": [Bar(2) for _ in range(NK)], "V": [Bar(2) for _ in range(NV)]}
    q_full, q_empty = [Bar(1), Bar(1)], [Bar(4), Bar(4)]           # q_empty: two MMA threads, two softmax groups
    s_full, p_full, o_full, turn_bar = ([Bar(1), Bar(1)] for _ in range(4))
    stage = {"K": [None] * NK, "V": [None] * NV}
    slots, cur, info, flight, wrong = [None, None], [None] * 4, [None] * NI, [], []
    queue = [[], []]

    def expect(what, got, want):
        if got != want:
            wrong.append((what, got, want))

    def copy(kind):
        N, st, phase, x, before = len(stage[kind]), 0, 1, 0, 0
        for k, (n, two) in enumerate(segs):
            def issue():
                nonlocal st, phase, x
                if kind == "K":
                    info[x % NI] = x
                yield empty[kind][st], phase
                stage[kind][st] = ("on its way", x)
                flight.append([kind, x, st, r.randint(0, 60) if r.random() < 0.15 else r.randint(0, 4)])
                x, st = x + 1, st + 1
                if st == N:
                    st, phase = 0, phase ^ 1
            j = 0
            if kind == "K":
                wait_for = k - 1 if two or before else k - 2
                before = two
                if wait_for == k - 1:
                    while j < min(n, 2):
                        yield from issue()
                        j += 1
                if wait_for >= 0:
                    yield q_empty[wait_for & 1], wait_for >> 1 & 1
                cur[k & 3] = (k, n, two)
                for h in (0, 1) if two else (k & 1,):
                    slots[h] = ("on its way", k)
                flight.append(["Q", k, None, r.randint(0, 10)])
            while j < n:
                yield from issue()
                j += 1
        if kind == "K":
            k = len(segs)
            if k > 1:
                yield q_empty[k & 1], (k >> 1) - 1 & 1
            cur[k & 3] = (k, 0, 0)
            q_full[k & 1].arrive()

    def release(bar, two):
        bar.arrive()
        if not two:
            bar.arrive()

    def mma(t):
        tile0, p_phase, turn, k = 0, 0, t ^ 1, 0
        while True:
            yield q_full[k & 1], k >> 1 & 1
            seg, n, two = cur[k & 3]
            expect("segment", seg, k)
            if n == 0 or seg != k:
                return
            first, step = (0, 1) if two else (t, 2)
            if first >= n:
                queue[t].append(q_empty[k & 1].arrive)
            for j in range(first, (n if two else n + 1) + 1, step):
                v, x, y = j - step, tile0 + j - step, tile0 + j
                do_v, do_s = first <= v < n, j < n
                if do_v:
                    yield full["V"][x % NF], x // NF & 1
                    expect("V", stage["V"][x % NV], ("there", x))
                if do_s:
                    yield full["K"][y % NF], y // NF & 1
                    expect("K", stage["K"][y % NK], ("there", y))
                if two:
                    yield turn_bar[t], turn
                    turn ^= 1
                if do_v:
                    yield p_full[t], p_phase
                    p_phase ^= 1

                    def values(x=x, two=two, last=v + step >= n):
                        expect("V in use", stage["V"][x % NV], ("there", x))
                        release(empty["V"][x % NV], two)
                        if last:
                            o_full[t].arrive()
                    queue[t].append(values)
                if two:
                    turn_bar[t ^ 1].arrive()
                if do_s:
                    def scores(x=y, k=k, two=two, last=j + step >= n):
                        expect("K in use", stage["K"][x % NK], ("there", x))
                        expect("queries", slots[t if two else k & 1], ("there", k))
                        s_full[t].arrive()
                        release(empty["K"][x % NK], two)
                        if last:
                            q_empty[k & 1].arrive()
                    queue[t].append(scores)
            tile0, k = tile0 + n, k + 1

    def softmax(t):
        tile0, s_phase, o_phase, k = 0, 0, 0, 0
        while True:
            yield q_full[k & 1], k >> 1 & 1
            seg, n, two = cur[k & 3]
            expect("segment", seg, k)
            if n == 0 or seg != k:
                return
            q_empty[k & 1].arrive()
            first, step = (0, 1) if two else (t, 2)
            for j in range(first, n, step):
                yield s_full[t], s_phase
                s_phase ^= 1
                x = tile0 + j
                if r.random() < 0.3:                     # a tile with missing keys: its V rows are zeroed
                    yield full["V"][x % NF], x // NF & 1
                    expect("V to zero", stage["V"][x % NV], ("there", x))
                for _ in range(slow[t]):
                    yield None
                expect("mask", info[x % NI], x)
                p_full[t].arrive()
            if n > first:
                yield o_full[t], o_phase
                o_phase ^= 1
            for _ in range(slow[t]):
                yield None
            expect("segment at its end", cur[k & 3][0], k)
            tile0, k = tile0 + n, k + 1

    agents = [copy("K"), copy("V"), mma(0), mma(1), softmax(0), softmax(1)]
    waits, alive = [None] * 6, set(range(6))
    while alive or queue[0] or queue[1]:
        for f in flight:
            f[3] -= r.random() < 0.5
        can = [("run", i) for i in sorted(alive) if waits[i] is None or waits[i][0].passes(waits[i][1])]
        can += [("done", t) for t in (0, 1) if queue[t]]
        can += [("land", i) for i, f in enumerate(flight) if f[3] <= 0]
        if not can:
            if flight:
                continue
            return "nobody can go on"
        what, i = r.choice(can)
        if what == "run":
            try:
                waits[i] = next(agents[i])
            except StopIteration:
                alive.discard(i)
        elif what == "done":
            queue[i].pop(0)()
        else:
            kind, x, st, _ = flight.pop(i)
            if kind == "Q":
                for h in (0, 1):
                    if slots[h] == ("on its way", x):
                        slots[h] = ("there", x)
                q_full[x & 1].arrive()
            else:
                stage[kind][st] = ("there", x)
                full[kind][x % NF].arrive()
        if wrong:
            return wrong[0]
    return None


def schedules(n):
    r = random.Random(1)
    for seed in range(n):
        most, pairs = r.choice([1, 2, 2, 3, 4, 9]), r.choice([0, 0, 0.1, 0.5])
        segs = [(r.randint(1, most), int(r.random() < pairs)) for _ in range(r.randint(1, 25))]
        yield seed, segs, r.choice([(0, 0), (3, 3), (0, 25), (25, 0), (1, 8)])


@pytest.mark.parametrize("NK,NV", [(2, 3), (5, 5)])      # head_dim 128, 64
def test_no_wait_takes_one_phase_for_another(NK, NV):
    for seed, segs, slow in schedules(500):
        assert play(segs, NK, NV, 8, seed, slow) is None, (seed, segs, slow)


@pytest.mark.parametrize("NK,NV,NF", [(2, 3, 3), (5, 5, 5)])
def test_a_barrier_a_stage_would_not_do(NK, NV, NF):
    assert any(play(segs, NK, NV, NF, seed, slow) for seed, segs, slow in schedules(400))
