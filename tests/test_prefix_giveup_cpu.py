"""What the lanes of a warp that issues products do when a bounded wait runs out (csrc/prefix_attn_tc.cuh, mma_role), played through in random order.

Every lane looks at a barrier by itself, until it finds the phase complete, finds that another role has given up, or its limit runs out. Lanes of one warp may
find different things. Behind the waits of a step stands a barrier of the whole warp, and another one behind the loop: all 32 lanes have to stand at the
same one for any to go on. With a vote behind the waits of a step the lanes go the same way; without one they do not."""
import random

import pytest


def play(steps, vote, seed):
    """steps: for each, when its phase completes (None: never). Returns how many steps the lanes acted on, or None if they are stuck."""
    r = random.Random(seed)
    abort = r.choice([None, None, r.randint(0, 60)])               # when another role gives up
    limit = r.randint(20, 60)
    now = [0] * 32                                                # a lane's own time
    acted = [0] * 32
    left = [False] * 32
    for done in steps:
        ok = [True] * 32
        for i in range(32):
            if left[i]:
                continue
            t0 = now[i]
            while True:
                now[i] += r.choice([1, 1, 2, 7])                  # lanes that have parted poll at their own pace
                if done is not None and now[i] >= done:
                    break
                if (abort is not None and now[i] >= abort) or now[i] - t0 > limit:
                    ok[i] = False
                    break
        if vote:
            assert len(set(left)) == 1                            # __all_sync names all lanes: they come together here
            ok = [all(ok)] * 32
            now = [max(now)] * 32
        for i in range(32):
            left[i] |= not ok[i]
            acted[i] += not left[i]
        if any(left) and not all(left):
            return None                                           # some at the step's barrier, some at the one behind the loop
        if all(left):
            break
        now = [max(now)] * 32
    assert len(set(acted)) == 1
    return acted[0]


def programs(n):
    r = random.Random(1)
    for seed in range(n):
        t, steps = 0, []
        for _ in range(r.randint(1, 12)):
            t += r.randint(0, 30)
            steps.append(t)
        if r.random() < 0.5:
            steps.append(None)
        yield seed, steps


def test_the_lanes_leave_together():
    for seed, steps in programs(3000):
        assert play(steps, True, seed) is not None


def test_without_a_vote_they_would_not():
    assert any(play(steps, False, seed) is None for seed, steps in programs(3000))


def end_of_block(tiles, stages, drain, seed):
    """A copy warp issues its tiles as stages come free, the roles behind it use them up, or give up at some time. Returns how many copies are in flight
    when the last of them has left."""
    r = random.Random(seed)
    give_up = r.choice([None, r.randint(0, 60)])
    t, lands, used = 0, [], []
    for x in range(tiles):
        if x >= stages:
            if used[x - stages] is None:
                break                                             # its stage stays taken: the copy warp sees the others give up
            t = max(t, used[x - stages])
        t += r.randint(1, 3)
        lands.append(t + (r.randint(10, 100) if r.random() < 0.2 else r.randint(1, 10)))
        at = max(lands[-1], max([u for u in used if u is not None], default=0)) + r.randint(1, 5)
        used.append(at if give_up is None or at < give_up and None not in used else None)
    end_copy = t
    complete = len(lands) == tiles
    if drain or not complete:                                     # the last copy into each stage; those before have been used up
        end_copy = max([end_copy] + lands[-stages:])
    end_roles = give_up if None in used else max([u for u in used if u is not None])
    end = max(end_copy, end_roles)
    return sum(at > end for at in lands)


def test_no_copy_is_in_flight_when_the_block_ends():
    r = random.Random(2)
    plans = [(r.randint(1, 20), r.choice([2, 3, 5]), seed) for seed in range(4000)]
    assert all(end_of_block(n, k, True, seed) == 0 for n, k, seed in plans)
    assert any(end_of_block(n, k, False, seed) for n, k, seed in plans)
