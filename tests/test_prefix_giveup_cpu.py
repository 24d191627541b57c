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
