"""The arithmetic by which the many-row cache attention's loading warp knows which copies may still be on their way when it ends."""
import random


def waited_for(asked, ring, lanes):
    """Units whose barrier is waited for: the last three of each lane, but for those whose place has been given to a later unit."""
    units = set()
    for lane in range(lanes):
        next_ = asked[(lane + ring) % lanes]
        for back in (1, 2, 3):
            if back <= asked[lane]:
                x = lane + (asked[lane] - back) * lanes
                if (x + ring) // lanes >= next_:
                    units.add(x)
    return units


def test_the_last_copies_are_waited_for_and_no_superseded_one():
    """Lanes ask for units lane, lane + 8, ... in turn; a warp that gives up leaves some of its lanes a unit behind the others."""
    rng, ring, lanes = random.Random(1), 14, 8
    for steps in list(range(0, 9)) + [rng.randrange(9, 500) for _ in range(200)]:
        for _ in range(20):
            asked = [steps + (rng.random() < 0.5) for _ in range(lanes)] if rng.random() < 0.7 else [steps] * lanes
            units = {lane + i * lanes for lane in range(lanes) for i in range(asked[lane])}
            latest = {}                                                   # of each place of the ring
            for u in sorted(units):
                latest[u % ring] = u
            waited = waited_for(asked, ring, lanes)
            assert waited <= set(latest.values())                         # (a superseded unit's phase has passed twice: it would never come)
            # a place is only filled again once its last copy has landed, so the latest ones are all that can be on their way
            assert waited == set(latest.values())
