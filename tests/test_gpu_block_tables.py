"""Steps that bring more than there is room for: what the tables, slots and counts say then, from the header's text."""
import random

import pytest
import torch

from tests.test_gpu_cache import run_tables, sb  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def pages_taken(old, new, free, count, columns, page):
    """{(request, column): page id or -1} of every page that a step takes, request after request from the top of the stack."""
    stack, taken = list(free[:max(0, min(count, len(free)))]), {}
    for b, (o, n) in enumerate(zip(old, new)):
        for j in range(-(-o // page), min(-(-(o + n) // page), columns)):
            taken[b, j] = stack.pop() if stack else -1
    return taken, len(stack)


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("B, longest, share", [(1, 700, 0.0), (1, 700, 0.6), (3, 90, 0.5), (3, 90, 0.01), (300, 40, 0.4), (600, 300, 0.9), (9, 3000, 0.3)])
@pytest.mark.parametrize("short", [0, 4])
def test_pages_behind_the_last_slot_are_entered(sb, page, B, longest, share, short):  # noqa: F811
    """Every page that leaves the stack is in a table, in place of what an earlier request left there: none is lost, and none is read as
    this request's that is another's."""
    rng = random.Random(B * page + longest)
    old = [rng.choice([0, page, page - 1, rng.randrange(3 * page)]) for _ in range(B)]
    new = [rng.randint(0, longest) for _ in range(B)]
    columns = max(1, max(-(-(o + n) // page) for o, n in zip(old, new)))
    table = [[1000000 + b * columns + j for j in range(columns)] for b in range(B)]       # stale ids
    need = sum(-(-(o + n) // page) - -(-o // page) for o, n in zip(old, new))
    free = rng.sample(range(500000), max(1, need - short + 3))
    count = max(0, need - short)
    total = sum(new)
    got_table, cu, kv, slots, _, result = run_tables(sb, old, new, free, count, table, page, int(total * share))
    taken, left = pages_taken(old, new, free, count, columns, page)
    want = [[taken.get((b, j), table[b][j]) for j in range(columns)] for b in range(B)]
    assert got_table == want
    assert result[0] == left and cu[-1] == total and kv == [o + n for o, n in zip(old, new)]
    want_slots = [want[b][p // page] * page + p % page if want[b][p // page] >= 0 else -1 for b, (o, n) in enumerate(zip(old, new)) for p in range(o, o + n)]
    kept = want_slots[:int(total * share)]
    assert slots == kept and result[1] == total - len(kept) + sum(s < 0 for s in kept)


@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("B, longest, share", [(1, 3000, 1.0), (7, 700, 1.0), (7, 700, 0.5), (600, 90, 1.0), (600, 90, 0.7)])
def test_pages_that_are_none_are_counted(sb, page, B, longest, share):  # noqa: F811
    """Negative ids and ids whose slots pass 31 bits, on the stack and in the page that was begun: the result counts every token without a slot."""
    rng = random.Random(B * page + longest)
    most = (2 ** 31 - 1) // page                                          # the largest page whose slots fit
    some = lambda: rng.choice([rng.randrange(most), rng.randrange(most), most, most + 1, 2 ** 31 - 1, -1, -5])  # noqa: E731
    old = [rng.choice([0, page, page - 1, rng.randrange(3 * page)]) for _ in range(B)]
    new = [rng.randint(0, longest) for _ in range(B)]
    columns = max(1, max(-(-(o + n) // page) for o, n in zip(old, new)))
    table = [[some() for _ in range(columns)] for _ in range(B)]
    need = sum(-(-(o + n) // page) - -(-o // page) for o, n in zip(old, new))
    free = [some() for _ in range(max(1, need - 2))]
    total = sum(new)
    got_table, _, _, slots, _, result = run_tables(sb, old, new, free, len(free), table, page, int(total * share))
    taken, left = pages_taken(old, new, free, len(free), columns, page)
    want = [[taken.get((b, j), table[b][j]) for j in range(columns)] for b in range(B)]
    assert got_table == want
    ids = [(want[b][p // page], p % page) for b, (o, n) in enumerate(zip(old, new)) for p in range(o, o + n)][:len(slots)]
    assert slots == [i * page + at if 0 <= i <= most else -1 for i, at in ids]
    assert result == [left, total - len(slots) + sum(s < 0 for s in slots)]
