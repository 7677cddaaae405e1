"""Page tables, slots and positions built on the GPU, against the same done on the host one request after the other."""
import pytest
import torch

import paper_2609_35800_gb300 as hg

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def plan(table, cached, new, free, count, size, room):
    """(table, lengths, begin, slots, positions, counts, free) after the call, on lists."""
    table, free = [list(r) for r in table], list(free)
    per, clip = len(table[0]) if table else 0, [max(c, 0) for c in cached]
    pages = lambda t: -(-t // size)  # noqa: E731
    pile = free[:count]
    for r, n in enumerate(new):
        if n < 0:
            pile += table[r][:min(pages(clip[r]), per)]
    want = [0 if n < 0 else pages(c + n) - pages(c) for c, n in zip(clip, new)]
    tokens = sum(max(n, 0) for n in new)
    outgrown = any(n >= 0 and pages(c + n) > per for c, n in zip(clip, new))
    left = len(pile) - sum(want)
    refused = -1 if outgrown else -2 if tokens > room else -left if left < 0 else -3 if left > len(free) else 0
    if refused:
        return (table, list(cached), [0] * (len(new) + 1), [-1] * room, [0] * room,
                [count, refused, 0, max(clip, default=0)], free)
    lengths, begin, slots, positions = [], [0], [], []
    for r, n in enumerate(new):
        if n >= 0:
            for i in range(want[r]):
                table[r][pages(clip[r]) + i] = pile.pop()
            for t in range(clip[r], clip[r] + n):
                slots.append(table[r][t // size] * size + t % size)
                positions.append(t)
        lengths.append(0 if n < 0 else clip[r] + n)
        begin.append(len(slots))
    free[count:left] = pile[count:left] if left > count else []
    return (table, lengths, begin, slots + [-1] * (room - len(slots)), positions + [0] * (room - len(slots)),
            [left, 0, tokens, max(lengths, default=0)], free)


def _run(table, cached, new, free, count, size, room, in_place=False, positions=True):
    n = len(new)
    width = len(table[0]) if table else 0
    t = _ints(table) if table else torch.empty((0, width), dtype=torch.int32, device="cuda")
    c, f = _ints(cached), _ints(free)
    guard = lambda m: torch.full((m + 2,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
    begin, slots, pos = guard(n + 1), guard(room), guard(room)
    counts = _ints([count, 77, 77, 77])
    lengths = c if in_place else guard(n)[1:1 + n]
    hg.hg_pages_plan(t, c, _ints(new), f, counts[:1] if in_place else _ints([count]), size, lengths, begin[:n + 1],
                     slots[:room], pos[:room] if positions else None, counts)
    assert begin[n + 1:].tolist() == [77, 77] and slots[room:].tolist() == [77, 77]
    assert pos.tolist() == pos[:room].tolist() + [77, 77]
    return (t.tolist() if table else [], lengths.tolist(), begin[:n + 1].tolist(), slots[:room].tolist(),
            pos[:room].tolist() if positions else None, counts.tolist(), f.tolist())


def _case(seed, batch, size, longest, ending, spare=3, context=100, columns=2):
    g = torch.Generator()
    g.manual_seed(seed)
    ints = lambda hi, n: [int(x) for x in torch.randint(0, hi + 1, (n,), generator=g)]  # noqa: E731
    cached, new = ints(context, batch), ints(longest, batch)
    ends = [x == 0 for x in ints(ending, batch)] if ending else [False] * batch
    width = max((-(-(c + n) // size) for c, n in zip(cached, new)), default=0) + columns
    held = [-(-c // size) for c in cached]
    need = sum(-(-(c + n) // size) for c, n, e in zip(cached, new, ends) if not e) - sum(h for h, e in zip(held, ends) if not e)
    back = sum(h for h, e in zip(held, ends) if e)
    count = max(0, need - back) + spare
    ids = [int(x) for x in torch.randperm(sum(held) + count, generator=g)]
    table = [[-9] * width for _ in range(batch)]
    for r, h in enumerate(held):
        for i in range(h):
            table[r][i] = ids.pop()
    free = ids + [-5] * sum(held)
    return table, cached, [-1 - r % 3 if e else n for r, (n, e) in enumerate(zip(new, ends))], free, len(ids), size


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,size,longest,ending", [(1, 16, 1, 0), (1, 16, 5000, 0), (7, 32, 60, 3), (33, 64, 1, 0),
                                                      (64, 16, 1, 5), (1000, 16, 40, 4), (1025, 128, 300, 2), (3, 256, 0, 0),
                                                      (2500, 16, 3, 1), (50, 16, 90, 1)])
def test_plan(batch, size, longest, ending, in_place):
    args = _case(batch + longest, batch, size, longest, ending)
    for room in (sum(max(n, 0) for n in args[2]), sum(max(n, 0) for n in args[2]) + 1003):
        want = plan(*args, room)
        assert want[5][1] == 0
        assert _run(*args, room, in_place=in_place) == want
    got = _run(*args, room, positions=False)
    assert got[:4] == want[:4] and got[5:] == want[5:]


def test_plan_of_nothing():
    assert _run([], [], [], [3, 4], 2, 16, 5) == plan([], [], [], [3, 4], 2, 16, 5)
    args = ([[1, 2], [3, 4]], [0, 16], [0, 0], [], 0, 16)
    assert _run(*args, 0) == plan(*args, 0)
    args = ([[1, 2]] * 3, [-4, -2 ** 31, 3], [2, -1, -2 ** 31], [9, 8, 7], 2, 16)  # below 0: no token; ended
    assert _run(*args, 4) == plan(*args, 4)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("change,why", [(dict(count=0), 4), (dict(count=3), 1), (dict(new=[49, 1, 2]), -1),
                                       (dict(cached=[500, 5, 20]), -1), (dict(room=4), -2), (dict(count=-7), 4),
                                       (dict(new=[2 ** 31 - 1, 2 ** 31 - 1, 3]), -1),
                                       (dict(new=[0, 0, -1], count=8), -3)])
def test_refused_plans_change_nothing(change, why, in_place):
    d = dict(table=[[1, 2, 3], [4, 5, 6], [7, 8, 9]], cached=[0, 16, 31], new=[1, 33, 2], free=[10, 11, 12, 13, 14, 15, 16, 17],
             count=8, room=64)
    d["new"] = [17, 16, 17]
    d.update(change)
    args = (d["table"], d["cached"], d["new"], d["free"], max(d["count"], 0), 16)
    want = plan(*args, d["room"])
    assert want[5][1] == why
    got = _run(d["table"], d["cached"], d["new"], d["free"], d["count"], 16, d["room"], in_place=in_place)
    assert got == want


def test_more_tokens_than_32_bits_are_refused():
    table = [[0] * 8] * 4
    got = _run(table, [0] * 4, [2 ** 31 - 1] * 4, [1, 2], 2, 16, 10)
    assert got[5] == [2, -1, 0, 0]


def test_requests_come_and_go():
    """Many calls on the same arrays: no page is ever in two places, and none is lost."""
    g = torch.Generator()
    g.manual_seed(1)
    size, n, pool = 16, 40, 300
    table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
    free, count = torch.randperm(pool, generator=g).to(torch.int32).cuda(), _ints([pool, 0, 0, 0])
    lens, begin, slots = _ints([0] * n), _ints([0] * (n + 1)), _ints([0] * 4000)
    refused = 0
    for _ in range(60):
        new = torch.randint(0, 60, (n,), generator=g)
        new[torch.rand(n, generator=g) < 0.2] = -1
        before = (table.tolist(), lens.tolist(), new.tolist(), free.tolist(), int(count[0]))
        hg.hg_pages_plan(table, lens, new.to(torch.int32).cuda(), free, count[:1], size, lens, begin, slots, None, count)
        want = plan(*before, size, 4000)
        assert (table.tolist(), lens.tolist(), begin.tolist(), slots.tolist(), count.tolist(), free.tolist()) == (
            want[0], want[1], want[2], want[3], want[5], want[6])
        refused += want[5][1] != 0
        held = [p for r, t in enumerate(lens.tolist()) for p in table[r, :-(-t // size)].tolist()]
        assert sorted(held + free[:int(count[0])].tolist()) == list(range(pool))
        if want[5][1] != 0:  # everybody leaves
            hg.hg_pages_plan(table, lens, _ints([-1] * n), free, count[:1], size, lens, begin, slots, None, count)
            assert int(count[0]) == pool
    assert refused > 2


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,size,longest,ending,context", [(1, 64, 300000, 0, 50), (900, 16, 700, 6, 300), (16384, 16, 3, 9, 40),
                                                              (5, 256, 9000, 2, 3000), (16384, 32, 1, 2, 5)])
def test_large_plans(batch, size, longest, ending, context, in_place):
    """More tokens than one CTA takes, and as many requests as a call may have."""
    args = _case(batch + longest, batch, size, longest, ending, context=context)
    room = sum(max(n, 0) for n in args[2])
    want = plan(*args, room + 10001)
    assert want[5][1] == 0
    assert _run(*args, room + 10001, in_place=in_place) == want
    if room > 0:  # refused: no token is placed
        assert _run(*args, room - 1, in_place=in_place) == plan(*args, room - 1)
    short = args[:4] + (max(args[4] - 5, 0), size)  # fewer free pages than needed
    assert _run(*short, room, in_place=in_place) == plan(*short, room)
