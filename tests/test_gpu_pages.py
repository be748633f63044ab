"""The pages of a step of serving, against the definition request by request (GPU): whole numbers, equal."""
import random

import pytest
import torch

from layer_util import DEV
from paper_1503_05032_amd import binding as B

pytestmark = pytest.mark.gpu


def step(fresh, length, table, pool, state, page, tokens):
    """The definition, on the host."""
    width, ring = len(table[0]) if table else 0, len(pool)
    table, pool = [list(r) for r in table], list(pool)
    first, count = (state[0] % ring if ring else 0), min(max(state[1], 0), ring)
    free = [pool[(first + i) % ring] for i in range(count)]
    asked = taken = back = 0
    offset, position, slot, length_out = [0], [], [], []
    for r, (new, have) in enumerate(zip(fresh, length)):
        have = min(max(have, 0), width * page)
        held = -(-have // page)
        offset.append(min(offset[-1] + max(new, 0), tokens))
        if new < 0:
            for p in table[r][:held]:
                if count + back < ring:
                    pool[(first + count + back) % ring] = p
                    back += 1
            length_out.append(0)
            continue
        want = -(-(have + new) // page)
        ok = want <= width
        if ok:
            need = want - held
            asked += need
            ok = need == 0 or asked <= count
            if ok:
                table[r][held:want] = free[asked - need:asked]
                taken += need
        length_out.append(have + new if ok else have)
        room = tokens - len(slot)
        at = range(have, have + min(new, room))
        position += at
        for i in at:
            p = table[r][i // page] if ok else -1
            slot.append(p * page + i % page if 0 <= p <= (2 ** 31 - 1) // page else -1)
    position += [0] * (tokens - len(position))
    slot += [-1] * (tokens - len(slot))
    return offset, position, slot, length_out, [(first + taken) % ring if ring else 0, count - taken + back], table, pool


def check(fresh, length, table, pool, state, page, tokens):
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    n, width = len(fresh), len(table[0]) if table else 0
    f, le, po, st = ints(fresh), ints(length), ints(pool), ints(state)
    wide = torch.full((n, width + 3), -7, dtype=torch.int32, device=DEV)
    ta = wide[:, :width]
    if n and width:
        ta.copy_(ints(table))
    out = [torch.full((m,), -99, dtype=torch.int32, device=DEV) for m in (n + 1, tokens + 1, tokens, n, 2)]
    offset, position, slot, length_out, state_out = out
    want = step(fresh, length, table, pool, state, page, tokens)
    for _ in range(2):                                   # the same state gives the same again
        B.csr5_pages(f, le, ta, po, st, page, offset, position, slot, length_out, state_out)
        got = [t.tolist() for t in (offset, position[:tokens], slot, length_out, state_out, ta, po)]
        for name, a, b in zip(("offset", "position", "slot", "length_out", "state_out", "table", "pool"), got, want):
            assert a == list(b), (name, [(i, x, y) for i, (x, y) in enumerate(zip(a, b)) if x != y][:5])
    assert int(position[tokens]) == -99 and bool((wide[:, width:] == -7).all()) and f.tolist() == list(fresh) and le.tolist() == list(length)


def serving(rng, n, page, most_new, cached, over, slack, spare=2):
    fresh = [-1 if rng.random() < over else rng.choice([0, 1, rng.randint(0, most_new)]) for _ in range(n)]
    length = [rng.choice([0, cached, rng.randint(0, cached)]) for _ in range(n)]
    held = [-(-x // page) for x in length]
    need = sum(max(0, -(-(x + max(f, 0)) // page) - h) for x, f, h in zip(length, fresh, held))
    width = max(-(-(cached + most_new) // page) + rng.randint(-1, 2), max(held + [1]))
    left = int(need * slack) + spare
    order = list(range(sum(held) + left))
    rng.shuffle(order)
    table = [[order.pop() for _ in range(h)] + [-1] * (width - h) for h in held]
    first, ring = rng.randint(0, sum(held) + left), sum(held) + left
    pool = [-5] * ring
    for i, p in enumerate(order):
        pool[(first + i) % ring] = p
    return fresh, length, table, pool, [first % ring, left], page, sum(max(f, 0) for f in fresh) + rng.choice([0, 0, 9])


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n,page,most_new,cached", [(1, 16, 1, 40), (48, 16, 1, 400), (300, 1, 5, 9), (700, 32, 90, 900), (1023, 64, 3, 200), (1500, 16, 20, 100), (40, 256, 4000, 3000)])
def test_steps(n, page, most_new, cached, seed):
    rng = random.Random(1000 * n + seed)
    check(*serving(rng, n, page, most_new, cached, over=(0.0, 0.1, 0.5)[seed % 3], slack=(0.3, 0.9, 1.0, 2.0)[seed % 4]))


def test_edges():
    check([], [], [], [3, 4], [1, 1], 16, 5)                                                  # no requests
    check([0, 0], [0, 5], [[-1], [2]], [], [0, 0], 16, 0)                                     # no tokens, no ring
    check([5], [30], [[1, 2]], [9], [0, 1], 16, 8)                                            # passes its table
    check([5, 2, 1], [30, 16, 3], [[1, 2], [4, -1], [5, -1]], [9], [0, 1], 16, 8)             # ... which takes nothing from the others
    check([17, 1, 16, 0], [0, 15, 0, 7], [[-1, -1], [3, -1], [-1, -1], [6, -1]], [9, 8], [1, 2], 16, 40)   # one that needs pages that are not there, and those after it
    check([-1, -1], [32, 33], [[1, 2, -1], [3, 4, 5]], [7, 0, 0, 0, 0, 0], [5, 1], 16, 3)     # all over, around the ring's end
    check([-1], [48], [[1, 2, 3]], [7, 0], [0, 1], 16, 0)                                     # more pages come back than the ring has places for
    check([3], [20], [[1, 2]], [7], [0, 1], 16, 2)                                            # more new tokens than room
    check([4, 4], [-9, 10 ** 9], [[-1, -1], [1, 2]], [3, 4, 5], [-1, 99], 16, 8)              # lengths and states of none
    check([4], [0], [[-1]], [2 ** 27], [0, 1], 16, 4)                                         # a page past all slots
    check([4], [0], [[-1]], [-3], [0, 1], 16, 4)
    check([2 ** 31 - 1] * 3, [1, 1, 1], [[1], [2], [3]], [4], [0, 1], 16, 3000)               # sums past 32 bits


def test_replayed_while_requests_go_on():
    """A captured step, its state, lengths and tables carried on from replay to replay: prompts, single tokens, the end."""
    page, n, width, ring = 16, 3, 8, 32
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    fresh, length, state = ints([20, 5, 0]), ints([0, 0, 0]), ints([0, ring])
    table, pool = torch.full((n, width), -1, dtype=torch.int32, device=DEV), torch.arange(ring, dtype=torch.int32, device=DEV)
    offset, position, slot, length_out, state_out = (torch.empty(m, dtype=torch.int32, device=DEV) for m in (n + 1, 32, 32, n, 2))
    run = lambda: B.csr5_pages(fresh, length, table, pool, state, page, offset, position, slot, length_out, state_out)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    host = dict(length=[0] * n, state=[0, ring], table=[[-1] * width for _ in range(n)], pool=list(range(ring)))
    for news in ([20, 5, 0], [1, 1, 30], [1, -1, 1], [1, 14, 1], [-1, 1, 15], [12, 1, -1]):
        fresh.copy_(ints(news))
        want = step(news, host["length"], host["table"], host["pool"], host["state"], page, 32)
        graph.replay()
        torch.cuda.synchronize()
        assert [t.tolist() for t in (offset, position, slot, length_out, state_out, table, pool)] == [list(w) for w in want]
        length.copy_(length_out), state.copy_(state_out)
        host = dict(length=want[3], state=want[4], table=want[5], pool=want[6])


def test_arrays_side_by_side():
    """All arrays of a step in one, without a word between them, and one of them between the rows of the table."""
    rng = random.Random(77)
    fresh, length, table, pool, state, page, tokens = serving(rng, 5, 16, 40, 90, over=0.2, slack=2.0)
    want = step(fresh, length, table, pool, state, page, tokens)
    n, width = len(fresh), len(table[0])
    sizes = dict(fresh=n, slot=tokens, length=n, offset=n + 1, pool=len(pool), state_out=2, position=tokens, state=2, table=n * (width + n))
    words = torch.full((sum(sizes.values()),), -7, dtype=torch.int32, device=DEV)
    at = dict(zip(sizes, words.split(list(sizes.values()))))
    wide = at["table"].view(n, width + n)
    here = at | dict(table=wide[:, :width], length_out=wide[2, width:])
    for name, values in dict(fresh=fresh, length=length, table=table, pool=pool, state=state).items():
        here[name].copy_(torch.tensor(values, dtype=torch.int32))
    B.csr5_pages(here["fresh"], here["length"], here["table"], here["pool"], here["state"], page, *(here[name] for name in ("offset", "position", "slot", "length_out", "state_out")))
    assert [here[name].tolist() for name in ("offset", "position", "slot", "length_out", "state_out", "table", "pool")] == [list(w) for w in want]
    assert here["fresh"].tolist() == fresh and here["length"].tolist() == length and here["state"].tolist() == state
    assert bool((wide[[0, 1, 3, 4], width:] == -7).all())
