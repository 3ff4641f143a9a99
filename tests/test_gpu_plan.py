"""ppd_paged_plan against the rule, one sequence after the other."""
import random

import pytest
import torch

from paper_2307_05908_amd import binding

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


def rule(pages, ring, counters, held, kept, wanted, page, n_rows):
    pages, ring, was = [list(r) for r in pages], list(ring), list(ring)
    n_pages, wide = len(ring), len(pages[0])
    head, tail = counters
    free = min(max(tail - head, 0), n_pages)
    asked = needed = taken = given = 0
    start, lens, granted, rows = [0], [], [], []
    for s in range(len(held)):
        h = min(max(held[s], 0), wide * page)
        k = h if kept is None else min(max(kept[s], 0), h)
        w = max(wanted[s], 0)
        have = -(-h // page)
        if k + w > wide * page:
            w = 0
        asked += w
        if asked > n_rows:
            w = 0
        need = max(0, -(-(k + w) // page) - have)
        needed += need
        if need and needed > free:
            w = 0
        want = -(-(k + w) // page)
        for j in range(have, want):
            pages[s][j] = was[(head + taken) % n_pages]
            taken += 1
        for j in range(want, have):
            if 0 <= pages[s][j] < n_pages and given < n_pages - free:
                ring[(tail + given) % n_pages] = pages[s][j]
                given += 1
        start.append(start[-1] + w)
        lens.append(k + w)
        granted.append(w)
        for p in range(k, k + w):
            at = pages[s][p // page]
            rows.append((s, p, at * page + p % page if 0 <= at < n_pages else -1))
    rows += [(-1, -1, -1)] * (n_rows - len(rows))
    return dict(pages=pages, ring=ring, counters=[head + taken, tail + given], q_start=start, kv_len=lens, granted=granted,
                row_seq=[r[0] for r in rows], positions=[r[1] for r in rows], slots=[r[2] for r in rows])


class Pool:
    """Conversations with their pages; `free` pages beside those in use, the ring begun anywhere."""

    def __init__(self, held, page, wide, free, seed=0, head=0):
        rng = random.Random(seed)
        need = [-(-h // page) for h in held]
        self.n_pages = max(1, sum(need) + free)
        order = list(range(self.n_pages))
        rng.shuffle(order)
        self.pages = [[-1] * wide for _ in held]
        for s, m in enumerate(need):
            for j in range(m):
                self.pages[s][j] = order.pop()
        self.ring = [-7] * self.n_pages
        for i, p in enumerate(order):
            self.ring[(head + i) % self.n_pages] = p
        self.counters, self.held, self.page = [head, head + len(order)], list(held), page


def dev(x, dt=torch.int32):
    return None if x is None else torch.tensor(x, dtype=dt, device="cuda")


def check(pool, wanted, n_rows, kept=None, in_place=False, want_rows=True):
    want = rule(pool.pages, pool.ring, pool.counters, pool.held, kept, wanted, pool.page, n_rows)
    pages, ring, counters, held = dev(pool.pages), dev(pool.ring), dev(pool.counters, torch.int64), dev(pool.held)
    more = dict(kv_len=held, counters_out=counters) if in_place else {}
    got = binding.ppd_paged_plan(pages, ring, counters, held, dev(wanted), pool.page, n_rows, kept=dev(kept), want_rows=want_rows, **more)
    torch.cuda.synchronize()
    if in_place:
        assert got.kv_len is held and got.counters is counters
    for name, x in dict(got._asdict(), pages=pages, ring=ring).items():
        if x is None:
            assert not want_rows and name in ("row_seq", "positions", "slots")
        else:
            x = x.tolist()
            assert x == want[name], (name, [(i, a, b) for i, (a, b) in enumerate(zip(x, want[name])) if a != b][:5])
    pool.pages, pool.ring, pool.counters, pool.held = want["pages"], want["ring"], want["counters"], want["kv_len"]
    return want


@pytest.mark.parametrize("page", [1, 3, 16, 64])
@pytest.mark.parametrize("seqs", [1, 2, 7, 64, 65, 255, 256, 257, 1000, 4096])
def test_steps_of_a_server(page, seqs):
    """Sequences begin, grow, lose drafts, end and begin again, step after step, with pages enough and with too few."""
    rng = random.Random(100 * seqs + page)
    wide = max(2, 60 // page)
    pool = Pool([rng.choice([0, 0, 1, page, rng.randint(1, wide * page // 2)]) for _ in range(seqs)], page, wide, seqs * rng.choice([1, 3]), seed=seqs, head=rng.randint(0, 10 ** 12))
    for step in range(6 if seqs < 4096 else 3):
        kept, wanted = [], []
        for h in pool.held:
            x = rng.random()
            kept.append(0 if x < 0.15 else max(0, h - rng.randint(0, 4)))
            wanted.append(rng.choice([0, 0, rng.randint(1, wide * page)]) if x < 0.15 else rng.randint(0, 6) if h else rng.randint(0, wide * page + 1))
        total = sum(wanted)
        check(pool, wanted, rng.choice([total, total + 5, total // 2, max(1, total // 10)]), kept, in_place=step % 2 == 1, want_rows=step != 4)
        used = [p for s, h in zip(pool.pages, pool.held) for p in s[:-(-h // page)]]
        head, tail = pool.counters
        free = [pool.ring[i % pool.n_pages] for i in range(head, tail)]
        assert sorted(used + free) == list(range(pool.n_pages))                # no page is lost, none has two owners


def test_one_token_and_none():
    check(Pool([0], 16, 4, 3), [1], 1)
    check(Pool([0], 16, 4, 3), [0], 4)
    check(Pool([16], 16, 4, 1), [1], 1)
    check(Pool([16], 16, 4, 0), [1], 1)                        # there is no page for it
    check(Pool([15], 16, 4, 0), [1], 1)                        # it needs none
    check(Pool([64], 16, 4, 2), [1], 1)                        # the table is full
    check(Pool([5, 9], 16, 4, 2), [3, 4], 0)                   # no rows at all
    check(Pool([5, 90], 16, 6, 0), [0, 0], 0, kept=[0, 3])     # ends without beginnings
    check(Pool([33], 16, 4, 2), [30], 30, kept=[2])            # lost positions' pages are used again


def test_pages_go_to_sequences_in_their_order():
    pool = Pool([0, 0, 15, 0, 0], 16, 8, 5)
    want = check(pool, [40, 40, 1, 16, 17], 200)               # 3 pages, 3 more than there are, none needed, 1 behind, 2 behind
    assert want["granted"] == [40, 0, 1, 0, 0]
    want = check(Pool([0, 0, 0, 0], 4, 8, 100), [5, 40, 9, 3], 10)
    assert want["granted"] == [5, 0, 0, 0]                     # 40 is more than a row of the table has; 5 + 9 + ... are too many rows
    want = check(Pool([0, 0, 0, 0], 4, 8, 100), [5, 4, 9, 0], 10)
    assert want["granted"] == [5, 4, 0, 0]


def test_lengths_outside_their_range():
    check(Pool([20, 30, 40, 0], 16, 3, 9), [-5, 2 ** 30, 1, MOST], 100, kept=[50, -2, MOST, -MOST])
    pool = Pool([20, 30, 40, 0], 16, 3, 9)
    pool.held = [MOST, -1, 48, -MOST]                          # behind the table; before the beginning
    for j in range(3):
        pool.pages[0][j] = 4
    check(pool, [1, 1, 0, 4], 100, kept=[0, 0, 1, 0])
    check(Pool([0] * 300, 1, 4, 9), [MOST] * 299 + [3], 50)


def test_entries_and_counters_that_no_call_leaves():
    pool = Pool([100, 100], 16, 8, 4)
    pool.pages[0][1], pool.pages[0][2], pool.pages[1][6], pool.pages[1][0] = -1, pool.n_pages, MOST, -MOST
    check(pool, [0, 3], 9, kept=[0, 0])                        # what is no page is given back by no one
    for counters in ([5, 3], [0, MOST], [-3, 2], [-2 ** 63, 2 ** 63 - 1], [2 ** 63 - 1, -2 ** 63]):
        pool = Pool([40, 20, 0], 16, 8, 4)
        head, tail = counters
        wrapped = (tail - head + 2 ** 63) % 2 ** 64 - 2 ** 63
        free = min(max(wrapped, 0), pool.n_pages)
        ring, pages = dev(pool.ring), dev(pool.pages)
        around = torch.full((pool.n_pages + 2000,), -9, dtype=torch.int32, device="cuda")
        around[1000:1000 + pool.n_pages] = ring
        got = binding.ppd_paged_plan(pages, around[1000:1000 + pool.n_pages], dev(counters, torch.int64), dev(pool.held), dev([1, 20, 5]), 16, 40, kept=dev([0, 20, 0]))
        torch.cuda.synchronize()
        assert (around[:1000] == -9).all() and (around[1000 + pool.n_pages:] == -9).all()
        assert got.granted.tolist() == [1, 20 if free >= 1 else 0, 5 if free >= 2 else 0]


def test_many_rows():
    pool = Pool([100, 0, 3000, 0, 17], 16, 4000, 9000, head=77)
    check(pool, [5, 30000, 2, 61000, 1], 91008, kept=[97, 0, 2999, 0, 17])
    check(pool, [0, 0, 70000, 0, 0], 70000, kept=[0] * 5)


def test_the_largest_pages():
    """2^30 places in a row of the table, slots beyond 32 bits."""
    page = 2 ** 20
    pool = Pool([2 ** 30 - 5, 3 * page, 0, 2 ** 30], page, 1024, 2000)
    assert pool.n_pages * page > 2 ** 31
    check(pool, [5, 4, 30000, 1], 40000, kept=None)
    check(pool, [0, 2 ** 30 - 3 * page - 4, 2, 0], 40000)              # (more than the rows)
    check(pool, [6, 1, 0, 2 ** 30], 40000, kept=[0, page, 30000, 0])
    check(Pool([2 ** 30, 0], 2 ** 30, 1, 3), [1, 4], 10, kept=[2 ** 30 - 1, 0])


def test_tables_wider_than_what_is_used():
    pool = Pool([20, 30, 40], 16, 6, 9)
    whole = torch.full((5, 50), 77, dtype=torch.int32, device="cuda")
    whole[1:4, 3:9] = dev(pool.pages)
    want = rule(pool.pages, pool.ring, pool.counters, pool.held, None, [20, 1, 33], 16, 60)
    got = binding.ppd_paged_plan(whole[1:4, 3:9], dev(pool.ring), dev(pool.counters, torch.int64), dev(pool.held), dev([20, 1, 33]), 16, 60)
    assert got.slots.tolist() == want["slots"] and whole[1:4, 3:9].tolist() == want["pages"]
    whole[1:4, 3:9] = 77
    assert (whole == 77).all()


def test_streams_and_replays():
    """A captured step in place: each replay goes on from where the one before has left it."""
    pool = Pool([20, 300, 0, 40], 16, 40, 60)
    pages, ring, counters, held = dev(pool.pages), dev(pool.ring), dev(pool.counters, torch.int64), dev(pool.held)
    kept, wanted = dev(pool.held), dev([1, 1, 1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    copies = pages.clone(), ring.clone()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.ppd_paged_plan(*copies, counters, held, wanted, 16, 60, kept=kept, stream=side)
    side.synchronize()
    assert got.slots.tolist() == rule(pool.pages, pool.ring, pool.counters, pool.held, None, [1] * 4, 16, 60)["slots"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.ppd_paged_plan(pages, ring, counters, held, wanted, 16, 60, kept=kept, kv_len=held, counters_out=counters)
    for step, (k, w) in enumerate([([20, 300, 0, 40], [1, 4, 50, 0]), ([21, 301, 48, 0], [2, 2, 2, 9]), ([0, 303, 50, 9], [0, 0, 1, 1]), ([0, 0, 0, 0], [60, 0, 0, 0])]):
        kept.copy_(torch.tensor(k)); wanted.copy_(torch.tensor(w))
        want = rule(pool.pages, pool.ring, pool.counters, pool.held, k, w, 16, 60)
        graph.replay()
        torch.cuda.synchronize()
        for name, x in dict(got._asdict(), pages=pages, ring=ring).items():
            assert x.tolist() == want[name], (step, name)
        pool.pages, pool.ring, pool.counters, pool.held = want["pages"], want["ring"], want["counters"], want["kv_len"]
