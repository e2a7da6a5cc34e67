"""Tables of a step against a plain restatement, list by list."""
import random

import pytest
import torch

from paper_2506_07533_b200 import binding as mq

pytestmark = pytest.mark.gpu


class Host:
    """The same in Python lists."""

    def __init__(self, past, table, ring, state, page):
        self.past, self.table, self.ring, self.state, self.page = past, table, ring, state, page

    def plan(self, n_new, rows):
        pages = lambda n: (n + self.page - 1) // self.page  # noqa: E731
        total = [max(p + n, 0) for p, n in zip(self.past, n_new)]
        grow = [max(t - p, 0) for t, p in zip(total, self.past)]
        take = [max(pages(t) - pages(p), 0) for t, p in zip(total, self.past)]
        first, free = self.state
        n = len(self.ring)
        width = len(self.table[0]) if self.table else 0
        code = [0, 0, 0]
        bad = [b for b in range(len(total)) if not (0 <= self.past[b] <= width * self.page and total[b] <= width * self.page)]
        if bad:
            code = [mq.ERR_CORRUPT_TABLE, bad[0], -1]
        elif sum(grow) > rows:
            code = [mq.ERR_INVALID_ARG, -1, sum(grow)]
        elif sum(take) > free:
            code = [mq.ERR_POOL_FULL, sum(take), free]
        if code[0]:
            return self.past, [0] * (len(total) + 1), [-1] * rows, [-1] * rows, code
        given = []
        for b in range(len(total)):
            given += self.table[b][pages(total[b]):pages(self.past[b])]
        at = 0
        for b in range(len(total)):
            for e in range(pages(self.past[b]), pages(total[b])):
                self.table[b][e] = self.ring[(first + at) % n]
                at += 1
        for i, p in enumerate(given):
            self.ring[(first + free + i) % n] = p
        self.state = [(first + at) % n if n else 0, free - at + len(given)]
        cu, pos, seq = [0], [], []
        for b in range(len(total)):
            cu.append(cu[-1] + grow[b])
            pos += range(self.past[b], self.past[b] + grow[b])
            seq += [b] * grow[b]
        pad = [-1] * (rows - len(pos))
        self.past = total
        return total, cu, pos + pad, seq + pad, code


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def both(rng, batch, page, width, n_pages, past, n_new, rows, *, four=False, apart=False, first=None, spare=None):
    used = [(p + page - 1) // page for p in past]
    order = list(range(n_pages))
    rng.shuffle(order)
    table, at = [], 0
    for u in used:
        table.append([order[at + i] if i < u else -5 for i in range(width)])
        at += u
    first = rng.randrange(n_pages) if first is None else first
    free = n_pages - at if spare is None else spare
    ring = [-9] * n_pages
    for i in range(free):
        ring[(first + i) % n_pages] = order[at + i]
    pages = torch.empty(n_pages, 1, page * 160, dtype=torch.uint8, device="cuda") if four else torch.empty(n_pages, 1, page, 128, dtype=torch.bfloat16, device="cuda")
    bind = (lambda *a: mq.moqae_paged4_bind(*a, torch.float16)) if four else (lambda p, *a: mq.moqae_paged_bind(p, p, *a))
    cache = bind(pages, ints(table).view(batch, width), ints([77] * batch if apart else past))
    pool = mq.PagePool(ints(ring), ints([0, 0, 0, 0] if apart else [first, free, 0, 0]))
    cu, pos, seq = ints([5] * (batch + 1)), ints([5] * rows), ints([5] * rows)
    kw = dict(past_len=ints(past), pool_state=ints([first, free, 0, 0])) if apart else {}
    mq.moqae_paged_plan(cache, pool, ints(n_new), cu, pos, seq, **kw)
    host = Host(list(past), table, ring, [first, free], page)
    total, hcu, hpos, hseq, code = host.plan(n_new, rows)
    assert cache.status.tolist()[:3] == code
    assert cache.kv_len.tolist() == total and cu.tolist() == hcu
    assert pos.tolist() == hpos and seq.tolist() == hseq
    assert cache.block_table.tolist() == host.table and pool.ring.tolist() == host.ring
    assert pool.state.tolist() == host.state + [0, 0]
    return cache, pool, host


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(seed):
    rng = random.Random(seed)
    batch = rng.choice((1, 2, 5, 61, 255, 256, 257, 600))
    page = rng.choice((16, 32, 64, 128, 256))
    width = rng.choice((3, 20))
    most = width * page
    past = [rng.choice((0, 1, page - 1, page, page + 1, rng.randint(0, most))) for _ in range(batch)]
    n_new = [rng.choice((1, 1, 1, 0, -1, -p, -(1 << 31), rng.randint(0, most - p), most - p)) if p < most else rng.choice((0, -1, -p)) for p in past]
    n_new = [min(n, most - p) for n, p in zip(n_new, past)]
    rows = max(1, sum(max(0, n) for n in n_new) + rng.choice((0, 1, 100)))
    used = sum((p + page - 1) // page for p in past)
    n_pages = used + sum((max(0, p + n) + page - 1) // page for n, p in zip(n_new, past)) + rng.choice((0, 5)) + 1
    cache, pool, host = both(rng, batch, page, width, n_pages, past, n_new, rows, four=seed % 2 == 0, apart=seed % 3 == 0)
    # and on from there, in place
    for _ in range(4):
        cache.status.zero_()
        n_new = [rng.choice((0, 1, 1, -1, -p, page)) for p in host.past]
        n_new = [min(n, most - p) for n, p in zip(n_new, host.past)]
        rows = max(1, sum(max(0, n) for n in n_new))
        cu, pos, seq = ints([5] * (batch + 1)), ints([5] * rows), ints([5] * rows)
        mq.moqae_paged_plan(cache, pool, ints(n_new), cu, pos, seq)
        total, hcu, hpos, hseq, code = host.plan(n_new, rows)
        assert cache.status.tolist()[:3] == code and cache.kv_len.tolist() == total and cu.tolist() == hcu
        assert pos.tolist() == hpos and seq.tolist() == hseq and pool.state.tolist() == host.state + [0, 0]
        assert cache.block_table.tolist() == host.table and pool.ring.tolist() == host.ring


def test_many_rows_and_many_sequences():
    rng = random.Random(99)
    both(rng, 3, 16, 2100, 4300, [0, 100, 0], [33000, 1, 20000], 53100)              # several CTAs, long rows
    both(rng, 3000, 16, 2, 6100, [rng.randint(0, 31) for _ in range(3000)], [1] * 3000, 3050)
    both(rng, 1, 256, 1, 1, [0], [256], 256, first=0)


def test_refusals_on_the_device():
    rng = random.Random(5)
    common = dict(batch=3, page=16, width=4)
    both(rng, n_pages=12, past=[10, 0, 20], n_new=[40, 64, 1], rows=200, spare=5, **common)      # 7 pages wanted
    both(rng, n_pages=12, past=[10, 0, 20], n_new=[40, 64, 1], rows=104, **common)               # rows for 104 of 105
    both(rng, n_pages=12, past=[10, 0, 20], n_new=[1, 65, 1], rows=100, **common)                # longer than its row of the table
    both(rng, n_pages=12, past=[10, 65, 20], n_new=[1, -1, 1], rows=100, spare=0, **common)
    both(rng, n_pages=12, past=[10, 0, 20], n_new=[1, (1 << 31) - 1, 1], rows=100, **common)


def test_sums_past_32_bits_are_refused():
    """Sequences that each bring 2^29 tokens: their sums, and those of their pages, must not wrap into something that fits."""
    batch, page, width = 70, 16, 1 << 25
    cache = mq.moqae_paged4_bind(torch.empty(9, 1, 2560, dtype=torch.uint8, device="cuda"), torch.empty(batch, 0, dtype=torch.int32, device="cuda"),
                                 ints([0] * batch), torch.float16)
    table = torch.zeros(4, dtype=torch.int32, device="cuda")          # never read or written: the batch is refused
    pool = mq.make_page_pool(9)
    cu, pos, seq = ints([5] * (batch + 1)), ints([5] * 8), ints([5] * 8)
    L, C = mq.lib(), mq.C
    view = mq.MoqaePagePool(pool.ring.data_ptr(), pool.state.data_ptr(), 9)
    for grow in (1 << 29, 1 << 27):
        cache.status.zero_()
        new = ints([grow] * batch)
        assert L.moqae_paged_plan(cache.kv_len.data_ptr(), new.data_ptr(), batch, page, width, table.data_ptr(), cache.kv_len.data_ptr(), C.byref(view), None,
                                  cu.data_ptr(), pos.data_ptr(), seq.data_ptr(), 8, cache.status.data_ptr(),
                                  torch.cuda.current_stream().cuda_stream) == 0
        code, _, tokens, _ = cache.status.tolist()
        assert code == mq.ERR_INVALID_ARG and tokens > 8 and cache.kv_len.tolist() == [0] * batch
        assert cu.tolist() == [0] * (batch + 1) and pos.tolist() == [-1] * 8 and pool.state.tolist() == [0, 9, 0, 0]


def test_a_state_that_cannot_be_and_a_page_that_does_not_exist():
    cache = mq.moqae_paged4_bind(torch.empty(4, 1, 2560, dtype=torch.uint8, device="cuda"), ints([[0, 99]]), ints([20]), torch.float16)
    for state in ([4, 1, 0, 0], [-1, 1, 0, 0], [0, 5, 0, 0], [0, -1, 0, 0], [0, 4, 0, 0]):       # the last: two pages in use, none missing
        pool = mq.PagePool(ints([1, 2, 3, 0]), ints(state))
        cu, pos, seq = ints([5, 5]), ints([5]), ints([5])
        cache.status.zero_()
        mq.moqae_paged_plan(cache, pool, ints([-20]), cu, pos, seq)
        assert cache.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, -1, -1]
        assert cache.kv_len.tolist() == [20] and cu.tolist() == [0, 0] and pos.tolist() == [-1] and seq.tolist() == [-1]
        assert pool.state.tolist() == state and pool.ring.tolist() == [1, 2, 3, 0]
    pool = mq.PagePool(ints([1, 2, 3, 0]), ints([0, 2, 0, 0]))
    cache.status.zero_()
    mq.moqae_paged_plan(cache, pool, ints([-20]), cu, pos, seq)
    assert cache.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, 0, 1]
    assert cache.kv_len.tolist() == [0] and pool.state.tolist() == [0, 4, 0, 0] and pool.ring.tolist() == [1, 2, 0, 99]


def test_an_empty_batch():
    cache = mq.moqae_paged4_bind(torch.empty(4, 1, 2560, dtype=torch.uint8, device="cuda"), ints([]).view(0, 3), ints([]), torch.float16)
    pool, cu, pos, seq = mq.make_page_pool(4), ints([5]), ints([5, 5]), ints([5, 5])
    mq.moqae_paged_plan(cache, pool, ints([]), cu, pos, seq)
    assert cu.tolist() == [0] and pos.tolist() == [-1, -1] and seq.tolist() == [-1, -1] and pool.state.tolist() == [0, 4, 0, 0]
