"""The cache plan from several host threads, with lengths that pass 31 bits, and with outputs that lie in its inputs."""
import threading

import pytest
import torch

from paper_2609_24519_b200 import binding as b
from tests.gpu_util import handle

pytestmark = pytest.mark.gpu


def test_calls_of_several_threads_with_many_and_few_requests():
    """More than 6,143 requests need more shared memory than a launch may have unasked: one thread's limit is no other's."""
    handle()
    wrong = []

    def work(B):
        h, i32 = b.awe_create(0), dict(dtype=torch.int32, device="cuda")
        cached, new, table = torch.arange(B, **i32) % 16, torch.ones(B, **i32), torch.zeros((B, 2), **i32)
        free, slots = torch.arange(B, **i32), torch.empty(B, dtype=torch.int64, device="cuda")
        start, ctx, counts = torch.empty(B + 1, **i32), torch.empty(B, **i32), torch.empty(4, **i32)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        try:
            for _ in range(3000):
                b.awe_kv_plan(h, cached, new, B, 16, free, B, table, 2, 2, slots, None, B, start, ctx, counts, stream=stream)
        except b.AweError as e:
            wrong.append((B, e))
        stream.synchronize()
        if not wrong and counts[1] != B:
            wrong.append((B, counts.tolist()))

    threads = [threading.Thread(target=work, args=(B,)) for B in (16384, 6200, 9000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


MOST = 2 ** 31 - 1


@pytest.mark.parametrize("cached,new", [([MOST, 0, 5], [MOST, 3, 4]), ([5, 0, 7], [2, MOST, 1]), ([MOST] * 40, [MOST] * 40), ([0] * 600, [MOST - 1] * 600),
                                        ([MOST, -MOST - 1], [1, -MOST - 1])])
@pytest.mark.parametrize("page", [16, 256])
def test_lengths_whose_sums_pass_31_bits(cached, new, page):
    """Sums stay at 2^31 - 1; nothing outside the tables is touched, and tokens beyond a table row have no slot."""
    B, width, n_free, most = len(cached), 4, 9, 70
    pool = torch.full((B + 2, width), 5, dtype=torch.int32, device="cuda")  # a row before and one behind the table's
    i32 = dict(dtype=torch.int32, device="cuda")
    d_cached, d_new, free = torch.tensor(cached, **i32), torch.tensor(new, **i32), torch.arange(100, 100 + n_free, **i32)
    slots, positions = torch.empty(most, dtype=torch.int64, device="cuda"), torch.empty(most, **i32)
    start, ctx, counts = torch.empty(B + 1, **i32), torch.empty(B, **i32), torch.empty(4, **i32)
    b.awe_kv_plan(handle(), d_cached, d_new, B, page, free, n_free, pool[1:], width, width, slots, positions, most, start, ctx, counts)
    table = [[5] * width for _ in cached]
    taken = tokens = missing = 0
    want_slots, want_pos, want_start = [], [], [0]
    for i, (c, n) in enumerate(zip(cached, new)):
        c, n = max(c, 0), max(n, 0)
        have, want = -(-c // page), -(-(c + n) // page)
        for j in range(have, min(want, width)):
            table[i][j] = 100 + taken if taken < n_free else -1
            taken += 1
        missing += want - have
        for pos in range(c, c + min(n, most - len(want_slots))):
            p = table[i][pos // page] if pos // page < width else -1
            want_slots.append(p * page + pos % page if p >= 0 else -1)
            want_pos.append(min(pos, MOST))
        tokens = min(tokens + n, MOST)
        want_start.append(tokens)
    pad = [-1] * (most - len(want_slots))
    taken = min(taken, n_free)
    assert slots.tolist() == want_slots + pad and positions.tolist() == want_pos + pad and start.tolist() == want_start
    assert ctx.tolist() == [min(max(c, 0) + max(n, 0), MOST) for c, n in zip(cached, new)]
    assert counts.tolist() == [taken, tokens, min(missing, MOST) - taken, max(ctx.tolist())]
    assert pool.tolist() == [[5] * width] + table + [[5] * width]


def test_outputs_that_lie_in_the_lengths_are_refused():
    B, i32 = 8, dict(dtype=torch.int32, device="cuda")
    both, new, table, slots = torch.ones(64, **i32), torch.ones(B, **i32), torch.zeros((B, 2), **i32), torch.empty(B, dtype=torch.int64, device="cuda")
    free, start, ctx, counts = torch.arange(B, **i32), torch.empty(B + 1, **i32), torch.empty(B, **i32), torch.empty(4, **i32)
    cached = both[20:20 + B]

    def plan(cached=cached, new=new, start=start, ctx=ctx, counts=counts):
        b.awe_kv_plan(handle(), cached, new, B, 16, free, B, table, 2, 2, slots, None, B, start, ctx, counts)

    launches = b.awe_launch_count(handle())
    for bad in (dict(ctx=cached), dict(ctx=new), dict(ctx=both[13:]), dict(ctx=both[27:]), dict(start=both[12:]), dict(start=new), dict(counts=both[17:]),
                dict(counts=both[27:])):
        with pytest.raises(b.AweError) as e:
            plan(**bad)
        assert e.value.status == 1
    assert b.awe_launch_count(handle()) == launches
    for fine in (dict(ctx=both[12:]), dict(ctx=both[28:]), dict(start=both[11:]), dict(counts=both[16:])):
        plan(**fine)
    torch.cuda.synchronize()
