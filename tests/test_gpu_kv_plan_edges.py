"""The cache plan from several host threads."""
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
