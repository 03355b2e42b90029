"""The serving example's parts that need no GPU: what it refuses, and its scheduler on the sequential page program."""

import os
import random
import sys

import numpy as np
import pytest

from oracle import paged as P

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_a_request_larger_than_the_pool_is_refused():
    import paged_serving
    with pytest.raises(ValueError):
        paged_serving.serve(requests=9, pages=3, longest=400)


@pytest.mark.parametrize("page,batch,chunk", [(16, 8, 64), (16, 3, 64), (1, 8, 5), (64, 16, 64), (100, 8, 7)])
@pytest.mark.parametrize("room", [1.0, 1.3, 2.0, 3.0, 10.0])
def test_all_requests_end_however_few_pages_there_are(page, batch, chunk, room):
    """`room`: pages, as a multiple of what the largest request needs."""
    import paged_serving
    for seed in range(6):
        rng = random.Random(seed)
        work = [(rng.randint(1, 300), rng.randint(1, 75)) for _ in range(24)]
        need = max(-(-sum(r) // page) for r in work)
        pages = int(need * room)
        plan = paged_serving.Scheduler(work, batch, chunk)
        table, free, left = np.zeros((batch, need), dtype=int), np.arange(pages), pages
        while plan.done < len(work):
            held = list(plan.held)
            new, owner = plan.ask()
            assert len(owner) <= batch * chunk
            w = P.page_update(page, held, new, table, free, left, len(owner))
            table, free, left = w["block_table"], w["free_pages"], int(w["free"][0])
            plan.answer(new, w["seq_len"].tolist())
            assert plan.steps < 20000
        assert plan.tokens >= sum(map(sum, work)) and not any(plan.running)
        assert plan.restarted == 0 or plan.refused
