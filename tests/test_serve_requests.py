"""What the scheduler takes as a request, on the host alone: no GPU, no model."""
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2607_21042_amd import ftts, serve


def scheduler(n_pages, max_pages, prefix_pages=0):
    """A scheduler's host state: its pool after the shared prefix has taken its pages, and two empty slots."""
    s = serve.Scheduler.__new__(serve.Scheduler)
    s.shape = SimpleNamespace(d_model=4)
    s.max_pages, s.pool = max_pages, ftts.PagePool(n_pages)
    s.pool.alloc(prefix_pages)
    s.slot_pages, s.waiting, s.next_rid = [[], []], [], 0
    return s


def request(rows, budget):
    return serve.Request(prefix=np.zeros((rows, 4), dtype=np.float32), max_new=budget)


@pytest.mark.parametrize("n_pages,prefix_pages,most", [(5, 3, 2), (5, 0, 3), (2, 0, 2), (3, 3, 0)])
def test_a_request_that_never_fits_the_pool_is_refused(n_pages, prefix_pages, most):
    """It would wait for pages that no request gives back, and hold up all behind it."""
    for pages in range(1, 4):
        s = scheduler(n_pages, 3, prefix_pages)
        if pages <= most:
            assert s.submit(request(64 * pages - 9, 9)).rid == 0 and len(s.waiting) == 1
        else:
            with pytest.raises(ValueError, match="pool"):
                s.submit(request(64 * pages - 9, 9))
            assert not s.waiting and s.next_rid == 0


def test_pages_in_use_count_as_pages_that_come_back():
    s = scheduler(5, 4, 1)
    s.slot_pages[1] = s.pool.alloc(3)
    s.submit(request(200, 56))
    with pytest.raises(ValueError, match="max_ctx"):
        s.submit(request(200, 57))
