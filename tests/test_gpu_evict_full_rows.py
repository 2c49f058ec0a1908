"""Eviction by one workgroup per row with as many slots as its LDS holds: 128 KB of ranks, counts near the limit of their 16 bits."""
import numpy as np
import pytest

from cache_util import Paged
from test_gpu_cache_evict import draw, run

import paper_2507_09071_amd as bs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("values", ["equal", "random", "but one"])
@pytest.mark.parametrize("keep,first,last", [(32767, 0, 0), (16384, 0, 16384), (700, 4, 64), (1, 0, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_of_32768_slots(values, keep, first, last, in_place):
    """33 rows: with fewer, rows this long are cut into chunks."""
    print(values, keep, flush=True)
    c = Paged("bf16", 11, 8, 256, [32768, 32768, 20481], capacity=32768, seed=1)
    # (the workspace of chunks would hold three histograms a row)
    assert bs.bs_cache_evict_workspace(c.cache, keep) < 33 * 8 * min(keep, 32768 - keep) + 33 * 1024
    w, order = draw(c, 3)
    if values != "random":
        w[:] = 1.5
    if values == "but one":
        w[:, :, 0] = 0.5       # ties for all places but one
        w[:, :, 20480] = 2.5   # the last slot of the shortest row
    run(c, keep, first, last, w, order, in_place)
