"""Sizes that an eviction cannot launch, or whose workspace does not fit 64 bits, are refused with a code that says so; others are not."""
import pytest

import paper_2507_09071_amd as bs
from paper_2507_09071_amd import binding
from test_cache_refusals import EUNSUPPORTED, P, cache, ref

MOST = 2 ** 31 - 65552   # slots of a sequence


@pytest.mark.parametrize("n_seqs,n_kv,slots,keep", [(2 ** 31 - 1, 1, MOST, 2 ** 30), (2 ** 30, 1, MOST, 2 ** 30), (2 ** 29, 2, MOST, 2 ** 30 - 2 ** 15), (2 ** 24, 1, MOST, 5),
                                                    (2 ** 24, 1, 2048, 5), (2 ** 23, 1, 2064, 5), (2 ** 23, 1, 8192, 5), (2 ** 22, 1, 8208, 5), (2 ** 19, 8, 32768, 5)])
def test_too_many_rows(n_seqs, n_kv, slots, keep):
    lib, s = binding.load_library(), bs.CacheSlots(P, P, 1 << 32)
    c = cache(n_seqs=n_seqs, n_kv_heads=n_kv, max_pages=slots // 16, page_stride=16 * 8 * 128)
    assert lib.bs_cache_evict_workspace(ref(c), keep) == EUNSUPPORTED
    assert lib.bs_cache_evict(ref(c), P, P, keep, 0, 0, ref(s), ref(s), P, 2 ** 63 - 1, None) == EUNSUPPORTED


@pytest.mark.parametrize("slots,rows", [(2048, 2 ** 24 - 1), (4096, 2 ** 23 - 1), (8192, 2 ** 23 - 1), (8208, 2 ** 22 - 1), (32768, 2 ** 22 - 1), (32784, 2 ** 24 - 1), (MOST, 2 ** 24 - 1)])
def test_as_many_rows_as_a_grid_has(slots, rows):
    assert binding.load_library().bs_cache_evict_workspace(ref(cache(n_seqs=rows, n_kv_heads=1, max_pages=slots // 16)), 10) > 80 * rows
