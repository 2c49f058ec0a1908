"""Rows that are written lie apart, all axes taken together: which strides of a cache and of heads are refused, on the host."""
import itertools

import numpy as np
import pytest

import paper_2507_09071_amd as bs
from paper_2507_09071_amd import binding
from test_cache_refusals import EINVAL, P, cache, heads, ref


def evict_workspace(**kw):
    return binding.load_library().bs_cache_evict_workspace(ref(cache(**kw)), 5)


def append(c, **kw):
    h = heads(c.n_kv_heads, token=128 * c.n_kv_heads)
    return binding.load_library().bs_cache_append(ref(c), ref(h), ref(h), kw.get("n", 0), None, P, None, None, 0, None, None, None, None, None)


# page, head, slot; 4 heads, pages of 16 slots, rows of 128
@pytest.mark.parametrize("strides", [(128, 128, 128), (8192, 128, 128), (2048, 2048, 128), (8192, 2048, 0), (8192, 256, 128), (8184, 2048, 128), (8192, 128, 504),
                                     (8192, 2040, 128), (2 ** 40, 128, 128), (512, 128, 1024)])
def test_strides_that_alias_rows_together(strides):
    kw = dict(zip(("page_stride", "head_stride", "slot_stride"), strides))
    assert evict_workspace(**kw) == EINVAL
    assert append(cache(**kw), n=3) == EINVAL


@pytest.mark.parametrize("strides", [
    (8192, 2048, 128),          # [page][head][slot][d]
    (8192, 128, 512),           # [page][slot][head][d]
    (2048, 20480, 128),         # [head][page][slot][d]
    (512, 128, 5120),           # [slot][page][head][d]
    (16384, 2048, 128),         # K and V of a page one behind the other
    (8192 * 32, 2048, 128),     # ... and of many layers
    (10000, 2208, 136)])        # gaps everywhere
def test_strides_of_every_order_of_axes(strides):
    kw = dict(zip(("page_stride", "head_stride", "slot_stride"), strides))
    assert evict_workspace(**kw) > 0
    assert append(cache(**kw)) == 0   # (no token: nothing is launched)


def test_axes_of_one_element_may_have_any_stride():
    assert evict_workspace(n_kv_heads=1, head_stride=0, page_stride=2048) > 0
    assert evict_workspace(n_pages=1, page_stride=0) > 0


def test_against_the_sets_of_elements():
    """Small caches: what is accepted never writes an element twice."""
    rng = np.random.default_rng(3)
    accepted = 0
    for _ in range(400):
        heads_, pages = int(rng.integers(1, 4)), int(rng.integers(1, 4))
        strides = [int(x) * 8 for x in rng.integers(0, 60, 3)]
        ok = evict_workspace(n_kv_heads=heads_, n_pages=pages, page_size=16, head_dim=8, page_stride=strides[0], head_stride=strides[1], slot_stride=strides[2]) > 0
        accepted += ok
        rows = [p * strides[0] + h * strides[1] + j * strides[2] for p, h, j in itertools.product(range(pages), range(heads_), range(16))]
        if ok:
            rows = np.sort(rows)
            assert (np.diff(rows) >= 8).all(), (heads_, pages, strides)
    assert accepted > 20


@pytest.mark.parametrize("head,token,tokens", [(2 ** 40, 2 ** 40, 2 ** 24 + 1), (128, 2 ** 40, 2 ** 24 + 1), (2 ** 39, 2 ** 40, 2 ** 25 + 1)])
def test_strides_times_counts_beyond_64_bits(head, token, tokens):
    """2^40 times 2^24 is nothing in 64 bits: such rows seemed to lie apart."""
    lib, rope = binding.load_library(), bs.bs_rope_init(64)
    assert lib.bs_rope_apply(ref(rope), ref(heads(2)), ref(heads(2, head=head, token=token)), 1, bs.BS_BF16, tokens, 128, P, 0, 0, None) == EINVAL
    assert lib.bs_rope_apply(ref(rope), ref(heads(2)), ref(heads(2, head=head, token=token)), 1, bs.BS_BF16, 0, 128, P, 0, 0, None) == 0
