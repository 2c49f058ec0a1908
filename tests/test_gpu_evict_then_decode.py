"""After an eviction a token attends to exactly the tokens that were kept: sequences that are cut back have all their pages, others may lack some."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, Paged, stream
from test_gpu_attn_decode import run as decode
from test_gpu_cache_evict import draw, kept_slots

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d,page,pool", [("bf16", 8, 2, 64, 16, "heads"), ("f32", 6, 3, 128, 32, "slots")])
@pytest.mark.parametrize("lens,capacity,keep", [([100, 300, 90, 200], 400, 120), ([5000, 9000, 12, 4000], 9008, 4500), ([3000, 33000, 2999], 33024, 3000)])
def test_exactly_the_kept_tokens_are_attended(dtype, hq, hkv, d, page, pool, lens, capacity, keep):
    print(dtype, hq, hkv, d, lens, keep, flush=True)
    c = Paged(dtype, hkv, d, page, lens, capacity=capacity, pool=pool, seed=21)
    for s, n in enumerate(lens):   # pages in front that were given back
        if n <= keep:
            c.table_np[s, :max(1, n // page // 2)] = -1
    c.table.copy_(torch.from_numpy(c.table_np))
    w, order = draw(c, 22)
    before = {(s, h): c.rows(s, h) for s in range(len(lens)) for h in range(hkv)}
    w_dev, o_dev = torch.from_numpy(w).to(DEV), torch.from_numpy(order).to(DEV)
    slots = bs.CacheSlots.of(w_dev, o_dev)
    ws = torch.empty(bs.bs_cache_evict_workspace(c.cache, keep) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_cache_evict(c.cache, c.lens, c.lens, keep, 4, 32, slots, slots, ws, stream=stream())
    torch.cuda.synchronize()
    # the cache as it is now, on the host: same pages, shorter sequences
    c.k_np, c.v_np = c.k.cpu(), c.v.cpu()
    c.lens_np = np.minimum(c.lens_np, keep)
    assert c.lens.tolist() == c.lens_np.tolist()
    for s, n in enumerate(lens):
        for h in range(hkv):
            k, v, there = before[s, h]
            stay = kept_slots(w[s, h, :n], order[s, h, :n], keep, 4, 32) if n > keep else np.ones(n, dtype=bool)
            now = o_dev[s, h, :c.lens_np[s]].cpu().numpy()
            assert (np.sort(now) == np.sort(order[s, h, :n][stay])).all()
            at = np.searchsorted(order[s, h, :n], now)   # the slot that the token had (orders ascend)
            k_now, v_now, there_now = c.rows(s, h)
            assert (there_now == there[at]).all()
            assert (k_now[there_now] == k[at][there_now]).all() and (v_now[there_now] == v[at][there_now]).all()
    decode(c, hq)   # against the plain form on these tokens: the kept ones, as was just seen
