"""Prompts on their way into the cache with normed keys: calls so long that a thread takes several heads, of numbers that its share does not divide, into both orders of
a page's axes.  Against the plain form in 64 bits (tolerances: test_gpu_norm_rope.py)."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, Paged, stream
from test_gpu_norm_rope import draw, draw_weight, near, plain

pytestmark = pytest.mark.gpu


# (heads of a thread: 5, 2, 6, 2 and 3, as 2^19 threads are shared out)
@pytest.mark.parametrize("dtype,hq,hkv,d,r,tokens", [("bf16", 28, 4, 128, 128, 9001), ("f32", 5, 3, 256, 256, 2600), ("bf16", 6, 3, 72, 18, 5003), ("bf16", 8, 5, 96, 96, 2003),
                                                     ("f32", 3, 7, 64, 32, 12007)])
@pytest.mark.parametrize("page,pool", [(16, "heads"), (48, "slots")])
@pytest.mark.parametrize("with_q", [True, False])
def test_a_prompt(dtype, hq, hkv, d, r, tokens, page, pool, with_q):
    print(dtype, hq, hkv, d, tokens, page, pool, with_q, flush=True)
    rng = np.random.default_rng([d, tokens])
    base, share = np.array([0, 15, 100, 33]), np.array([0.6, 0.05, 0.3, 0.05])
    new = (share * tokens).astype(np.int64)
    new[0] += tokens - new.sum()
    c = Paged(dtype, hkv, d, page, base, pool=pool, more=int(new.max()), seed=d, bad=0.05)
    before = [x.clone() for x in (c.k, c.v)]
    seq, slot = np.repeat(np.arange(4), new), np.concatenate([b + np.arange(n) for b, n in zip(base, new)])
    lost = rng.random(tokens)
    seq, slot = np.where(lost < 0.01, rng.choice([-1, 4, 2 ** 30], tokens), seq), np.where(lost > 0.99, rng.choice([-1, c.slots, 2 ** 31 - 1], tokens), slot)
    order = rng.permutation(tokens)
    seq, slot = seq[order].astype(np.int32), slot[order].astype(np.int32)
    q, k, v = draw(hq, tokens, d, dtype), draw(hkv, tokens, d, dtype, 1), draw(hkv, tokens, d, dtype, 2)
    ws = [draw_weight(d, dtype, 1, i) for i in range(2)]
    wd = [w.to(DEV) for w in ws]
    rope, pos = bs.bs_rope_init(r), rng.integers(0, 100000, (1, tokens)).astype(np.int32)
    dev = lambda x: torch.from_numpy(x).to(DEV)
    heads = lambda x: x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)   # token by token, as a projection leaves them
    q_in = heads(q) if with_q else None
    q_out = torch.full_like(q_in, float("nan")) if with_q else None
    w_rows, o_rows = torch.full((4, hkv, c.slots), 7.0, device=DEV), torch.full((4, hkv, c.slots), -3, dtype=torch.int32, device=DEV)
    token_order = rng.permutation(tokens).astype(np.int32) + 1000
    bs.bs_cache_append_norm(c.cache, heads(k), heads(v), tokens, dev(seq), dev(slot), bs.Norm.of(wd, 1e-5, 1.0), rope=rope, positions=dev(pos), q=q_in, q_out=q_out,
                            slots=bs.CacheSlots.of(w_rows, o_rows), token_order=dev(token_order), stream=stream())
    torch.cuda.synchronize()
    eps = float(np.float32(1e-5))
    if with_q:
        near(q_out, *plain(rope, q.double().numpy(), ws[0].double().numpy() + 1, eps, pos), dtype)
    # which tokens have a slot, and those that have a page
    has = np.flatnonzero((seq >= 0) & (seq < 4) & (slot >= 0) & (slot < c.slots))
    p = c.table_np[seq[has], slot[has] // page]
    has, p = has[(p >= 0) & (p < c.n_pages)], p[(p >= 0) & (p < c.n_pages)].astype(np.int64)
    assert tokens * 0.8 < len(has) < tokens
    at = torch.from_numpy(p), torch.from_numpy(slot[has].astype(np.int64) % page)
    now = [x.cpu() for x in (c.k, c.v)]
    want, tol = plain(rope, k.double().numpy(), ws[1].double().numpy() + 1, eps, pos)
    near(now[0].transpose(1, 2)[at].transpose(0, 1), want[:, has], tol[:, has], dtype)
    mine = torch.from_numpy(has)
    assert torch.equal(now[1].transpose(1, 2)[at], v.transpose(0, 1)[mine])
    written = torch.zeros((c.n_pages, page), dtype=torch.bool)
    written[at] = True
    for old, new_ in zip(before, now):   # all else as it was, NaN too
        kept = ~written[:, None, :, None].expand(old.shape)
        assert torch.equal(old.cpu().contiguous()[kept].view(torch.uint8), new_.contiguous()[kept].view(torch.uint8))
    w_want, o_want = torch.full((4, hkv, c.slots), 7.0), torch.full((4, hkv, c.slots), -3, dtype=torch.int32)
    to = torch.from_numpy(seq[has].astype(np.int64)), torch.from_numpy(slot[has].astype(np.int64))
    w_want[to[0], :, to[1]] = 0.0
    o_want[to[0], :, to[1]] = torch.from_numpy(token_order[has])[:, None].expand(-1, hkv)
    assert torch.equal(w_rows.cpu(), w_want) and torch.equal(o_rows.cpu(), o_want)
