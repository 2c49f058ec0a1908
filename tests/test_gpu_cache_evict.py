"""Eviction from a paged cache: which slots stay, where they go, and that all else stays as it was, exactly."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, Paged, stream
from test_gpu_cache_append import bits

pytestmark = pytest.mark.gpu


def kept_slots(w, order, keep, first, last):
    value = np.where(np.isnan(w), -np.inf, w.astype(np.float64))
    rank = np.where(np.isnan(w), 0, 1)   # a NaN is below everything, -inf included
    safe = (order < first) | (order.astype(np.int64) > int(order.max()) - last)
    value, rank = np.where(safe, np.inf, value), np.where(safe, 2, rank)   # (more of them than `keep`: the lowest slots)
    by = np.lexsort((np.arange(len(w)), -value, -rank))
    stay = np.zeros(len(w), dtype=bool)
    stay[by[:keep]] = True
    return stay


def run(c, keep, first, last, weights, order, in_place):
    n_seqs = len(c.lens_np)
    w, o = torch.from_numpy(weights).to(DEV), torch.from_numpy(order).to(DEV)
    w_out, o_out = (w, o) if in_place else (torch.full_like(w, -5.0), torch.full_like(o, -5))
    lens_out = c.lens if in_place else torch.full_like(c.lens, -5)
    ws = torch.full((bs.bs_cache_evict_workspace(c.cache, keep) + 16,), 0xff, dtype=torch.uint8, device=DEV)
    bs.bs_cache_evict(c.cache, c.lens, lens_out, keep, first, last, bs.CacheSlots.of(w, o), bs.CacheSlots.of(w_out, o_out), ws, stream=stream())
    torch.cuda.synchronize()
    want_k, want_v = bits(c.k_np).clone(), bits(c.v_np).clone()
    want_w, want_o = (weights.copy(), order.copy()) if in_place else (np.full_like(weights, -5), np.full_like(order, -5))
    for s in range(n_seqs):
        n = c.used(s)
        for h in range(c.hkv):
            m = min(n, keep)
            want_w[s, h, :m], want_o[s, h, :m] = weights[s, h, :m], order[s, h, :m]
            if n <= keep:
                continue
            stay = kept_slots(weights[s, h, :n], order[s, h, :n], keep, first, last)
            to, src = np.flatnonzero(~stay[:keep]), keep + np.flatnonzero(stay[keep:])
            want_w[s, h, to], want_o[s, h, to] = weights[s, h, src], order[s, h, src]
            for a, b in zip(to, src):
                pa, pb = c.table_np[s, a // c.page], c.table_np[s, b // c.page]
                if 0 <= pa < c.n_pages and 0 <= pb < c.n_pages:
                    for x in (want_k, want_v):
                        x[pa, h, a % c.page] = x[pb, h, b % c.page]
    assert (lens_out.cpu().numpy() == np.minimum(np.clip(c.lens_np, 0, c.slots), keep)).all()
    assert (w_out.cpu().numpy().view(np.int32) == want_w.view(np.int32)).all()
    assert (o_out.cpu().numpy() == want_o).all()
    assert torch.equal(bits(c.k.cpu()), want_k) and torch.equal(bits(c.v.cpu()), want_v)


def draw(c, seed, zeros=0.1):
    rng = np.random.default_rng([77, seed])
    shape = (len(c.lens_np), c.hkv, c.slots)
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    w[rng.random(shape) < zeros] = 0
    order = np.cumsum(rng.integers(1, 4, shape), axis=2).astype(np.int32) - 1
    return w, order


@pytest.mark.parametrize("dtype,hkv,d,page,pool", [("bf16", 4, 128, 16, "heads"), ("bf16", 2, 64, 48, "slots"), ("f32", 1, 64, 16, "heads"), ("f32", 3, 256, 32, "slots"), ("bf16", 1, 8, 16, "heads")])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (33, 4, 16), (64, 0, 0), (200, 4, 196), (1023, 5, 100), (5000, 0, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(dtype, hkv, d, page, pool, keep, first, last, in_place):
    c = Paged(dtype, hkv, d, page, [0, 1, 2, 32, 33, 34, 64, 65, 199, 201, 1025, 2600], pool=pool, seed=keep)
    run(c, keep, first, last, *draw(c, keep), in_place)


@pytest.mark.parametrize("lens", [[23000, 0, 63, 6000], [1, 8193, 200, 20000, 5, 777] * 9, [5000, 3, 7000] * 14, [5000, 3, 7000] * 90, [3000, 4000] * 20])
@pytest.mark.parametrize("keep,first,last", [(1, 0, 1), (200, 4, 196), (1023, 5, 100), (5000, 0, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_of_other_lengths(lens, keep, first, last, in_place):
    """In chunks; one workgroup each with ranks in LDS; one each with ranks in registers, of 1024 threads, of 512 with 16 and with 8 slots."""
    c = Paged("bf16", 1, 8, 16, lens, seed=keep)
    run(c, keep, first, last, *draw(c, keep), in_place)


@pytest.mark.parametrize("n,keep", [(9000, 1000), (9000, 8999), (40000, 8192), (70001, 65536), (140000, 10)])
def test_long(n, keep):
    c = Paged("bf16", 2, 8, 256, [n, n // 2], seed=1)
    run(c, keep, min(4, keep), min(64, keep - min(4, keep)), *draw(c, n), True)


@pytest.mark.parametrize("values", ["equal", "zeros", "few", "special", "one bit apart"])
@pytest.mark.parametrize("capacity", [3008, 6000, 18000, 40000])   # few rows: one workgroup each, ranks in LDS, or in chunks
def test_ties_and_special_weights(values, capacity):
    make = lambda: Paged("bf16", 2, 8, 16, [700, 3000], capacity=capacity, seed=2)
    c = make()
    w, order = draw(c, 5)
    rng = np.random.default_rng(6)
    if values == "equal":
        w[:] = 1.5
    elif values == "zeros":
        w[:] = 0
        w[rng.random(w.shape) < 0.5] = -0.0
    elif values == "few":
        w = rng.integers(0, 3, w.shape).astype(np.float32)
    elif values == "special":
        w = rng.choice(np.array([np.inf, -np.inf, np.nan, -np.nan, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0], dtype=np.float32), size=w.shape)
    else:
        w = (np.full(w.shape, 0x3f800000, dtype=np.int32) + rng.integers(0, 5, w.shape, dtype=np.int32)).view(np.float32)
    for keep in (1, 350, 699, 2999):
        run(make(), keep, 0, 0, w, order, False)


@pytest.mark.parametrize("capacity", [1008, 5000, 16000, 24000])
def test_orders_that_an_eviction_mixed(capacity):
    c = Paged("bf16", 2, 64, 16, [500, 900], capacity=capacity, seed=3)
    w, order = draw(c, 7)
    rng = np.random.default_rng(8)
    for s, n in enumerate((500, 900)):
        for h in range(2):
            order[s, h, :n] = rng.permutation(order[s, h, :n])
    run(c, 300, 20, 100, w, order, True)


def test_orders_at_the_ends_of_their_type():
    c = Paged("bf16", 1, 8, 16, [100], seed=4)
    w, order = draw(c, 9)
    order[0, 0, :100] = np.arange(100)
    order[0, 0, 50] = 2 ** 31 - 1
    order[0, 0, 60] = -2 ** 31
    run(c, 40, 3, 20, w, order, True)
    order[0, 0, :100] = -2 ** 31
    run(Paged("bf16", 1, 8, 16, [100], seed=4), 40, 0, 40, w, order, True)


def test_slots_without_a_page_and_lengths_out_of_range():
    c = Paged("bf16", 2, 64, 16, [300, -5, 2 ** 31 - 1, 200], capacity=400, bad=0.3, seed=5)
    run(c, 120, 4, 30, *draw(c, 10), True)


def test_rows_longer_than_the_sequences_and_others_out_than_in():
    c = Paged("bf16", 2, 64, 16, [300, 100], seed=6)
    w, order = draw(c, 11)
    w, order = (np.concatenate([x, np.full(x.shape[:2] + (9,), 7, dtype=x.dtype)], axis=2) for x in (w, order))
    run(c, 120, 4, 30, w, order, False)
