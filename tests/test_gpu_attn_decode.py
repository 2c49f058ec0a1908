"""Attention of one new token per sequence over a paged cache against a plain form in 64 bits.

Tolerance, per element, with A = sum_j p_j |v_j|, S = the largest sum |q k| scale and n = the longest sequence:
  scores are sums of d products in fp32: off by at most d 2^-24 S, which changes a probability by twice that, relatively;
  sums over slots: at most n roundings of 2^-24; exponentials, reference points and the joining of parts: 64 steps of 2^-24;
  bf16: each probability is the sum of two bf16 numbers, off by at most 2^-8 of the second, which is at most 2^-8 of the whole: 2^-16 A; the
  result is rounded once: 2^-8 |out|."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, TYPES, Paged, attention, stream

pytestmark = pytest.mark.gpu


def step(d, S, n):
    return (2 * d * S + n + 64) * 2.0 ** -24


def bounds(dtype, d, S, n, out, spread):
    tol = step(d, S, n) * spread * 2
    if dtype == "bf16":
        tol = tol + 2.0 ** -16 * spread
    return tol + HALF_STEP[dtype] * (np.abs(out) + tol)


def run(c, hq, window=0, weights=None, token_major=True, seed=0, in_place=False, scale=None):
    g = torch.Generator()
    g.manual_seed(100 + seed)
    n_seqs, d = len(c.lens_np), c.d
    scale = d ** -0.5 if scale is None else scale
    q = torch.randn((n_seqs, hq, d), generator=g).to(TYPES[c.dtype])
    dev = q.to(DEV) if token_major else q.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    out = torch.full_like(dev, float("nan"))
    slots = slots_out = w_out = None
    if weights is not None:
        w = weights.to(DEV)
        w_out = w if in_place else torch.full_like(w, -5.0)
        slots, slots_out = bs.CacheSlots.of(w), bs.CacheSlots.of(w_out)
    ws = torch.full((bs.bs_attn_decode_workspace(c.cache, hq, weights is not None) + 16,), 0xff, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(c.cache, dev.transpose(0, 1), out.transpose(0, 1), c.lens, scale, ws, window=window, slots=slots, slots_out=slots_out, stream=stream())
    torch.cuda.synchronize()
    want, spread, probs, S = attention(c, q.double().numpy(), scale, window)
    n = int(np.clip(c.lens_np, 0, c.slots).max())
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    tol = bounds(c.dtype, d, S, n, want, spread)
    worst = np.abs(got - want) - tol
    assert (worst <= 0).all(), (float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))
    if weights is not None:
        G, got_w = hq // c.hkv, w_out.double().cpu().numpy()
        for s in range(n_seqs):
            m = c.used(s)
            for h in range(c.hkv):
                p = sum(probs[s, h * G + i] for i in range(G))
                before = weights[s, h].double().numpy()
                tol = step(d, S, n) * 2 * p + (G + 2) * 2.0 ** -24 * (before[:m] + p)
                assert (np.abs(got_w[s, h, :m] - before[:m] - p) <= tol).all(), (s, h)
                assert (got_w[s, h, m:] == (before[m:] if in_place else -5.0)).all()
    return out, w_out


def test_more_items_than_threads_and_none_of_them_used():
    """One sequence of 400 KV heads: fewer items than shares, more than a workgroup has threads."""
    for n in (0, 5, 40):
        run(Paged("bf16", 400, 64, 16, [n], capacity=64, seed=13), 400)
    run(Paged("bf16", 150, 64, 16, [0, 40, 0], capacity=64, seed=13), 300)


SHAPES = [("bf16", 28, 4, 128), ("bf16", 8, 8, 64), ("bf16", 32, 2, 128), ("bf16", 20, 1, 64), ("f32", 2, 1, 64), ("f32", 14, 2, 128), ("f32", 40, 2, 64),
          ("bf16", 66, 2, 64), ("f32", 33, 1, 128)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page,pool", [(16, "heads"), (48, "slots")])
def test_lengths(dtype, hq, hkv, d, page, pool):
    print(dtype, hq, hkv, d, page, pool, flush=True)
    run(Paged(dtype, hkv, d, page, [1, 0, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 700], pool=pool, seed=hq), hq, token_major=pool == "heads")


@pytest.mark.parametrize("dtype,hq,hkv,d,lens,page", [
    ("bf16", 28, 4, 128, [5001], 16), ("bf16", 32, 16, 128, [9000, 1, 3], 64), ("bf16", 32, 8, 64, [4097, 4096], 256), ("f32", 8, 2, 128, [3333], 32),
    ("f32", 2, 1, 64, [1136, 7], 16), ("bf16", 40, 8, 128, [17, 300, 2000, 1, 64, 999, 4, 1200, 31, 33], 32), ("bf16", 2, 1, 64, [30000], 16)])
def test_long(dtype, hq, hkv, d, lens, page):
    print(dtype, hq, hkv, d, lens, page, flush=True)
    run(Paged(dtype, hkv, d, page, lens, seed=3), hq)


def test_many_short_sequences():
    rng = np.random.default_rng(9)
    for n_seqs in (300, 1100):
        print(n_seqs, flush=True)
        run(Paged("bf16", 2, 64, 16, rng.integers(0, 50, n_seqs), seed=4), 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 5000])
def test_window(dtype, window):
    run(Paged(dtype, 2, 64, 16, [1, 0, 33, 64, 100, 131, 900], seed=5), 8, window=window)


def test_pages_out_of_a_window_may_be_gone():
    c = Paged("bf16", 2, 128, 16, [500, 300, 120], seed=6)
    gone = c.table.clone()
    for s, n in enumerate([500, 300, 120]):
        gone[s, :(n - 100) // 16] = -1
    c.table.copy_(gone)
    run(c, 4, window=100)


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 28, 4, 128), ("f32", 2, 1, 64), ("bf16", 40, 2, 64)])
def test_slots_without_a_page_are_not_seen(dtype, hq, hkv, d):
    c = Paged(dtype, hkv, d, 16, [1, 20, 33, 100, 400, 1500], bad=0.4, seed=7)
    run(c, hq)
    c = Paged(dtype, hkv, d, 16, [1, 200], bad=1.0, seed=7)
    out, _ = run(c, hq)
    assert (out == 0).all()


def test_lengths_out_of_range():
    c = Paged("bf16", 2, 64, 32, [-3, 70, 1000, 2 ** 31 - 1, -2 ** 31], capacity=96, seed=8)
    run(c, 6)


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("in_place", [False, True])
def test_weights(dtype, hq, hkv, d, in_place):
    c = Paged(dtype, hkv, d, 16, [1, 0, 33, 129, 1700], seed=9)
    g = torch.Generator()
    g.manual_seed(1)
    run(c, hq, weights=torch.rand((5, hkv, c.slots), generator=g), in_place=in_place)


def test_weights_of_slots_without_a_page_stay():
    c = Paged("bf16", 2, 128, 16, [40, 900], bad=0.5, seed=10)
    run(c, 8, weights=torch.zeros((2, 2, c.slots)))


def test_rows_of_slots_may_be_longer_than_the_sequences():
    c = Paged("bf16", 2, 128, 16, [40, 900], seed=10)
    run(c, 8, weights=torch.ones((2, 2, c.slots + 37)))


def test_large_scores():
    run(Paged("bf16", 2, 128, 16, [1000, 50], seed=11), 8, scale=3.0)
    run(Paged("f32", 2, 64, 16, [1000, 50], seed=11), 8, scale=3.0)


def test_same_bits_again():
    c = Paged("bf16", 4, 128, 16, [20000, 33, 700], seed=12)
    g = torch.Generator()
    w = torch.rand((3, 4, c.slots), generator=g)
    a = run(c, 28, weights=w)
    for _ in range(3):
        b = run(c, 28, weights=w)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_beyond_32_bits():
    """A pool of 3 GB whose last pages are used."""
    page, hkv, d = 16, 8, 128
    n_pages = 3 * 2 ** 30 // (page * hkv * d * 2)
    k = torch.zeros((n_pages, hkv, page, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    last = torch.arange(n_pages - 4, n_pages)
    g = torch.Generator()
    g.manual_seed(2)
    kk, vv = (torch.randn((4, hkv, page, d), generator=g).to(torch.bfloat16) for _ in range(2))
    k[last.to(DEV)], v[last.to(DEV)] = kk.to(DEV), vv.to(DEV)
    table = last.to(torch.int32)[None].contiguous().to(DEV)
    lens = torch.tensor([60], dtype=torch.int32, device=DEV)
    cache = bs.KVCache.of(k, v, table, bs.BS_BF16)
    q = torch.randn((hkv, 1, d), generator=g).to(torch.bfloat16)
    out = torch.empty_like(q, device=DEV)
    ws = torch.empty(bs.bs_attn_decode_workspace(cache, hkv) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(cache, q.to(DEV), out, lens, d ** -0.5, ws, stream=stream())
    for h in range(hkv):
        keys, values = kk[:, h].reshape(-1, d)[:60].double(), vv[:, h].reshape(-1, d)[:60].double()
        p = torch.softmax(keys @ q[h, 0].double() * d ** -0.5, 0)
        S = float((keys.abs() @ q[h, 0].double().abs()).max() * d ** -0.5)
        tol = (2 * step(d, S, 60) + 2.0 ** -16) * (p @ values.abs()) * 1.01 + 2.0 ** -8 * (p @ values).abs()
        assert ((out[h, 0].double().cpu() - p @ values).abs() <= tol).all()
