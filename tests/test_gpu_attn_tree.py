"""Attention of drafted tokens over a paged cache against a plain form in 64 bits (tolerances: tree_util.bounds)."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, Paged, stream
from tree_util import Drafts, bounds, draw_q, run, tree_bits, words_of

pytestmark = pytest.mark.gpu


def trees(counts, seed=0):
    rng = np.random.default_rng([7, seed])
    return [tree_bits(rng, n) for n in counts]


# (rows of a sequence and KV head: up to 16, 32, 64, 128, 256 and beyond)
SHAPES = [("bf16", 28, 4, 128), ("bf16", 8, 8, 64), ("bf16", 32, 2, 128), ("bf16", 20, 1, 64), ("f32", 2, 1, 64), ("f32", 14, 2, 128), ("f32", 8, 8, 128),
          ("bf16", 33, 1, 64)]


@pytest.mark.parametrize("dtype,hq,hkv,d", SHAPES)
@pytest.mark.parametrize("most", [1, 2, 5, 9, 26, 64, 65])
def test_rows_and_lengths(dtype, hq, hkv, d, most):
    print(dtype, hq, hkv, d, most, flush=True)
    lens = [1, 0, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 700]
    counts = [1 + (5 * i) % most for i in range(len(lens))]
    counts[3], counts[7] = most, 0
    page, pool = ((16, "heads"), (48, "slots"))[most % 2]
    run(Drafts(dtype, hkv, d, page, lens, counts, trees(counts), pool=pool, seed=hq), hq, token_major=pool == "heads")


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 28, 4, 128), ("bf16", 2, 1, 64), ("f32", 4, 1, 128), ("bf16", 128, 2, 64)])
def test_most_tokens(dtype, hq, hkv, d):
    """256 tokens: several groups of rows, four words of mask."""
    for counts in ([256], [3, 256, 0, 200]):
        print(dtype, hq, hkv, d, counts, flush=True)
        run(Drafts(dtype, hkv, d, 16, [333, 40, 7, 90][:len(counts)], counts, trees(counts), seed=1), hq)


@pytest.mark.parametrize("dtype,hq,hkv,d,lens,counts,page", [
    ("bf16", 28, 4, 128, [5001], [26], 16), ("bf16", 32, 16, 128, [9000, 1, 3], [64, 64, 2], 64), ("bf16", 32, 8, 64, [4097, 4096], [4, 3], 256),
    ("f32", 8, 2, 128, [3333], [11], 32), ("f32", 2, 1, 64, [1131, 7], [5, 1], 16), ("bf16", 40, 8, 128, [17, 300, 2000, 1, 64, 999, 4, 1200, 31, 33], list(range(1, 11)), 32),
    ("bf16", 2, 1, 64, [30000], [8], 16), ("bf16", 16, 2, 128, [12001, 500], [16, 40], 64), ("f32", 32, 2, 64, [2500], [30], 16)])
def test_long(dtype, hq, hkv, d, lens, counts, page):
    print(dtype, hq, hkv, d, lens, page, flush=True)
    run(Drafts(dtype, hkv, d, page, lens, counts, trees(counts), seed=3), hq)


def test_many_short_sequences():
    rng = np.random.default_rng(9)
    for n_seqs in (300, 1100):
        print(n_seqs, flush=True)
        counts = rng.integers(0, 4, n_seqs)
        run(Drafts("bf16", 2, 64, 16, rng.integers(0, 50, n_seqs), counts, seed=4), 4)
    counts = rng.integers(0, 20, 700)
    run(Drafts("bf16", 1, 64, 16, rng.integers(0, 20, 700), counts, seed=4), 8)


@pytest.mark.parametrize("hq,hkv,most", [(8, 2, 4), (8, 2, 7), (8, 2, 60), (64, 2, 7), (28, 4, 70)])
def test_a_chain_is_a_tree_without_branches(hq, hkv, most):
    counts, lens = [most, 1, most // 2, 2], [100, 0, 31, 600]
    chains = [np.tril(np.ones((n, n), dtype=bool)) for n in counts]
    a = run(Drafts("bf16", hkv, 128, 16, lens, counts, None, seed=5), hq)
    b = run(Drafts("bf16", hkv, 128, 16, lens, counts, chains, seed=5), hq, words=3)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 28, 4, 128), ("f32", 8, 2, 64)])
def test_masks_that_are_no_trees(dtype, hq, hkv, d):
    """Tokens that see later ones, not themselves, or nothing drafted; rows that see nothing at all are zero."""
    rng = np.random.default_rng(11)
    counts, lens = [9, 33, 70, 5], [0, 40, 0, 16]
    bits = [rng.random((n, n)) < 0.4 for n in counts]
    bits[0][3] = bits[2][0] = bits[2][69] = bits[1][5] = False
    out = run(Drafts(dtype, hkv, d, 16, lens, counts, bits, seed=6), hq)
    first = np.concatenate([[0], np.cumsum(counts)])
    assert (out[first[0] + 3] == 0).all() and (out[first[2]] == 0).all() and (out[first[2] + 69] == 0).all() and (out[first[1] + 5] != 0).any()


def test_bits_of_tokens_that_are_not_there_mean_nothing():
    rng = np.random.default_rng(12)
    counts, lens = [3, 20, 64], [10, 0, 50]
    bits = trees(counts)
    d = Drafts("bf16", 2, 64, 16, lens, counts, bits, seed=7)
    a = run(d, 8, most=70)
    d.bits = [np.concatenate([b, rng.random((n, 128 - n)) < 0.5], 1) for b, n in zip(bits, counts)]   # the same, with more bits
    mask = torch.cat([words_of(b, 2) for b in d.bits]).to(DEV)
    q = draw_q(d, 8).to(DEV)
    out = torch.empty_like(q)
    ws = torch.empty(bs.bs_attn_tree_workspace(d.c.cache, 8, d.n, 70) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(d.c.cache, q.transpose(0, 1), out.transpose(0, 1), d.n, torch.from_numpy(d.first.astype(np.int32)).to(DEV), d.lens, 70, 0.125, ws, mask=mask, stream=stream())
    assert torch.equal(a, out)


@pytest.mark.parametrize("dtype,hq", [("bf16", 8), ("f32", 8), ("bf16", 64)])
@pytest.mark.parametrize("window", [1, 2, 6, 31, 32, 33, 100, 5000])
def test_window(dtype, hq, window):
    counts = [1, 5, 12, 3, 40, 7, 20]
    run(Drafts(dtype, 2, 64, 16, [1, 0, 33, 64, 100, 131, 900], counts, trees(counts), seed=8), hq, window=window)
    run(Drafts(dtype, 2, 64, 16, [1, 0, 33, 64, 100, 131, 900], counts, None, seed=8), hq, window=window)


def test_pages_out_of_a_window_may_be_gone_and_their_rows_anything():
    lens, counts = [500, 300, 120], [6, 1, 17]
    d = Drafts("bf16", 2, 128, 16, lens, counts, trees(counts), seed=6)
    gone = d.c.table.clone()
    for s, n in enumerate(lens):
        gone[s, :(n - 100) // 16] = -1
    d.c.table.copy_(gone)
    for s, n in enumerate(lens):   # slots before every row's window, in pages that are there
        for j in range((n - 100) // 16 * 16, n - 100):
            d.c.k[d.c.table_np[s, j // 16], :, j % 16] = float("nan")
            d.c.v[d.c.table_np[s, j // 16], :, j % 16] = float("-inf")
    run(d, 4, window=100)


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 28, 4, 128), ("f32", 2, 1, 64), ("bf16", 40, 2, 64)])
def test_slots_without_a_page_are_not_seen(dtype, hq, hkv, d):
    lens, counts = [1, 20, 33, 100, 400, 1500], [4, 1, 20, 9, 2, 30]
    run(Drafts(dtype, hkv, d, 16, lens, counts, trees(counts), bad=0.4, seed=7), hq)
    out = run(Drafts(dtype, hkv, d, 16, [1, 200], [3, 6], None, bad=1.0, seed=7), hq)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype,hq", [("bf16", 8), ("f32", 6), ("bf16", 32), ("bf16", 80)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_that_only_some_rows_see(dtype, hq, value):
    """A drafted token's K and V that are not finite reach the rows that see it and no others."""
    counts, lens = [12, 20], [37, 5]
    bits = trees(counts, 3)
    for what in "kv":
        d = Drafts(dtype, 2, 64, 16, lens, counts, bits, seed=9)
        clean = run(d, hq)
        for s, a in ((0, 4), (1, 7)):
            j = lens[s] + a
            getattr(d.c, what)[d.c.table_np[s, j // 16], :, j % 16, 5] = value
        q = draw_q(d, hq).to(DEV)
        out = torch.empty_like(q)
        mask = torch.cat([words_of(b, 1) for b in bits]).to(DEV)
        ws = torch.empty(bs.bs_attn_tree_workspace(d.c.cache, hq, d.n, d.most) + 16, dtype=torch.uint8, device=DEV)
        bs.bs_attn_tree(d.c.cache, q.transpose(0, 1), out.transpose(0, 1), d.n, torch.from_numpy(d.first.astype(np.int32)).to(DEV), d.lens, d.most, 0.125, ws, mask=mask,
                        stream=stream())
        sees = np.concatenate([bits[0][:, 4], bits[1][:, 7]])
        assert 0 < sees.sum() < d.n
        assert torch.equal(out[~torch.from_numpy(sees).to(DEV)], clean[~torch.from_numpy(sees).to(DEV)])
        if what == "v":
            assert not torch.isfinite(out[torch.from_numpy(sees).to(DEV)][..., 5]).any()


@pytest.mark.parametrize("dtype,hq", [("bf16", 8), ("f32", 8), ("bf16", 70)])
@pytest.mark.parametrize("cap,scale", [(50.0, None), (1.0, None), (5.0, 2.0), (1e4, None), (0.01, 1.0)])
def test_capped_scores(dtype, hq, cap, scale):
    counts = [3, 17, 1]
    run(Drafts(dtype, 2, 128, 16, [400, 33, 90], counts, trees(counts), seed=10), hq, cap=cap, scale=scale)


@pytest.mark.parametrize("dtype,hq", [("bf16", 8), ("f32", 8), ("bf16", 70)])
def test_small_scores_beside_capped_ones(dtype, hq):
    """Every other token has scores of a thousand times the others', far beyond the cap: the others keep the tolerance of their own scores."""
    counts = [6, 1, 12]
    d = Drafts(dtype, 2, 128, 16, [200, 31, 500], counts, trees(counts), seed=14)
    q, scale, cap = draw_q(d, hq), 128 ** -0.5, 300.0
    large = torch.arange(d.n) % 2 == 1
    q[large] *= 1000
    dev = q.to(DEV)
    out = torch.empty_like(dev)
    mask = torch.cat([words_of(b, 1) for b in d.bits]).to(DEV)
    first = torch.from_numpy(d.first.astype(np.int32)).to(DEV)
    ws = torch.empty(bs.bs_attn_tree_workspace(d.c.cache, hq, d.n, d.most), dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(d.c.cache, dev.transpose(0, 1), out.transpose(0, 1), d.n, first, d.lens, d.most, scale, ws, mask=mask, cap=cap, stream=stream())
    want, spread, _ = d.expect(q.double().numpy(), scale, 0, cap)
    small = ~large.numpy()
    S = d.expect(torch.where(large[:, None, None], torch.zeros_like(q), q).double().numpy(), scale, 0, cap)[2]
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - want)[small] <= bounds(dtype, 128, S, 512, want, spread)[small]).all()


def test_large_scores():
    run(Drafts("bf16", 2, 128, 16, [1000, 50], [5, 9], None, seed=11), 8, scale=3.0)
    run(Drafts("f32", 2, 64, 16, [1000, 50], [5, 9], None, seed=11), 8, scale=3.0)


def test_lengths_out_of_range():
    """Negative lengths are none; drafted tokens behind the last slot that a sequence can have are seen by nobody, and rows with them still see the rest."""
    for lens, counts in (([-3, 70, 1000, 2 ** 31 - 70, -2 ** 31], [2, 30, 5, 9, 4]), ([90, 96, 95], [40, 1, 2])):
        d = Drafts("bf16", 2, 64, 32, lens, counts, None, capacity=96, seed=8)
        d.base = np.clip(d.base, 0, 96)
        d.c.lens_np = d.base + d.counts
        d.c = Paged("bf16", 2, 64, 32, d.c.lens_np, capacity=96, seed=8)
        run(d, 6)


def test_tokens_that_no_sequence_has_are_left():
    counts = [4, 0, 9]
    run(Drafts("bf16", 2, 128, 16, [30, 40, 5], counts, trees(counts), seed=12), 8, tail=13)
    run(Drafts("f32", 2, 64, 16, [30, 40, 5], [0, 0, 0], None, seed=12), 8, tail=3)


def test_tokens_behind_the_most_are_left():
    d = Drafts("bf16", 2, 64, 16, [30, 40], [9, 2], None, seed=13)
    q = draw_q(d, 8).to(DEV)
    full, out = torch.empty_like(q), torch.full_like(q, -7.0)
    first = torch.from_numpy(d.first.astype(np.int32)).to(DEV)
    for most, to in ((9, full), (5, out)):
        ws = torch.empty(bs.bs_attn_tree_workspace(d.c.cache, 8, d.n, most) + 16, dtype=torch.uint8, device=DEV)
        bs.bs_attn_tree(d.c.cache, q.transpose(0, 1), to.transpose(0, 1), d.n, first, d.lens, most, 0.125, ws, stream=stream())
    assert (out[5:9] == -7.0).all()
    a, b = full.float(), out.float()
    assert torch.allclose(a[:5], b[:5], rtol=2 ** -7, atol=2 ** -14) and torch.allclose(a[9:], b[9:], rtol=2 ** -7, atol=2 ** -14)


@pytest.mark.parametrize("first", [[-5, 4, 13], [0, 4, 2 ** 31 - 1], [0, 13, 4], [9, 4, 4], [2 ** 31 - 1, -2 ** 31, 50]])
def test_firsts_that_are_no_order_stay_within_the_tokens(first):
    d = Drafts("bf16", 2, 64, 16, [30, 40], [4, 9], None, seed=14)
    q = draw_q(d, 8).to(DEV)
    guard = torch.full((d.n + 64, 8, 64), -7.0, dtype=torch.bfloat16, device=DEV)
    out = guard[32:32 + d.n]
    ws = torch.empty(bs.bs_attn_tree_workspace(d.c.cache, 8, d.n, 13) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(d.c.cache, q.transpose(0, 1), out.transpose(0, 1), d.n, torch.tensor(first, dtype=torch.int64).to(torch.int32).to(DEV), d.lens, 13, 0.125, ws, stream=stream())
    torch.cuda.synchronize()
    assert (guard[:32] == -7.0).all() and (guard[32 + d.n:] == -7.0).all()


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 28, 4, 128), ("f32", 2, 1, 64), ("bf16", 40, 2, 64)])
def test_one_token_is_a_decoding_step(dtype, hq, hkv, d):
    """The same as bs_attn_decode of the token, within both calls' tolerances."""
    lens = [1, 16, 33, 400, 0]
    x = Drafts(dtype, hkv, d, 16, lens, [1] * 5, None, seed=15)
    tree = run(x, hq)
    q = draw_q(x, hq)
    out = torch.empty_like(q, device=DEV)
    ws = torch.empty(bs.bs_attn_decode_workspace(x.c.cache, hq) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(x.c.cache, q.to(DEV).transpose(0, 1), out.transpose(0, 1), x.c.lens, d ** -0.5, ws, stream=stream())
    want, spread, S = x.expect(q.double().numpy(), d ** -0.5)
    assert (np.abs((tree.double() - out.double()).cpu().numpy()) <= 2 * bounds(dtype, d, S, 401, want, spread)).all()


def test_same_bits_again():
    counts = [26, 3, 60]
    d = Drafts("bf16", 4, 128, 16, [20000, 33, 700], counts, trees(counts), seed=12)
    a = run(d, 28)
    for i in range(3):
        assert torch.equal(a, run(d, 28, workspace_fill=i))


def test_pages_may_be_shared():
    """Two sequences with the same prefix pages."""
    d = Drafts("bf16", 2, 128, 16, [64, 64], [3, 5], None, seed=16)
    d.c.table_np[1, :4] = d.c.table_np[0, :4]
    d.c.table.copy_(torch.from_numpy(d.c.table_np))
    run(d, 8)


def test_offsets_beyond_32_bits():
    """A pool of 3 GB whose last pages are used."""
    page, hkv, dim = 16, 8, 128
    n_pages = 3 * 2 ** 30 // (page * hkv * dim * 2)
    d = Drafts("bf16", hkv, dim, page, [50], [9], trees([9]), seed=17)
    k = torch.zeros((n_pages, hkv, page, dim), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    last = np.arange(n_pages - d.c.max_pages, n_pages)
    src = torch.from_numpy(d.c.table_np[0].astype(np.int64)).to(DEV)
    k[torch.from_numpy(last).to(DEV)], v[torch.from_numpy(last).to(DEV)] = d.c.k[src], d.c.v[src]
    table = torch.from_numpy(last.astype(np.int32))[None].contiguous().to(DEV)
    before = d.c.cache
    a = run(d, 16)
    d.c.cache = bs.KVCache.of(k, v, table, bs.BS_BF16)
    assert torch.equal(a, run(d, 16))
    d.c.cache = before
