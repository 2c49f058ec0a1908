"""Attention of drafted tokens on the paths that set its kernels apart, each at every number of rows that has a kernel of its own: capped scores, windows and pages that
are not there together, and values that only some rows see (tolerances: tree_util.bounds)."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, stream
from tree_util import Drafts, draw_q, run, tree_bits, words_of

pytestmark = pytest.mark.gpu

# rows of a sequence and KV head: up to 16, 32, 128 and beyond, in fp32 also up to 64
ROWS = [("bf16", 3, 5), ("bf16", 4, 8), ("bf16", 7, 15), ("bf16", 8, 26), ("f32", 2, 7), ("f32", 3, 9), ("f32", 6, 10), ("f32", 5, 25), ("f32", 8, 20)]


def trees(counts, seed=0):
    rng = np.random.default_rng([21, seed])
    return [tree_bits(rng, n) for n in counts]


@pytest.mark.parametrize("dtype,G,most", ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,scale", [(50.0, None), (1.5, None), (0.01, 1.0)])
def test_capped_scores(dtype, G, most, d, cap, scale):
    counts = [3, most, 1]
    run(Drafts(dtype, 2, d, 16, [400, 33, 90], counts, trees(counts), seed=30), 2 * G, cap=cap, scale=scale)


@pytest.mark.parametrize("dtype,G,most", ROWS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [5, 33, 200])
def test_cap_window_and_missing_pages(dtype, G, most, d, window):
    counts, lens = [most, 2, 1, max(1, most // 2)], [901, 0, 64, 131]
    for bits in (trees(counts, 1), None):
        run(Drafts(dtype, 2, d, 16, lens, counts, bits, seed=31, bad=0.3), 2 * G, window=window, cap=4.0)


@pytest.mark.parametrize("dtype,G", [("bf16", 4), ("f32", 3), ("f32", 4), ("f32", 8)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_values_that_only_some_rows_see(dtype, G, d, cap, value):
    """A drafted token's V that is not finite reaches the rows that see it and no others; 80 to 160 rows of the second sequence among them."""
    counts, lens, hq = [12, 20], [37, 5], 2 * G
    bits = trees(counts, 3)
    x = Drafts(dtype, 2, d, 16, lens, counts, bits, seed=9)
    clean = run(x, hq, cap=cap)
    for s, a in ((0, 4), (1, 7)):
        j = lens[s] + a
        x.c.v[x.c.table_np[s, j // 16], :, j % 16, 5] = value
    q = draw_q(x, hq).to(DEV)
    out = torch.empty_like(q)
    mask = torch.cat([words_of(b, 1) for b in bits]).to(DEV)
    ws = torch.empty(bs.bs_attn_tree_workspace(x.c.cache, hq, x.n, x.most) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(x.c.cache, q.transpose(0, 1), out.transpose(0, 1), x.n, torch.from_numpy(x.first.astype(np.int32)).to(DEV), x.lens, x.most, d ** -0.5, ws, mask=mask, cap=cap,
                    stream=stream())
    sees = np.concatenate([bits[0][:, 4], bits[1][:, 7]])
    assert 0 < sees.sum() < x.n
    sees = torch.from_numpy(sees).to(DEV)
    assert torch.equal(out[~sees], clean[~sees])
    assert not torch.isfinite(out[sees][..., 5]).any()
