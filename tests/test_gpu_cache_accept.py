"""Accepted drafted tokens move together behind their sequence: exact, against numpy."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, Paged, stream

pytestmark = pytest.mark.gpu


def expect(c, lens, path, n_path, k, v, w, o):
    """The pools [page][head][slot][d] and rows [seq][head][slot] behind the call; new lengths."""
    k, v, w, o = k.clone(), v.clone(), w.clone(), o.clone()
    k0, v0, w0, o0 = k.clone(), v.clone(), w.clone(), o.clone()
    out = []
    for s in range(len(lens)):
        n = int(np.clip(lens[s], 0, c.slots))
        m = int(np.clip(n_path[s], 0, path.shape[1]))
        for i in range(m):
            p = int(path[s, i])
            if not 0 <= p < 256 or n + p >= c.slots or n + i >= c.slots:
                continue
            src, dst = c.table_np[s, (n + p) // c.page], c.table_np[s, (n + i) // c.page]
            if not (0 <= src < c.n_pages and 0 <= dst < c.n_pages):
                continue
            k[dst, :, (n + i) % c.page], v[dst, :, (n + i) % c.page] = k0[src, :, (n + p) % c.page], v0[src, :, (n + p) % c.page]
            w[s, :, n + i], o[s, :, n + i] = w0[s, :, n + p], o0[s, :, n + p]
        out.append(min(n + m, c.slots))
    return k, v, w, o, out


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))   # bits: NaN is NaN


def run(c, lens, path, n_path, in_place=False, what="wo", seed=0):
    lens, path, n_path = np.asarray(lens, dtype=np.int64), np.asarray(path, dtype=np.int64), np.asarray(n_path, dtype=np.int64)
    g = torch.Generator()
    g.manual_seed(seed)
    rows = (len(lens), c.hkv, c.slots + 5)
    w, o = torch.rand(rows, generator=g), torch.randint(-9, 10 ** 6, rows, generator=g, dtype=torch.int32)
    dev = lambda x: torch.from_numpy(x.astype(np.int32)).to(DEV)
    lens_d, path_d, n_d, w_d, o_d = dev(lens), dev(path), dev(n_path), w.to(DEV), o.to(DEV)
    out = lens_d if in_place else torch.full_like(lens_d, -5)
    slots = None if not what else bs.CacheSlots.of(w_d if "w" in what else None, o_d if "o" in what else None)
    bs.bs_cache_accept(c.cache, lens_d, out, path_d, n_d, slots=slots, stream=stream())
    torch.cuda.synchronize()
    k, v, w1, o1, n = expect(c, lens, path, n_path, c.k_np, c.v_np, w, o)
    assert out.tolist() == n
    assert same(c.k.cpu(), k) and same(c.v.cpu(), v)
    assert same(w_d.cpu(), w1 if "w" in what else w) and same(o_d.cpu(), o1 if "o" in what else o)


def paths(rng, seqs, most, drafts):
    """Ascending, as a tree's are."""
    n = rng.integers(0, most + 1, seqs)
    path = np.full((seqs, most), -1)
    for s in range(seqs):
        path[s, :n[s]] = np.sort(rng.choice(drafts, n[s], replace=False))
    return path, n


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 256), ("bf16", 72), ("f32", 8), ("bf16", 8), ("bf16", 256)])
@pytest.mark.parametrize("page,pool", [(16, "heads"), (48, "slots")])
@pytest.mark.parametrize("most,drafts", [(1, 1), (4, 8), (12, 64), (100, 256), (256, 256)])
def test_paths(dtype, d, page, pool, most, drafts):
    rng = np.random.default_rng([most, d])
    lens = np.array([0, 1, 15, 16, 17, 250])
    path, n = paths(rng, len(lens), most, drafts)
    n[-1] = most
    path[-1] = np.sort(rng.choice(drafts, most, replace=False))
    run(Paged(dtype, 3, d, page, lens, pool=pool, more=drafts, seed=most), lens, path, n, in_place=most % 2 == 1)


@pytest.mark.parametrize("what", ["", "w", "o", "wo"])
def test_weights_and_order_move_along(what):
    run(Paged("bf16", 2, 64, 16, [40, 7], more=20), [40, 7], [[0, 5, 9], [3, 4, 19]], [3, 2], what=what)


def test_any_path():
    """Not ascending, the same token more than once, forwards and back, longer than the accepted part."""
    rng = np.random.default_rng(4)
    path = rng.integers(0, 30, (5, 40))
    run(Paged("bf16", 2, 128, 16, [3, 90, 17, 16, 0], more=40), [3, 90, 17, 16, 0], path, [40, 3, 0, 17, 39])


def test_entries_that_are_no_tokens_and_counts_out_of_range():
    path = [[-1, 3, 2 ** 31 - 1, 1], [5, 256, 2, -2 ** 31], [1, 2, 3, 4], [0, 3, 6, 2], [4, 3, 2, 1]]
    run(Paged("f32", 2, 64, 16, [20, 3, 70, 5, 0], more=10), [20, 3, 70, 5, 0], path, [4, 2 ** 31 - 1, -1, -2 ** 31, 4])


def test_slots_without_a_page_and_behind_the_last():
    c = Paged("bf16", 2, 64, 16, [20, 33, 100, 64], bad=0.5, more=30, seed=3)
    rng = np.random.default_rng(5)
    run(c, [20, 33, 100, 64], rng.integers(0, 60, (4, 30)), [30, 30, 30, 30])
    run(Paged("bf16", 2, 64, 16, [90, 96, 80], capacity=96, more=20), [90, 96, 80], rng.integers(0, 40, (3, 20)), [20, 20, 20], in_place=True)


def test_lengths_out_of_range():
    c = Paged("bf16", 2, 64, 32, [0, 70, 0], capacity=96, more=9, seed=8)
    run(c, [-3, 2 ** 31 - 1, -2 ** 31], [[2, 1, 5]] * 3, [3, 3, 3])


def test_no_path():
    c = Paged("bf16", 2, 64, 16, [5, 6])
    lens, out = c.lens.clone(), torch.zeros_like(c.lens)
    bs.bs_cache_accept(c.cache, lens, out, torch.zeros((2, 0), dtype=torch.int32, device=DEV), torch.tensor([3, 0], dtype=torch.int32, device=DEV), stream=stream())
    assert out.tolist() == [5, 6]


def test_many_sequences():
    rng = np.random.default_rng(6)
    lens = rng.integers(0, 60, 700)
    path, n = paths(rng, 700, 7, 12)
    run(Paged("bf16", 2, 64, 16, lens, more=12), lens, path, n, in_place=True)
