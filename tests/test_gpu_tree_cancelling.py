"""Attention of drafted tokens where the values cancel, so that what a probability loses before P V shows in the result.

Every query row has one channel that is not zero, so its scores are products of two bf16 numbers, exact in fp32.  Per row, in a channel of its own (rows that share
one are alike), the values of three slots are chosen so that p1 v1 + p0 v0 + p2 v2 vanishes up to some 2^-18 (fp32: up to 2^-24): v1 = 1, v0 = -bf16(p1),
v2 = -bf16((p1 - bf16(p1)) / p2), p0 = 1; fp32: v0 = -p1, v2 = 0.  All other slots, those of the drafted tokens too, have values of zero.

Tolerance per element, with A = sum p |v| before the division by the sum l of the probabilities:
  the exponent x = score * scale * log2(e): two roundings (the constant, the product), 2^-24 |x| each; capped, eight in their place: the factors and the products on
  both sides of the tanh, and four for the tanh itself; the reference point is the score 0, exact;
  the exponential: one step, 2^-23;
  P V in fp32: the products of bf16 numbers are exact, and a value of fp32 is used as it is, its product rounded with the sum; each of the at most three additions of a
  slot's parts is off by at most a step of the running sum, 2^-23 A: 6 2^-24 A;
  l, its reciprocal and the last product are off relative to the result: (n + 6) 2^-24 |out|; the result is rounded once."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, TYPES, dtype_of, stream

pytestmark = pytest.mark.gpu


def rounded(x, dtype):
    return torch.tensor(x, dtype=torch.float64).to(TYPES[dtype]).double().numpy()


# (rows of a sequence and KV head: up to 16, 32, 128 and beyond, in fp32 also up to 64)
@pytest.mark.parametrize("dtype,d,G,T", [("bf16", 64, 16, 1), ("bf16", 128, 4, 3), ("bf16", 64, 6, 5), ("bf16", 128, 8, 4), ("bf16", 64, 7, 9), ("bf16", 128, 5, 16),
                                         ("bf16", 128, 16, 8), ("bf16", 128, 7, 26), ("bf16", 64, 8, 40), ("f32", 64, 2, 5), ("f32", 128, 8, 3), ("f32", 128, 8, 7),
                                         ("f32", 64, 10, 12)])
@pytest.mark.parametrize("cap", [0.0, 50.0])
@pytest.mark.parametrize("tail", [0, 29, 300, 5000])   # slots behind the three: one wave has all, all waves have some, many workgroups have some
def test_values_that_cancel(dtype, d, G, T, cap, tail):
    print(dtype, d, G, T, cap, tail, flush=True)
    base, page = 3 + tail, 16
    n, rows = base + T, G * T
    pages = -(-n // page)
    q = np.zeros((rows, d))
    own = np.arange(rows) % d
    q[:, 0] = rounded(0.9 + 0.4 * own / d, "bf16")
    k, v = np.zeros((pages * page, d)), np.zeros((pages * page, d))
    k[:3, 0] = rounded(np.array([0.0, -0.31, -5.4]), "bf16")
    k[3:n, 0] = -7.0
    score = q @ k[:n].T
    x = cap * np.tanh(score / cap) if cap else score
    see = np.arange(n)[None] <= base + np.arange(rows)[:, None] // G   # a chain
    p = np.where(see, np.exp(x), 0.0)   # (the largest score is 0)
    for r in range(rows):
        c = own[r]
        v[1, c] = 1.0
        v[0, c] = -rounded(p[r, 1], dtype)
        v[2, c] = -rounded((p[r, 1] + v[0, c]) / p[r, 2], "bf16") if dtype == "bf16" else 0.0
    total = p.sum(1, keepdims=True)
    want, spread = p @ v[:n] / total, p @ np.abs(v[:n]) / total
    moved = (p * ((8 if cap else 2) * np.abs(x) * 1.4427 + 2)) @ np.abs(v[:n]) / total * 2.0 ** -24
    tol = moved + 6 * 2.0 ** -24 * spread + (n + 6) * 2.0 ** -24 * np.abs(want)
    tol = tol + HALF_STEP[dtype] * (np.abs(want) + tol)
    dev = lambda a: torch.from_numpy(a).to(TYPES[dtype]).to(DEV)
    pool = lambda a: dev(a).view(pages, page, 1, d).transpose(1, 2)
    kd, vd = pool(k), pool(v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous()
    cache = bs.KVCache.of(kd, vd, table, dtype_of(dtype))
    lens, first = torch.tensor([base], dtype=torch.int32, device=DEV), torch.tensor([0, T], dtype=torch.int32, device=DEV)
    qd = dev(q).view(T, G, d)
    out = torch.empty_like(qd)
    ws = torch.empty(bs.bs_attn_tree_workspace(cache, G, T, T) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(cache, qd.transpose(0, 1), out.transpose(0, 1), T, first, lens, T, 1.0, ws, cap=cap, stream=stream())
    off = np.abs(out.view(rows, d).double().cpu().numpy() - want)
    mine = np.arange(rows), own
    assert (np.abs(want[mine]) < (2.0 ** -15 if dtype == "bf16" else 2.0 ** -23)).all()   # (they do cancel)
    print("largest error in parts of the bound", float((off / np.maximum(tol, 1e-30)).max()), "of the sum", float((off[mine] / spread[mine]).max()), flush=True)
    assert (off <= tol).all()
