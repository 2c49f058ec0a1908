"""Attention of one token where the values cancel, so that what a probability loses before P V shows in the result.

Every query row has one channel that is not zero, so its scores are products of two bf16 numbers, exact in fp32.  Per head, in a channel of its own, the
values of three slots are chosen so that p1 v1 + p0 v0 + p2 v2 vanishes up to some 2^-18: v1 = 1, v0 = -bf16(p1), v2 = -bf16((p1 - bf16(p1)) / p2), p0 = 1.

Tolerance per element, with A = sum p |v| before the division by the sum l of the probabilities:
  the exponent x = score * scale * log2(e): two roundings (the constant, the product), 2^-24 |x| each; the reference point is the score 0, exact;
  the exponential: one step, 2^-23;
  P V in fp32: the products of bf16 numbers are exact; each of the at most three additions of a slot's parts is off by at most a step of the running sum,
  2^-23 A: 6 2^-24 A;
  l, its reciprocal and the last product are off relative to the result: (n + 6) 2^-24 |out|; the result is rounded once, 2^-8 |out| at most."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, stream

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.tensor(x, dtype=torch.float64).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("d,hq", [(64, 16), (128, 16), (128, 32), (64, 40)])
@pytest.mark.parametrize("tail", [0, 29, 300])   # slots behind the three, with values of zero: one wave has all, all waves have some
def test_values_that_cancel(d, hq, tail):
    print(d, hq, tail, flush=True)
    n, page = 3 + tail, 16
    pages = -(-n // page)
    q = np.zeros((hq, d))
    q[:, 0] = bf16(0.9 + 0.4 * np.arange(hq) / hq)
    k, v = np.zeros((pages * page, d)), np.zeros((pages * page, d))
    k[:3, 0] = bf16(np.array([0.0, -0.31, -5.4]))
    k[3:n, 0] = -7.0
    score = q @ k[:n].T
    p = np.exp(score)   # (the largest score is 0)
    for h in range(hq):
        c = h % d
        v[1, c] = 1.0
        v[0, c] = -bf16(p[h, 1])
        v[2, c] = -bf16((p[h, 1] + v[0, c]) / p[h, 2])
    total = p.sum(1, keepdims=True)
    want, spread = p @ v[:n] / total, p @ np.abs(v[:n]) / total
    x = np.abs(score) * 1.4427
    moved = (p * (2 * x + 2)) @ np.abs(v[:n]) / total * 2.0 ** -24
    tol = moved + 6 * 2.0 ** -24 * spread + (n + 6) * 2.0 ** -24 * np.abs(want)
    tol = tol + HALF_STEP["bf16"] * (np.abs(want) + tol)
    dev = lambda a: torch.from_numpy(a).to(torch.bfloat16).to(DEV)
    pool = lambda a: dev(a).view(pages, page, 1, d).transpose(1, 2)
    kd, vd = pool(k), pool(v)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous()
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    cache = bs.KVCache.of(kd, vd, table, bs.BS_BF16)
    qd = dev(q).view(hq, 1, d)
    out = torch.empty_like(qd)
    ws = torch.empty(bs.bs_attn_decode_workspace(cache, hq) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(cache, qd, out, lens, 1.0, ws, stream=stream())
    off = np.abs(out[:, 0].double().cpu().numpy() - want)
    own = np.arange(hq), np.arange(hq) % d
    assert (np.abs(want[own]) < 2.0 ** -15).all()   # (they do cancel)
    print("largest error in parts of the bound", float((off / np.maximum(tol, 1e-30)).max()), "of the sum", float((off[own] / spread[own]).max()), flush=True)
    assert (off <= tol).all()
