"""Drafted tokens for tests: trees and other masks, and attention over a paged cache in 64 bits."""
import numpy as np
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, TYPES, Paged, stream


def tree_bits(rng, n):
    """bool [n][n]: what a token of a random tree sees of the tokens."""
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if i:
            see[i] = see[i - 1 if rng.random() < 0.5 else rng.integers(0, i)]
        see[i, i] = True
    return see


def words_of(bits, words):
    """bool [n][m] -> int64 [n][words]."""
    out = np.zeros((bits.shape[0], words), dtype=np.uint64)
    for a in range(bits.shape[1]):
        out[:, a // 64] |= bits[:, a].astype(np.uint64) << np.uint64(a % 64)
    return torch.from_numpy(out.view(np.int64))


class Drafts:
    """A cache whose sequences have `lens` slots and behind them `counts` drafted tokens.  bits: a list of bool [count][count], or None: chains."""

    def __init__(self, dtype, hkv, d, page, lens, counts, bits=None, capacity=None, pool="heads", seed=0, bad=0.0):
        self.base, self.counts, self.bits = np.asarray(lens, dtype=np.int64), np.asarray(counts, dtype=np.int64), bits
        self.c = Paged(dtype, hkv, d, page, self.base + self.counts, capacity=capacity, pool=pool, seed=seed, bad=bad)
        self.first = np.concatenate([[0], np.cumsum(self.counts)])
        self.n = int(self.first[-1])
        self.most = int(max(1, self.counts.max()))
        self.lens = torch.from_numpy(self.base.astype(np.int32)).to(DEV)

    def sees(self, s, window):
        """bool [count][slots in use]: what each drafted token of a sequence sees, pages apart."""
        c, n, t = self.c, self.c.used(s), int(self.counts[s])
        base = int(np.clip(self.base[s], 0, c.slots))
        see = np.zeros((t, base + t), dtype=bool)
        see[:, :base] = True
        see[:, base:] = np.tril(np.ones((t, t), dtype=bool)) if self.bits is None else self.bits[s]
        if window:
            for r in range(t):
                see[r, np.flatnonzero(see[r])[:-window]] = False
        return see[:, :n]

    def expect(self, q, scale, window=0, cap=0.0):
        """q [tokens][heads][d], 64 bits: out, sum p |v|, the largest sum |q k| scale."""
        out, spread, largest = np.zeros(q.shape), np.zeros(q.shape), 0.0
        c, hq = self.c, q.shape[1]
        for s in range(len(self.counts)):
            mine = slice(self.first[s], self.first[s + 1])
            see = self.sees(s, window)
            for h in range(c.hkv):
                k, v, there = c.rows(s, h)
                k, v, there = k[:see.shape[1]], v[:see.shape[1]], there[:see.shape[1]]
                k0, v0 = np.where(np.isfinite(k), k, 0.0), np.where(np.isfinite(v), v, 0.0)
                for e in range(h * hq // c.hkv, (h + 1) * hq // c.hkv):
                    x = q[mine, e] @ k0.T * scale
                    largest = max(largest, float((np.abs(q[mine, e]) @ np.abs(k0).T).max(initial=0.0) * scale))
                    if cap:
                        x = cap * np.tanh(x / cap)
                    x = np.where(see & there, x, -np.inf)
                    m = x.max(axis=1, keepdims=True, initial=-np.inf)
                    p = np.exp(x - np.where(np.isfinite(m), m, 0.0))
                    total = p.sum(axis=1, keepdims=True)
                    p = p / np.where(total > 0, total, 1.0)
                    out[mine, e], spread[mine, e] = p @ v0, p @ np.abs(v0)
        return out, spread, largest


def bounds(dtype, d, S, n, out, spread):
    """Tolerance per element, with A = sum_j p_j |v_j|, S = the largest sum |q k| scale, n = the longest sequence:
      scores are sums of d products in fp32, off by at most d 2^-24 S; capped, by 8 steps of 2^-24 more; a probability changes by twice that, relatively;
      sums over slots: at most n roundings of 2^-24; exponentials, reference points and the joining of parts: 64 steps;
      bf16: each probability is the sum of two bf16 numbers, off by at most 2^-8 of the second, which is at most 2^-8 of the whole: 2^-16 A;
      the result is rounded once."""
    tol = (2 * (d + 8) * S + n + 64) * 2.0 ** -24 * 2 * spread
    if dtype == "bf16":
        tol = tol + 2.0 ** -16 * spread
    return tol + HALF_STEP[dtype] * (np.abs(out) + tol)


def draw_q(drafts, hq, tail=0, seed=0):
    g = torch.Generator()
    g.manual_seed(300 + seed)
    return torch.randn((drafts.n + tail, hq, drafts.c.d), generator=g).to(TYPES[drafts.c.dtype])


def run(drafts, hq, window=0, cap=0.0, scale=None, token_major=True, tail=0, most=None, words=None, seed=0, first=None, workspace_fill=0xff):
    """The call, and its comparison.  tail: tokens behind the last sequence; most: max_tokens; words: of the mask."""
    c = drafts.c
    scale = c.d ** -0.5 if scale is None else scale
    most = drafts.most if most is None else most
    q = draw_q(drafts, hq, tail, seed)
    dev = q.to(DEV) if token_major else q.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    out = torch.full_like(dev, -7.0)
    mask = None
    if drafts.bits is not None:
        words = -(-most // 64) if words is None else words
        mask = torch.cat([words_of(b, words) for b in drafts.bits] + [torch.full((tail, words), -1)]).to(DEV)
    first = torch.from_numpy((drafts.first if first is None else first).astype(np.int32)).to(DEV)
    n = drafts.n + tail
    ws = torch.full((bs.bs_attn_tree_workspace(c.cache, hq, n, most) + 16,), workspace_fill, dtype=torch.uint8, device=DEV)
    bs.bs_attn_tree(c.cache, dev.transpose(0, 1), out.transpose(0, 1), n, first, drafts.lens, most, scale, ws, mask=mask, window=window, cap=cap, stream=stream())
    torch.cuda.synchronize()
    want, spread, S = drafts.expect(q[:drafts.n].double().numpy(), scale, window, cap)
    got = out.double().cpu().numpy()
    assert (got[drafts.n:] == -7.0).all()   # tokens that no sequence has
    got = got[:drafts.n]
    assert np.isfinite(got).all()
    longest = int(max(c.used(s) for s in range(len(drafts.counts))))
    tol = bounds(c.dtype, c.d, S, longest, want, spread)
    worst = np.abs(got - want) - tol
    assert (worst <= 0).all(), (float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))
    return out
