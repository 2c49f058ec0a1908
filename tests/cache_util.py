"""A paged KV cache for tests: pools in either order of axes, everything that no sequence uses filled with NaN, and plain forms in 64 bits."""
import numpy as np
import torch

import paper_2507_09071_amd as bs

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # relative error of a rounding


def dtype_of(t):
    return bs.BS_BF16 if t == "bf16" else bs.BS_F32


def stream():
    return torch.cuda.current_stream().cuda_stream


class Paged:
    """capacity: slots a sequence may have (whole pages)."""

    def __init__(self, dtype, hkv, d, page, lens, capacity=None, pool="heads", seed=0, bad=0.0, more=0):
        rng = np.random.default_rng([5, seed])
        self.dtype, self.hkv, self.d, self.page, self.lens_np = dtype, hkv, d, page, np.asarray(lens, dtype=np.int64)
        n_seqs = len(lens)
        capacity = max(int(self.lens_np.max()) + more, 1) if capacity is None else capacity
        self.max_pages = -(-capacity // page)
        self.slots = self.max_pages * page
        used = np.clip(self.lens_np + more, 0, self.slots)
        need = -(-used // page)
        n_pages = int(need.sum()) + 2
        ids = rng.permutation(n_pages)[:int(need.sum())]
        table = np.full((n_seqs, self.max_pages), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = ids[at:at + n]
            at += n
        if bad:   # some of the pages in use are none
            hit = (rng.random(table.shape) < bad) & (table >= 0)
            table[hit] = rng.choice([-1, -7, n_pages, n_pages + 5, 2 ** 31 - 1, -2 ** 31], size=int(hit.sum()))
        self.table_np, self.n_pages = table, n_pages
        g = torch.Generator()
        g.manual_seed(seed + 1)
        t = TYPES[dtype]
        self.k_np = torch.randn((n_pages, hkv, page, d), generator=g).to(t)
        self.v_np = torch.randn((n_pages, hkv, page, d), generator=g).to(t)
        mine = torch.zeros((n_pages, page), dtype=torch.bool)   # slots that some sequence has
        for s in range(n_seqs):
            for j in range(int(np.clip(self.lens_np[s], 0, self.slots))):
                p = table[s, j // page]
                if 0 <= p < n_pages:
                    mine[p, j % page] = True
        hole = ~mine[:, None, :, None]
        self.k_np = torch.where(hole, torch.tensor(float("nan"), dtype=t), self.k_np)
        self.v_np = torch.where(hole, torch.tensor(float("inf"), dtype=t), self.v_np)
        view = lambda x: x.to(DEV) if pool == "heads" else x.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
        self.k, self.v = view(self.k_np), view(self.v_np)
        self.table = torch.from_numpy(table).to(DEV)
        self.lens = torch.from_numpy(self.lens_np.astype(np.int32)).to(DEV)
        self.cache = bs.KVCache.of(self.k, self.v, self.table, dtype_of(dtype))

    def used(self, s):
        return int(np.clip(self.lens_np[s], 0, self.slots))

    def rows(self, s, h):
        """K and V of the sequence's slots in 64 bits, and which of them have a page."""
        j = np.arange(self.used(s))
        p = self.table_np[s, j // self.page].astype(np.int64)
        there = (p >= 0) & (p < self.n_pages)
        p = np.where(there, p, 0)
        k, v = (x[torch.from_numpy(p), h, torch.from_numpy(j % self.page)].double().numpy() for x in (self.k_np, self.v_np))
        return k, v, there


def attention(cache, q, scale, window):
    """q [n_seqs][n_q_heads][d] (64 bits).  out; sum p |v| per element; probabilities per sequence and head; largest sum |q k| scale."""
    n_seqs, hq, d = q.shape
    out, spread, probs, largest = np.zeros(q.shape), np.zeros(q.shape), {}, 0.0
    for s in range(n_seqs):
        n = cache.used(s)
        for h in range(hq):
            k, v, there = cache.rows(s, h * cache.hkv // hq)
            see = there & (np.arange(n) >= (n - window if window else 0))
            p = np.zeros(n)
            if see.any():
                x = (k[see] @ q[s, h]) * scale
                e = np.exp(x - x.max())
                p[see] = e / e.sum()
                out[s, h], spread[s, h] = p[see] @ v[see], p[see] @ np.abs(v[see])
                largest = max(largest, float((np.abs(k[see]) @ np.abs(q[s, h])).max() * scale))
            probs[s, h] = p
    return out, spread, probs, largest
