"""The calls around the KV cache together, as a model uses them: a prompt is rotated, attended and stored, tokens are decoded, the cache is cut back,
and decoding goes on; the same in a captured graph, on several streams and in several threads."""
import threading

import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, TYPES, dtype_of, stream

pytestmark = pytest.mark.gpu


class Layer:
    """One attention layer's cache and buffers for n_seqs sequences."""

    def __init__(self, n_seqs, hq, hkv, d, page, capacity, dtype="bf16", seed=0):
        self.n_seqs, self.hq, self.hkv, self.d, self.dtype = n_seqs, hq, hkv, d, dtype
        t = TYPES[dtype]
        pages = capacity // page
        g = torch.Generator()
        g.manual_seed(seed)
        self.table = torch.randperm(n_seqs * pages, generator=g).to(torch.int32).view(n_seqs, pages).to(DEV)
        self.k = torch.full((n_seqs * pages, hkv, page, d), float("nan"), dtype=t, device=DEV)
        self.v = torch.full_like(self.k, float("nan"))
        self.cache = bs.KVCache.of(self.k, self.v, self.table, dtype_of(dtype))
        self.weights = torch.zeros((n_seqs, hkv, capacity), device=DEV)
        self.order = torch.zeros((n_seqs, hkv, capacity), dtype=torch.int32, device=DEV)
        self.slots = bs.CacheSlots.of(self.weights, self.order)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
        self.position = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
        self.rope = bs.bs_rope_init(d, base=1e4)
        self.q_rot = torch.empty((n_seqs, hq, d), dtype=t, device=DEV)
        self.out = torch.empty_like(self.q_rot)
        self.ws = torch.empty(bs.bs_attn_decode_workspace(self.cache, hq, True) + 16, dtype=torch.uint8, device=DEV)

    def evict_workspace(self, keep):
        return torch.empty(bs.bs_cache_evict_workspace(self.cache, keep) + 16, dtype=torch.uint8, device=DEV)

    def step(self, q, k, v, st):
        """q, k, v: [n_seqs][heads][d] of the new tokens.  lens, position: before, then after."""
        h = lambda x: x.transpose(0, 1)
        bs.bs_cache_append(self.cache, h(k), h(v), self.n_seqs, None, self.lens, rope=self.rope, positions=self.position, q=h(q), q_out=h(self.q_rot),
                           slots=self.slots, token_order=self.position, stream=st)
        self.lens.add_(1)
        self.position.add_(1)
        bs.bs_attn_decode(self.cache, h(self.q_rot), h(self.out), self.lens, self.d ** -0.5, self.ws, slots=self.slots, slots_out=self.slots, stream=st)

    def slots_of(self, s, n):
        page = self.k.shape[2]
        j = torch.arange(n)
        p = self.table[s].cpu().long()[j // page]
        return (x.cpu()[p, :, j % page].transpose(0, 1).double() for x in (self.k, self.v))   # [head][slot][d]


def draw(n, h, d, dtype, gen):
    return torch.randn((n, h, d), generator=gen).to(TYPES[dtype]).to(DEV)


def expect(layer, s, q, keys, values):
    """q [hq][d], keys, values [hkv][n][d] in 64 bits.  Output, its tolerance (see test_gpu_attn_decode.py), and the probabilities."""
    g = layer.hq // layer.hkv
    x = torch.matmul(q.view(layer.hkv, g, -1), keys.transpose(1, 2)) * layer.d ** -0.5
    p = torch.softmax(x, -1)
    out, spread = torch.matmul(p, values), torch.matmul(p, values.abs())
    n = keys.shape[1]
    S = float((q.abs().view(layer.hkv, g, -1) @ keys.abs().transpose(1, 2)).max() * layer.d ** -0.5)
    step = (2 * layer.d * S + n + 64) * 2.0 ** -24
    tol = 2 * step * spread + (2.0 ** -16 * spread if layer.dtype == "bf16" else 0)
    tol = tol + (2.0 ** -8 if layer.dtype == "bf16" else 2.0 ** -24) * (out.abs() + tol)
    return out.flatten(0, 1), tol.flatten(0, 1), p.sum(1), 2 * step * p.sum(1) + (g + 2) * 2.0 ** -24 * p.sum(1)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_prompt_then_tokens_then_eviction(dtype, d):
    hq, hkv, L, n_new, keep = 8, 2, 333, 9, 120
    t = TYPES[dtype]
    gen = torch.Generator()
    gen.manual_seed(5)
    layer = Layer(1, hq, hkv, d, 16, 400, dtype)
    st = stream()
    # the prompt: rotate, attend (text and one picture, Dense heads), store
    q, k, v = (torch.randn((h, L, d), generator=gen).to(t).to(DEV) for h in (hq, hkv, hkv))
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    positions = torch.arange(L, dtype=torch.int32, device=DEV)
    bs.bs_rope_apply(layer.rope, [q, k], [qr, kr], dtype_of(dtype), L, d, positions, stream=st)
    tm = bs.bs_build_tilemap([(20, 220, 20)], L, [0] * hq)
    out = torch.empty_like(q)
    bs.bs_attn_prefill(qr, kr, v, out, tm, dtype_of(dtype), hq, hq // hkv, d, d ** -0.5, st)
    bs.bs_cache_append(layer.cache, k, v, L, torch.zeros(L, dtype=torch.int32, device=DEV), positions, rope=layer.rope, positions=positions,
                       slots=layer.slots, stream=st)
    layer.lens.fill_(L)
    layer.position.fill_(L)
    keys, values = layer.slots_of(0, L)
    assert torch.equal(keys, kr.cpu().double()) and torch.equal(values, v.cpu().double())
    # the last prompt row once more, through the cache
    bs.bs_attn_decode(layer.cache, qr[:, L - 1:], layer.out.transpose(0, 1), layer.lens, d ** -0.5, layer.ws, slots=layer.slots, slots_out=layer.slots, stream=st)
    want, tol, received, w_tol = expect(layer, 0, qr[:, L - 1].cpu().double(), keys, values)
    assert ((layer.out[0].cpu().double() - want).abs() <= tol).all()
    assert ((out[:, L - 1].cpu().double() - want).abs() <= tol + 2.0 ** -7 * want.abs().max()).all()
    weights, total_tol = received, w_tol
    # new tokens
    for i in range(n_new):
        q1, k1, v1 = draw(1, hq, d, dtype, gen), draw(1, hkv, d, dtype, gen), draw(1, hkv, d, dtype, gen)
        layer.step(q1, k1, v1, st)
        torch.cuda.synchronize()
        keys, values = layer.slots_of(0, L + i + 1)
        assert torch.equal(values[:, -1], v1[0].cpu().double())
        want, tol, received, w_tol = expect(layer, 0, layer.q_rot[0].cpu().double(), keys, values)
        assert ((layer.out[0].cpu().double() - want).abs() <= tol).all()
        weights = torch.cat([weights, torch.zeros((hkv, 1))], 1) + received
        total_tol = torch.cat([total_tol, torch.zeros((hkv, 1))], 1) + w_tol + 2.0 ** -24 * weights
    n = L + n_new
    got = layer.weights[0, :, :n].cpu().double()
    assert ((got - weights).abs() <= total_tol).all()
    assert abs(float(got.sum()) - hq * (n_new + 1)) < 1e-3   # every head gave each of its queries one
    assert (layer.order[0, :, :n].cpu() == torch.arange(n)).all()
    # cut back, in place
    w, o = layer.weights.cpu().numpy()[0], layer.order.cpu().numpy()[0]
    bs.bs_cache_evict(layer.cache, layer.lens, layer.lens, keep, 4, 32, layer.slots, layer.slots, layer.evict_workspace(keep), stream=st)
    torch.cuda.synchronize()
    assert layer.lens.tolist() == [keep]
    left = layer.order[0, :, :keep].cpu().numpy()
    new_keys, new_values = layer.slots_of(0, keep)
    for h in range(hkv):
        value = w[h, :n].astype(np.float64)
        value[:4], value[n - 32:] = np.inf, np.inf
        stay = np.sort(np.lexsort((np.arange(n), -value))[:keep])
        assert (np.sort(left[h]) == stay).all()
        assert torch.equal(new_keys[h], keys[h][left[h].astype(np.int64)]) and torch.equal(new_values[h], values[h][left[h].astype(np.int64)])
    # and on: positions count on, slots do not
    for i in range(3):
        q1, k1, v1 = draw(1, hq, d, dtype, gen), draw(1, hkv, d, dtype, gen), draw(1, hkv, d, dtype, gen)
        layer.step(q1, k1, v1, st)
        torch.cuda.synchronize()
        keys, values = layer.slots_of(0, keep + i + 1)
        want, tol, _, _ = expect(layer, 0, layer.q_rot[0].cpu().double(), keys, values)
        assert ((layer.out[0].cpu().double() - want).abs() <= tol).all()
        assert (layer.order[0, :, keep + i].cpu() == n + i).all()


STATE = ("k", "v", "weights", "order", "lens", "position", "out", "q_rot")


def bits(x):
    return x.view(torch.int16) if x.element_size() == 2 else x.view(torch.int32)


def fill(layer, lens, gen):
    """Tokens into an empty cache."""
    n = int(max(lens))
    seq = torch.arange(layer.n_seqs, dtype=torch.int32).repeat_interleave(n)
    slot = torch.arange(n, dtype=torch.int32).repeat(layer.n_seqs)
    slot[slot >= torch.tensor(lens, dtype=torch.int32).repeat_interleave(n)] = -1
    k, v = draw(layer.n_seqs * n, layer.hkv, layer.d, layer.dtype, gen), draw(layer.n_seqs * n, layer.hkv, layer.d, layer.dtype, gen)
    slot = slot.to(DEV)
    bs.bs_cache_append(layer.cache, k.transpose(0, 1), v.transpose(0, 1), len(slot), seq.to(DEV), slot, rope=layer.rope, positions=slot, slots=layer.slots,
                       stream=stream())
    layer.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    layer.position.copy_(layer.lens)
    torch.cuda.synchronize()


@pytest.mark.parametrize("capacity,keep,lens", [(512, 300, [300, 7, 0, 299]), (6000, 4500, [4500, 0, 4499]), (24576, 300, [299, 300, 4]), (40960, 3000, [2999] * 40)])
def test_replays_of_a_captured_step(capacity, keep, lens):
    """Append, decode and evict in one graph, replayed, with eager work between the replays, against the same steps run eagerly."""
    make = lambda: Layer(len(lens), 8, 2, 64, 16, capacity, seed=3)
    a, b = make(), make()
    for layer in (a, b):
        gen = torch.Generator()
        gen.manual_seed(8)
        fill(layer, lens, gen)
    n = len(lens)
    q, k, v = (torch.empty((n, h, 64), dtype=torch.bfloat16, device=DEV) for h in (8, 2, 2))
    ws_a, ws_b = a.evict_workspace(keep), b.evict_workspace(keep)

    def step(layer, ws, st):
        layer.step(q, k, v, st)
        bs.bs_cache_evict(layer.cache, layer.lens, layer.lens, keep, 4, 16, layer.slots, layer.slots, ws, stream=st)

    gen = torch.Generator()
    gen.manual_seed(9)
    inputs = [[draw(n, h, 64, "bf16", gen) for h in (8, 2, 2)] for _ in range(5)]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    saved = {name: getattr(a, name).clone() for name in STATE}
    for x, y in zip((q, k, v), inputs[0]):
        x.copy_(y)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):   # once before the capture
        step(a, ws_a, side.cuda_stream)
    torch.cuda.synchronize()
    for name in STATE:
        getattr(a, name).copy_(saved[name])
    torch.cuda.synchronize()
    print("capacity", capacity, flush=True)
    with torch.cuda.graph(graph, stream=side):
        step(a, ws_a, side.cuda_stream)
    for i in range(5):
        for x, y in zip((q, k, v), inputs[i]):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(b, ws_b, stream())   # eager, between the replays
        torch.cuda.synchronize()
        for name in STATE:
            assert torch.equal(bits(getattr(a, name)), bits(getattr(b, name))), (i, name)
    assert b.lens.tolist() == [min(x + 5, keep) for x in lens]


def test_streams_and_threads():
    """Layers of their own, stepped by a thread each on a stream each, give what they give one after the other."""
    lens, n_steps = [700, 3, 129], 4
    gen = torch.Generator()
    gen.manual_seed(10)
    inputs = [[draw(3, h, 128, "bf16", gen) for h in (28, 4, 4)] for _ in range(n_steps)]
    layers = [[Layer(3, 28, 4, 128, 16, 800, seed=i) for i in range(4)] for _ in range(2)]
    for group in layers:
        for layer in group:
            gen = torch.Generator()
            gen.manual_seed(11)
            fill(layer, lens, gen)
    work = [[layer.evict_workspace(500) for layer in group] for group in layers]
    torch.cuda.synchronize()

    def steps(layer, ws, st):
        with torch.cuda.stream(st):
            for x in inputs:
                layer.step(*x, st.cuda_stream)
                bs.bs_cache_evict(layer.cache, layer.lens, layer.lens, 500, 4, 16, layer.slots, layer.slots, ws, stream=st.cuda_stream)

    for layer, ws in zip(layers[0], work[0]):
        steps(layer, ws, torch.cuda.current_stream())
    torch.cuda.synchronize()
    threads = [threading.Thread(target=steps, args=(layer, ws, torch.cuda.Stream())) for layer, ws in zip(layers[1], work[1])]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    torch.cuda.synchronize()
    for one, two in zip(*layers):
        for name in STATE:
            assert torch.equal(bits(getattr(one, name)), bits(getattr(two, name))), name


def test_pages_shared_by_sequences():
    """A common prompt's pages in the tables of two sequences, and one page twice in a table: reading them needs nothing of its own."""
    layer = Layer(2, 8, 2, 64, 16, 64)
    gen = torch.Generator()
    gen.manual_seed(12)
    fill(layer, [64, 64], gen)
    layer.table[1, 0] = layer.table[0, 0]
    layer.table[1, 3] = layer.table[1, 2]
    q = draw(2, 8, 64, "bf16", gen)
    bs.bs_attn_decode(layer.cache, q.transpose(0, 1), layer.out.transpose(0, 1), layer.lens, 0.125, layer.ws, slots=layer.slots, slots_out=layer.slots, stream=stream())
    for s in range(2):
        keys, values = layer.slots_of(s, 64)
        want, tol, received, w_tol = expect(layer, s, q[s].cpu().double(), keys, values)
        assert ((layer.out[s].cpu().double() - want).abs() <= tol).all()
        assert ((layer.weights[s].cpu().double() - received).abs() <= w_tol).all()
