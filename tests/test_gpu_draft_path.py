"""The calls around drafted tokens together, as a model uses them: a step appends a tree with normed keys, attends it, and keeps the path that was accepted; after
some steps the cache holds what one token at a time would have left.  The same in a captured graph, on several streams, in several threads; a layer's training step."""
import threading

import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, TYPES, dtype_of, stream
from tree_util import bounds, tree_bits, words_of

pytestmark = pytest.mark.gpu


class Layer:
    """One attention layer's cache, weights and buffers for n_seqs sequences with `drafts` drafted tokens a step each."""

    def __init__(self, n_seqs, hq, hkv, d, page, capacity, drafts, dtype="bf16", seed=0):
        self.n_seqs, self.hq, self.hkv, self.d, self.page, self.drafts, self.dtype = n_seqs, hq, hkv, d, page, drafts, dtype
        t = TYPES[dtype]
        pages = capacity // page
        g = torch.Generator()
        g.manual_seed(seed)
        self.table = torch.randperm(n_seqs * pages, generator=g).to(torch.int32).view(n_seqs, pages).to(DEV)
        self.k = torch.full((n_seqs * pages, hkv, page, d), float("nan"), dtype=t, device=DEV)
        self.v = torch.full_like(self.k, float("nan"))
        self.cache = bs.KVCache.of(self.k, self.v, self.table, dtype_of(dtype))
        self.weights = [(torch.randn(d, generator=g) * 0.3 + 1).to(t).to(DEV) for _ in range(2)]
        self.norm = bs.Norm.of(self.weights)
        self.rope = bs.bs_rope_init(d, base=1e4)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=DEV)
        n = n_seqs * drafts
        self.first = torch.arange(0, n + 1, drafts, dtype=torch.int32, device=DEV)
        self.seq = torch.arange(n_seqs, dtype=torch.int32, device=DEV).repeat_interleave(drafts)
        self.number = torch.arange(drafts, dtype=torch.int32, device=DEV).repeat(n_seqs)
        self.q_rot = torch.empty((n, hq, d), dtype=t, device=DEV)
        self.out = torch.empty_like(self.q_rot)
        self.ws = torch.empty(bs.bs_attn_tree_workspace(self.cache, hq, n, drafts) + 16, dtype=torch.uint8, device=DEV)

    def step(self, q, k, v, depth, mask, path, n_path, st):
        """q, k, v: [token][heads][d]; depth [token] and mask [token][words] of the trees; path [seq][..], n_path [seq]: what is accepted."""
        h = lambda x: x.transpose(0, 1)
        slot = torch.index_select(self.lens, 0, self.seq) + self.number
        position = torch.index_select(self.lens, 0, self.seq) + depth
        bs.bs_cache_append_norm(self.cache, h(k), h(v), len(self.seq), self.seq, slot, self.norm, rope=self.rope, positions=position, q=h(q), q_out=h(self.q_rot), stream=st)
        bs.bs_attn_tree(self.cache, h(self.q_rot), h(self.out), len(self.seq), self.first, self.lens, self.drafts, self.d ** -0.5, self.ws, mask=mask, stream=st)
        bs.bs_cache_accept(self.cache, self.lens, self.lens, path, n_path, stream=st)

    def rows(self, s, n):
        j = torch.arange(n)
        p = self.table[s].cpu().long()[j // self.page]
        return (x.cpu()[p, :, j % self.page].transpose(0, 1).double() for x in (self.k, self.v))   # [head][slot][d]


def draw_step(layer, rng):
    """Trees, an accepted path of each from the root down, and the tokens."""
    n, m = layer.n_seqs, layer.drafts
    bits = [tree_bits(rng, m) for _ in range(n)]
    leaf = [int(rng.integers(0, m)) for _ in range(n)]
    paths = [np.flatnonzero(b[e]) for b, e in zip(bits, leaf)]
    path = np.full((n, m), -1, dtype=np.int32)
    for s, p in enumerate(paths):
        path[s, :len(p)] = p
    depth = np.concatenate([b.sum(1) - 1 for b in bits]).astype(np.int32)
    g = torch.Generator()
    g.manual_seed(int(rng.integers(0, 2 ** 31)))
    t = TYPES[layer.dtype]
    q, k, v = (torch.randn((n * m, h, layer.d), generator=g).to(t).to(DEV) for h in (layer.hq, layer.hkv, layer.hkv))
    dev = lambda x: torch.from_numpy(x).to(DEV)
    return bits, paths, (q, k, v, dev(depth), torch.cat([words_of(b, -(-m // 64)) for b in bits]).to(DEV), dev(path), dev(np.array([len(p) for p in paths], dtype=np.int32)))


@pytest.mark.parametrize("dtype,hq,hkv,d,drafts", [("bf16", 8, 2, 128, 9), ("f32", 4, 1, 64, 5), ("bf16", 16, 2, 64, 70)])
def test_steps(dtype, hq, hkv, d, drafts):
    rng = np.random.default_rng(3)
    layer = Layer(3, hq, hkv, d, 16, 512, drafts, dtype)
    keys = [torch.empty((hkv, 0, d), dtype=torch.float64) for _ in range(3)]
    values = [x.clone() for x in keys]
    for i in range(5):
        bits, paths, args = draw_step(layer, rng)
        q, k, v, depth = args[:4]
        base = [x.shape[1] for x in keys]
        layer.step(*args, stream())
        torch.cuda.synchronize()
        # what each token's K is, from the call without a cache
        kn, qn = torch.empty_like(k), torch.empty_like(q)
        h = lambda x: x.transpose(0, 1)
        position = torch.tensor(base, dtype=torch.int32, device=DEV).repeat_interleave(drafts) + depth
        bs.bs_norm_rope(layer.norm, layer.rope, [h(q), h(k)], [h(qn), h(kn)], dtype_of(dtype), 3 * drafts, d, position[None].contiguous(), stream=stream())
        assert torch.equal(qn, layer.q_rot)
        for s in range(3):
            mine = slice(s * drafts, (s + 1) * drafts)
            K = torch.cat([keys[s], kn[mine].cpu().double().transpose(0, 1)], 1)
            V = torch.cat([values[s], v[mine].cpu().double().transpose(0, 1)], 1)
            see = torch.cat([torch.ones((drafts, base[s]), dtype=torch.bool), torch.from_numpy(bits[s])], 1)
            x = torch.matmul(qn[mine].cpu().double().view(drafts, hkv, hq // hkv, d).permute(1, 2, 0, 3), K[:, None].transpose(2, 3).contiguous()) * d ** -0.5
            S = float(torch.matmul(qn[mine].cpu().double().abs().view(drafts, hkv, hq // hkv, d).permute(1, 2, 0, 3), K[:, None].abs().transpose(2, 3).contiguous()).max() * d ** -0.5)
            p = torch.softmax(torch.where(see, x, -torch.inf), -1)
            want, spread = (torch.matmul(p, y[:, None]).permute(2, 0, 1, 3).reshape(drafts, hq, d).numpy() for y in (V, V.abs()))
            got = layer.out[mine].double().cpu().numpy()
            assert (np.abs(got - want) <= bounds(dtype, d, S, base[s] + drafts, want, spread)).all()
            # the accepted path, as if only it had been there
            taken = torch.from_numpy(paths[s])
            keys[s] = torch.cat([keys[s], kn[mine].cpu().double().transpose(0, 1)[:, taken]], 1)
            values[s] = torch.cat([values[s], v[mine].cpu().double().transpose(0, 1)[:, taken]], 1)
            assert int(layer.lens[s]) == keys[s].shape[1]
            a, b = layer.rows(s, keys[s].shape[1])
            assert torch.equal(a, keys[s]) and torch.equal(b, values[s])
    # and the next token, one at a time, over what was accepted
    q = torch.randn((3, hq, d), device=DEV).to(TYPES[dtype])
    out = torch.empty_like(q)
    ws = torch.empty(bs.bs_attn_decode_workspace(layer.cache, hq) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(layer.cache, q.transpose(0, 1), out.transpose(0, 1), layer.lens, d ** -0.5, ws, stream=stream())
    assert torch.isfinite(out).all()


def test_a_step_is_captured_and_replayed():
    """One graph, replayed with other trees, lengths and paths in its buffers, eager work in between; each replay is what the calls leave."""
    rng = np.random.default_rng(5)
    eager, graphed = Layer(3, 8, 2, 128, 16, 512, 9, seed=1), Layer(3, 8, 2, 128, 16, 512, 9, seed=1)
    buffers = [x.clone() for x in draw_step(graphed, rng)[2]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # once, so that everything that a first call sets up is there
        graphed.step(*buffers, side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    graphed.lens.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(*buffers, torch.cuda.current_stream().cuda_stream)
    graphed.lens.zero_()
    for i in range(6):
        args = draw_step(graphed, rng)[2]
        for b, x in zip(buffers, args):
            b.copy_(x)
        graph.replay()
        eager.step(*args, stream())
        torch.cuda.synchronize()
        assert torch.equal(eager.out, graphed.out) and torch.equal(eager.lens, graphed.lens) and torch.equal(eager.q_rot, graphed.q_rot)
        for s in range(3):
            n = int(eager.lens[s])
            for a, b in zip(eager.rows(s, n), graphed.rows(s, n)):
                assert torch.equal(a, b)


def test_the_gradient_is_captured_and_replayed():
    d, t = 64, 300
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    rope, pos = bs.bs_rope_init(d), torch.arange(t, dtype=torch.int32, device=DEV)[None].contiguous()
    xs, dys = ([torch.randn((h, t, d), generator=gen, device=DEV) for h in (6, 2)] for _ in range(2))
    ws = [torch.rand(d, generator=gen, device=DEV) for _ in range(2)]
    norm = bs.Norm.of(ws)

    def call(to, dw, work, st):
        bs.bs_norm_rope_grad(norm, rope, xs, dys, to, dw, bs.BS_F32, t, d, pos, work, stream=st)

    def buffers():
        return [torch.empty_like(x) for x in xs], torch.empty((2, d), device=DEV), torch.empty(bs.bs_norm_rope_grad_workspace(2, bs.BS_F32, t, d), dtype=torch.uint8, device=DEV)

    a, b = buffers(), buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*a, torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for x in (*xs, *dys, *ws):
            x.normal_(generator=gen)
        graph.replay()
        call(*b, stream())
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a[0], b[0])) and torch.equal(a[1], b[1])


def test_streams_and_threads():
    """Four layers, each in a thread of its own with a stream of its own, give what they give one behind the other."""
    def work(i, st, out):
        rng = np.random.default_rng(20 + i)
        layer = Layer(2, 8, 2, 64, 16, 512, 6 + 7 * i, seed=i)
        with torch.cuda.stream(st):
            for _ in range(4):
                layer.step(*draw_step(layer, rng)[2], st.cuda_stream)
            st.synchronize()
        out[i] = (layer.out.clone(), layer.lens.clone(), layer.k.clone().view(torch.int16))

    one, many = {}, {}
    for i in range(4):
        work(i, torch.cuda.Stream(), one)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i, torch.cuda.Stream(), many)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(4):
        assert all(torch.equal(a, b) for a, b in zip(one[i], many[i]))


def test_a_training_step():
    """Queries and keys of a layer through bs_norm_rope as a torch function: its gradients are those of the same layer in plain torch, in 64 bits."""
    d, t, hq, hkv = 64, 40, 4, 2
    rope = bs.bs_rope_init(d)
    pos = torch.arange(t, dtype=torch.int32, device=DEV)[None].contiguous()
    freq = torch.tensor(list(rope.freq[:d // 2]), dtype=torch.float64)

    class NormRope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, wq, wk):
            ctx.save_for_backward(q, k, wq, wk)
            out = [torch.empty_like(q), torch.empty_like(k)]
            bs.bs_norm_rope(bs.Norm.of([wq, wk]), rope, [q, k], out, bs.BS_F32, t, d, pos, stream=stream())
            return tuple(out)

        @staticmethod
        def backward(ctx, dq, dk):
            q, k, wq, wk = ctx.saved_tensors
            out, dw = [torch.empty_like(q), torch.empty_like(k)], torch.empty((2, d), device=DEV)
            ws = torch.empty(bs.bs_norm_rope_grad_workspace(2, bs.BS_F32, t, d), dtype=torch.uint8, device=DEV)
            bs.bs_norm_rope_grad(bs.Norm.of([wq, wk]), rope, [q, k], [dq.contiguous(), dk.contiguous()], out, dw, bs.BS_F32, t, d, pos, ws, stream=stream())
            return out[0], out[1], dw[0], dw[1]

    def plain(x, w):
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(np.float32(1e-6))) * w
        angle = torch.arange(t, dtype=torch.float64)[:, None] * freq
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * torch.cos(angle) - b * torch.sin(angle), b * torch.cos(angle) + a * torch.sin(angle)], -1)

    g = torch.Generator()
    g.manual_seed(4)
    leaves = [torch.randn(s, generator=g) for s in ((hq, t, d), (hkv, t, d), (d,), (d,))]
    target = torch.randn((hq, t, t), generator=g)
    got = [x.to(DEV).requires_grad_() for x in leaves]
    want = [x.double().requires_grad_() for x in leaves]

    def loss(q, k, target):
        return (torch.softmax(torch.matmul(q, k.repeat_interleave(hq // hkv, 0).transpose(1, 2).contiguous()) * d ** -0.5, -1) * target).sum()

    loss(*NormRope.apply(*got), target.to(DEV)).backward()
    loss(plain(want[0], want[2]), plain(want[1], want[3]), target.double()).backward()
    for a, b in zip(got, want):   # (scores, softmax and their gradients around it are torch's, in fp32: a few hundred steps of 2^-24 of the largest)
        assert (a.grad.cpu().double() - b.grad).abs().max() <= 1e-4 * b.grad.abs().max()
