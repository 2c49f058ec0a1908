"""What drafted steps leave in the cache, as a step of one token each sees it; and steps on several streams, each layer made on the stream that uses it."""
import threading

import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, TYPES, dtype_of, stream
from test_gpu_draft_path import Layer, draw_step
from tree_util import bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d,drafts", [("bf16", 8, 2, 128, 9), ("f32", 4, 1, 64, 5), ("bf16", 16, 2, 64, 40)])
def test_the_next_token_sees_what_was_accepted(dtype, hq, hkv, d, drafts):
    rng = np.random.default_rng(31)
    layer = Layer(3, hq, hkv, d, 16, 512, drafts, dtype, seed=5)
    keys = [torch.empty((hkv, 0, d), dtype=torch.float64) for _ in range(3)]
    values = [x.clone() for x in keys]
    h = lambda x: x.transpose(0, 1)
    for _ in range(6):
        _, paths, args = draw_step(layer, rng)
        k, v, depth = args[1:4]
        position = torch.tensor([x.shape[1] for x in keys], dtype=torch.int32, device=DEV).repeat_interleave(drafts) + depth
        kn = torch.empty_like(k)
        bs.bs_norm_rope(bs.Norm.of(layer.weights[1:]), layer.rope, [h(k)], [h(kn)], dtype_of(dtype), 3 * drafts, d, position[None].contiguous(), stream=stream())
        layer.step(*args, stream())
        for s in range(3):
            mine, taken = slice(s * drafts, (s + 1) * drafts), torch.from_numpy(paths[s])
            keys[s] = torch.cat([keys[s], h(kn[mine].cpu().double())[:, taken]], 1)
            values[s] = torch.cat([values[s], h(v[mine].cpu().double())[:, taken]], 1)
    g = torch.Generator()
    g.manual_seed(8)
    q = torch.randn((3, hq, d), generator=g).to(TYPES[dtype]).to(DEV)
    out = torch.empty_like(q)
    ws = torch.empty(bs.bs_attn_decode_workspace(layer.cache, hq) + 16, dtype=torch.uint8, device=DEV)
    bs.bs_attn_decode(layer.cache, h(q), h(out), layer.lens, d ** -0.5, ws, stream=stream())
    torch.cuda.synchronize()
    for s in range(3):
        assert int(layer.lens[s]) == keys[s].shape[1]
        x = q[s].cpu().double().view(hkv, hq // hkv, d)
        scores, sizes = (torch.matmul(a, b.transpose(1, 2).contiguous()) * d ** -0.5 for a, b in ((x, keys[s]), (x.abs(), keys[s].abs())))
        p = torch.softmax(scores, -1)
        want, spread = (torch.matmul(p, y).reshape(hq, d).numpy() for y in (values[s], values[s].abs()))
        assert (np.abs(out[s].double().cpu().numpy() - want) <= bounds(dtype, d, float(sizes.max()), keys[s].shape[1], want, spread)).all()


def test_streams_and_threads():
    """Four layers, each made and stepped on a stream of its own in a thread of its own, give what they give one behind the other."""
    def work(i, st, out):
        rng = np.random.default_rng(50 + i)
        with torch.cuda.stream(st):
            layer = Layer(2, 8, 2, 64, 16, 512, 6 + 7 * i, seed=i)
            for _ in range(4):
                layer.step(*draw_step(layer, rng)[2], st.cuda_stream)
            out[i] = (layer.out.clone(), layer.lens.clone(), layer.k.clone().view(torch.int16))
            st.synchronize()

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
