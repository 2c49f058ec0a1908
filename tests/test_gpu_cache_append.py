"""New tokens into a paged cache: K rotated, V as it is, q rotated along; everything else in the cache stays."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, TYPES, Paged, stream
from test_gpu_rope import plain

pytestmark = pytest.mark.gpu


def bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def run(c, tokens, rope, with_q, token_seq=None, token_slot=None, with_order=True, with_slots=True, token_major=True, hq=6):
    """tokens new ones per sequence behind its present ones, unless token_seq / token_slot (host) say otherwise."""
    n_seqs, d = len(c.lens_np), c.d
    if token_slot is None:
        token_seq = np.repeat(np.arange(n_seqs), tokens).astype(np.int32)
        token_slot = (c.lens_np[:, None] + np.arange(tokens)).reshape(-1).astype(np.int32)
    n = len(token_slot)
    g = torch.Generator()
    g.manual_seed(31)
    shape = lambda h: (n, h, d) if token_major else (h, n, d)
    heads = lambda x: x.transpose(0, 1) if token_major else x
    q, k, v = (torch.randn(shape(h), generator=g).to(TYPES[c.dtype]) for h in (hq, c.hkv, c.hkv))
    pos = (np.arange(n, dtype=np.int32) * 13 + 5)[None]
    order = (np.arange(n, dtype=np.int32) + 100000)
    weights = torch.full((n_seqs, c.hkv, c.slots), 3.0, device=DEV)
    orders = torch.full((n_seqs, c.hkv, c.slots), -9, dtype=torch.int32, device=DEV)
    q_out = torch.empty_like(q, device=DEV)
    to = lambda x: None if x is None else torch.from_numpy(x).to(DEV)
    k_dev, v_dev, q_dev = k.to(DEV), v.to(DEV), q.to(DEV)
    seq_dev, slot_dev, order_dev, pos_dev = to(token_seq), to(token_slot), to(order) if with_order else None, to(pos)
    bs.bs_cache_append(c.cache, heads(k_dev), heads(v_dev), n, seq_dev, slot_dev, rope=rope, positions=pos_dev if rope else None,
                       q=heads(q_dev) if with_q else None, q_out=heads(q_out) if with_q else None,
                       slots=bs.CacheSlots.of(weights, orders) if with_slots else None, token_order=order_dev, stream=stream())
    torch.cuda.synchronize()
    if with_q:
        want, tol = plain(rope, heads(q).double().numpy(), pos, False)
        got = heads(q_out).double().cpu().numpy()
        assert (np.abs(got - want) <= tol * 1.01 + HALF_STEP[c.dtype] * (np.abs(want) + tol)).all()
    if rope:
        want_k, tol_k = plain(rope, heads(k).double().numpy(), pos, False)
    k_new, v_new = c.k.cpu(), c.v.cpu()
    written = torch.zeros((c.n_pages, c.page), dtype=torch.bool)
    w, o = weights.cpu(), orders.cpu()
    for t in range(n):
        s, j = (t if token_seq is None else token_seq[t]), token_slot[t]
        if not (0 <= s < n_seqs and 0 <= j < c.slots):
            continue
        p = c.table_np[s, j // c.page]
        if not 0 <= p < c.n_pages:
            continue
        written[p, j % c.page] = True
        got = k_new[p, :, j % c.page].double().numpy()
        if rope:
            assert (np.abs(got - want_k[:, t]) <= tol_k[:, t] * 1.01 + HALF_STEP[c.dtype] * (np.abs(want_k[:, t]) + tol_k[:, t])).all()
        else:
            assert (got == heads(k)[:, t].double().numpy()).all()
        assert torch.equal(v_new[p, :, j % c.page], heads(v)[:, t])
        if with_slots:
            assert (w[s, :, j] == 0).all() and (o[s, :, j] == (order[t] if with_order else j)).all()
            w[s, :, j], o[s, :, j] = 3.0, -9
    assert (w == 3).all() and (o == -9).all()
    stay = ~written[:, None, :, None]
    for new, old in ((k_new, c.k_np), (v_new, c.v_np)):
        assert torch.equal(torch.where(stay, bits(new), 0), torch.where(stay, bits(old), 0))
    return n


@pytest.mark.parametrize("dtype,hkv,d,page,pool,tokens", [
    ("bf16", 4, 128, 16, "heads", 1), ("bf16", 8, 128, 64, "slots", 1), ("f32", 1, 64, 16, "heads", 1), ("bf16", 2, 64, 48, "slots", 50), ("f32", 3, 128, 32, "heads", 129),
    ("bf16", 1, 8, 16, "heads", 3), ("bf16", 1, 256, 16, "slots", 3), ("f32", 2, 24, 16, "heads", 17)])
@pytest.mark.parametrize("layout", [bs.BS_ROPE_HALF, bs.BS_ROPE_INTERLEAVED])
def test_append(dtype, hkv, d, page, pool, tokens, layout):
    rope = bs.bs_rope_init(d, layout, 1e4, magnitude=1.1)
    run(Paged(dtype, hkv, d, page, [0, 1, 15, 16, 33, 200], pool=pool, more=tokens), tokens, rope, True, token_major=pool == "slots")


def test_without_rotation_part_of_the_head_and_no_slots():
    run(Paged("bf16", 2, 128, 16, [3, 40], more=5), 5, None, False)
    run(Paged("f32", 2, 128, 16, [3, 40], more=5), 5, bs.bs_rope_init(36), True, with_order=False)
    run(Paged("bf16", 2, 64, 16, [3, 40], more=5), 5, bs.bs_rope_init(20, bs.BS_ROPE_INTERLEAVED), False, with_slots=False)


def test_tokens_without_a_place_are_left_out():
    """A padded batch, slots and sequences out of range, pages that are none."""
    c = Paged("bf16", 2, 64, 16, [3, 40, 100], more=40, bad=0.3, seed=2)
    seq = np.array([0, -1, 2, 3, 1, 1, 0, 2, 2, 2 ** 31 - 1, -2 ** 31], dtype=np.int32)
    slot = np.array([3, 5, 100, 0, -1, 41, c.slots, 2 ** 31 - 1, 117, 4, 4], dtype=np.int32)
    run(c, 0, bs.bs_rope_init(64), True, seq, slot)


def test_one_token_per_sequence_without_a_list():
    c = Paged("bf16", 2, 128, 16, [3, 40, 0, 7], more=1, seed=3)
    run(c, 1, bs.bs_rope_init(128), True, None, c.lens_np.astype(np.int32))


def test_no_tokens():
    c = Paged("bf16", 2, 128, 16, [3], seed=3)
    x = torch.empty((2, 1, 128), dtype=torch.bfloat16, device=DEV)
    bs.bs_cache_append(c.cache, x, x, 0, None, c.lens, stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(bits(c.k.cpu()), bits(c.k_np))
