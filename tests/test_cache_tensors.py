"""Tensors that the calls around the KV cache would read or write past their ends, or misread, are refused before anything is launched."""
import numpy as np
import pytest

import paper_2507_09071_amd as bs
from paper_2507_09071_amd import binding

torch = pytest.importorskip("torch")

D, HQ, HKV, SEQS, PAGES, PAGE = 64, 8, 2, 3, 4, 16
WORKSPACE = (4096, 1 << 40)


@pytest.fixture(autouse=True)
def nothing_is_launched(monkeypatch):
    """The library's calls that launch are replaced by ones that only say that they were reached."""
    lib, reached = binding.load_library(), []

    class Library:
        def __getattr__(self, name):
            if name in ("bs_rope_apply", "bs_cache_append", "bs_attn_decode", "bs_cache_evict"):
                return lambda *a: reached.append(name) or 0
            return getattr(lib, name)

    monkeypatch.setattr(binding, "load_library", lambda: Library())
    return reached


def rows(heads, tokens, d=D, t=torch.float32):
    return torch.zeros((heads, tokens, d), dtype=t)


def ints(*shape, t=torch.int32):
    return torch.zeros(shape, dtype=t)


def the_cache(t=torch.float32, n_seqs=SEQS):
    k = torch.zeros((PAGES, HKV, PAGE, D), dtype=t)
    return bs.KVCache.of(k, k.clone(), ints(n_seqs, 2), bs.BS_F32 if t == torch.float32 else bs.BS_BF16)


def the_slots(n_seqs=SEQS, heads=HKV, slots=2 * PAGE):
    return bs.CacheSlots.of(torch.zeros((n_seqs, heads, slots)), ints(n_seqs, heads, slots))


def rope_apply(**kw):
    f = dict(xs=[rows(HQ, 5), rows(HKV, 5)], ys=[rows(HQ, 5), rows(HKV, 5)], dtype=bs.BS_F32, n_tokens=5, head_dim=D, positions=ints(1, 5), axis_stride=None, sections=None)
    f.update(kw)
    rope = bs.bs_rope_init(32, sections=f.pop("sections"))
    bs.bs_rope_apply(rope, **f)


def append(**kw):
    f = dict(cache=the_cache(), k=rows(HKV, 5), v=rows(HKV, 5), n_tokens=5, token_seq=ints(5), token_slot=ints(5), rope=bs.bs_rope_init(32), positions=ints(5), axis_stride=None,
             q=rows(HQ, 5), q_out=rows(HQ, 5), slots=the_slots(), token_order=ints(5))
    f.update(kw)
    bs.bs_cache_append(**f)


def decode(**kw):
    f = dict(cache=the_cache(), q=rows(HQ, SEQS), out=rows(HQ, SEQS), lens=ints(SEQS), scale=0.1, workspace=WORKSPACE, slots=the_slots(), slots_out=the_slots())
    f.update(kw)
    bs.bs_attn_decode(**f)


def evict(**kw):
    f = dict(cache=the_cache(), lens=ints(SEQS), lens_out=ints(SEQS), keep=5, keep_first=0, keep_last=0, slots=the_slots(), slots_out=the_slots(), workspace=WORKSPACE)
    f.update(kw)
    bs.bs_cache_evict(**f)


BF16 = torch.bfloat16
REFUSED = [
    # rows of another size than the call's: read or written past their end
    (rope_apply, dict(ys=[rows(HQ, 5), rows(HKV, 5, t=BF16)])), (rope_apply, dict(xs=[rows(HQ, 5, t=BF16), rows(HKV, 5)])), (rope_apply, dict(xs=[rows(HQ, 4), rows(HKV, 5)])),
    (rope_apply, dict(ys=[rows(HQ, 5), rows(HKV, 4)])), (rope_apply, dict(ys=[rows(HQ, 5, 32), rows(HKV, 5)])), (rope_apply, dict(dtype=bs.BS_BF16)), (rope_apply, dict(n_tokens=6)),
    (append, dict(k=rows(HKV, 4))), (append, dict(v=rows(HKV, 5, 32))), (append, dict(k=rows(HKV, 5, t=BF16))), (append, dict(q=rows(HQ, 4))), (append, dict(q_out=rows(HQ, 5, t=BF16))),
    (append, dict(cache=the_cache(BF16))),
    (decode, dict(out=rows(HQ, SEQS, t=BF16))), (decode, dict(q=rows(HQ, SEQS, t=BF16))), (decode, dict(out=rows(HQ, SEQS - 1))), (decode, dict(q=rows(HQ, SEQS, 32))),
    (decode, dict(cache=the_cache(n_seqs=SEQS + 1))),
    # whole numbers of another size, too few, or with gaps
    (rope_apply, dict(positions=ints(1, 5, t=torch.int64))), (rope_apply, dict(positions=ints(1, 4))), (rope_apply, dict(positions=ints(5, 2)[:, 0])),
    (rope_apply, dict(positions=ints(2, 5), sections=[4, 6, 6])), (rope_apply, dict(positions=ints(2, 5), sections=[8, 8], axis_stride=6)),
    (rope_apply, dict(positions=ints(2, 9)[:, :5], sections=[8, 8])),
    (append, dict(token_seq=ints(5, t=torch.int64))), (append, dict(token_slot=ints(4))), (append, dict(token_slot=ints(10)[::2])), (append, dict(token_order=ints(5, t=torch.int16))),
    (append, dict(positions=ints(5, t=torch.int64))), (append, dict(token_seq=None, n_tokens=5, token_slot=ints(3))),
    (decode, dict(lens=ints(SEQS, t=torch.int64))), (decode, dict(lens=ints(SEQS - 1))), (decode, dict(lens=ints(SEQS, 2)[:, 1])),
    (evict, dict(lens=ints(SEQS, t=torch.int64))), (evict, dict(lens_out=ints(SEQS, t=torch.int64))), (evict, dict(lens_out=ints(SEQS - 1))),
    # what is known of the slots: of fewer sequences or heads than the cache has
    (append, dict(slots=the_slots(SEQS - 1))), (decode, dict(slots=the_slots(SEQS, HKV - 1))), (decode, dict(slots_out=the_slots(SEQS - 1))), (evict, dict(slots=the_slots(SEQS - 1))),
    (evict, dict(slots_out=the_slots(heads=1)))]


@pytest.mark.parametrize("call,change", REFUSED)
def test_refused(call, change, nothing_is_launched):
    call()
    assert len(nothing_is_launched) == 1   # (as it is, it goes through)
    with pytest.raises(ValueError):
        call(**change)
    assert len(nothing_is_launched) == 1


@pytest.mark.parametrize("call,change", [
    (rope_apply, dict(n_tokens=3)), (rope_apply, dict(xs=[rows(5, HQ).transpose(0, 1), rows(HKV, 9)[:, 2:7]])), (rope_apply, dict(positions=ints(5))), (rope_apply, dict(positions=4096)),
    (rope_apply, dict(positions=ints(2, 9)[:, :5], sections=[8, 8], axis_stride=9)), (rope_apply, dict(positions=ints(18)[3:], sections=[8, 8], axis_stride=9)),
    (rope_apply, dict(positions=ints(2, 9)[0, 4:], sections=[8, 8], axis_stride=9)), (rope_apply, dict(positions=ints(1, 5), sections=[8, 8], axis_stride=0)),
    (rope_apply, dict(xs=[binding.Heads(4096, D, D, HQ), rows(HKV, 5)])),
    (append, dict(token_seq=None, n_tokens=SEQS, token_order=None, slots=None)), (append, dict(q=None, q_out=None, rope=None, positions=None)), (append, dict(token_slot=ints(9)[2:])),
    (decode, dict(slots=None, slots_out=None)), (decode, dict(q=rows(SEQS + 2, HQ).transpose(0, 1))), (decode, dict(lens=ints(9))),
    (decode, dict(lens=4096)), (decode, dict(slots=bs.CacheSlots(4096, 4096, 32))), (evict, dict(slots=the_slots(SEQS + 1))), (evict, dict(workspace=torch.zeros(64)))])
def test_what_lies_within_its_memory_goes_through(call, change, nothing_is_launched):
    call(**change)
    assert len(nothing_is_launched) == 1


def test_weights_and_order_are_alike():
    for order in (ints(SEQS, HKV - 1, 32), ints(SEQS - 1, HKV, 32), ints(SEQS * HKV, 32)):
        with pytest.raises(ValueError):
            bs.CacheSlots.of(torch.zeros((SEQS, HKV, 32)), order)
    with pytest.raises(ValueError):
        bs.CacheSlots.of(torch.zeros((SEQS, HKV, 32), dtype=torch.int32), None)
    with pytest.raises(ValueError):
        bs.CacheSlots.of(None, torch.zeros((SEQS, HKV, 32)))


def test_numbers_of_numpy_go_through(nothing_is_launched):
    rope_apply(n_tokens=np.int64(5), head_dim=np.int32(D))
    assert nothing_is_launched == ["bs_rope_apply"]
