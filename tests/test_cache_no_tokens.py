"""Calls without a token do nothing, whatever an empty array's address is: nothing is launched, so they run on the host."""
import ctypes

import pytest

import paper_2507_09071_amd as bs
from paper_2507_09071_amd import binding
from test_cache_refusals import EINVAL, P, cache, heads, ref

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("token_major", [False, True])
def test_empty_tensors(token_major):
    """The address of an empty tensor is null."""
    make = lambda h: torch.empty((0, h, 128), dtype=torch.bfloat16).transpose(0, 1) if token_major else torch.empty((h, 0, 128), dtype=torch.bfloat16)
    none = torch.empty(0, dtype=torch.int32)
    assert make(8).data_ptr() == 0 and none.data_ptr() == 0
    rope = bs.bs_rope_init(64)
    bs.bs_rope_apply(rope, [make(8), make(2)], [make(8), make(2)], bs.BS_BF16, 0, 128, none)
    bs.bs_cache_append(cache(), make(4), make(4), 0, none, none)
    bs.bs_cache_append(cache(), make(4), make(4), 0, none, none, rope=rope, positions=none, q=make(8), q_out=make(8), slots=bs.CacheSlots(P, P, 112), token_order=none)


def test_what_else_is_wrong_is_still_refused():
    lib, rope, none = binding.load_library(), bs.bs_rope_init(64), heads(data=None)
    assert lib.bs_rope_apply(ref(rope), ref(none), ref(none), 1, bs.BS_BF16, 0, 128, None, 0, 0, None) == 0
    assert lib.bs_rope_apply(ref(rope), ref(none), ref(heads(7, None)), 1, bs.BS_BF16, 0, 128, None, 0, 0, None) == EINVAL
    assert lib.bs_rope_apply(ref(rope), ref(none), ref(none), 1, bs.BS_BF16, 0, 62, None, 0, 0, None) == EINVAL
    assert lib.bs_rope_apply(ref(rope), ref(none), ref(none), 1, bs.BS_BF16, 1, 128, P, 0, 0, None) == EINVAL
    c = cache()
    for n, k, slot, code in ((0, heads(4, None), None, 0), (0, heads(3, None), None, EINVAL), (1, heads(4, None), P, EINVAL), (1, heads(4), None, EINVAL), (-1, heads(4), P, EINVAL)):
        assert lib.bs_cache_append(ref(c), ref(k), ref(k), n, None, slot, None, None, 0, None, None, None, None, ctypes.c_void_p()) == code, n
