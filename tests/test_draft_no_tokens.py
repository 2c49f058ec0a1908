"""Calls around drafted tokens in a step without any: the address of an empty tensor is null, that of an empty mask too."""
import pytest

import paper_2507_09071_amd as bs
from test_cache_refusals import EINVAL, P, cache, heads
from test_draft_refusals import call_tree

torch = pytest.importorskip("torch")


def test_an_empty_mask_is_no_mistake():
    """(Without a GPU the library cannot tell how large a workspace has to be, and says so: what a call without a mask gets.)"""
    none = dict(n=0, q=heads(data=None), out=heads(data=None), mask=None)
    assert call_tree(**none, words=2) == call_tree(**none, words=0) != EINVAL
    assert call_tree(**none, words=5) != EINVAL


@pytest.mark.parametrize("change", [dict(words=-1), dict(words=1, mask=P), dict(mask=P + 4), dict(most=0), dict(lens=None), dict(q=heads(3, None))])
def test_what_else_is_wrong_is_still_refused(change):
    none = dict(n=0, q=heads(data=None), out=heads(data=None), mask=None, words=0)
    none.update(change)
    assert call_tree(**none) == EINVAL
    assert call_tree(n=1, mask=None, words=2) == EINVAL


def make(h, token_major, device):
    return torch.empty((0, h, 128), dtype=torch.bfloat16, device=device).transpose(0, 1) if token_major else torch.empty((h, 0, 128), dtype=torch.bfloat16, device=device)


@pytest.mark.gpu
@pytest.mark.parametrize("token_major", [False, True])
def test_empty_tensors(token_major):
    dev = "cuda:0"
    k = torch.full((4, 4, 16, 128), 3.0, dtype=torch.bfloat16, device=dev)
    v, table, none = k.clone(), torch.zeros((2, 2), dtype=torch.int32, device=dev), torch.empty(0, dtype=torch.int32, device=dev)
    c = bs.KVCache.of(k, v, table, bs.BS_BF16)
    lens, first = torch.tensor([3, 17], dtype=torch.int32, device=dev), torch.zeros(3, dtype=torch.int32, device=dev)
    h = lambda n: make(n, token_major, dev)
    norm = bs.Norm.of([torch.ones(128, dtype=torch.bfloat16, device=dev)] * 2)
    ws = torch.empty(bs.bs_attn_tree_workspace(c, 8, 0, 5), dtype=torch.uint8, device=dev)
    st = torch.cuda.current_stream().cuda_stream
    bs.bs_cache_append_norm(c, h(4), h(4), 0, none, none, norm, rope=bs.bs_rope_init(128), positions=none, q=h(8), q_out=h(8), stream=st)
    for mask in (torch.empty((0, 1), dtype=torch.int64, device=dev), torch.empty((0, 3), dtype=torch.int64, device=dev), None):
        bs.bs_attn_tree(c, h(8), h(8), 0, first, lens, 5, 0.1, ws, mask=mask, stream=st)
    bs.bs_cache_accept(c, lens, lens, torch.empty((2, 0), dtype=torch.int32, device=dev), torch.zeros(2, dtype=torch.int32, device=dev), stream=st)
    torch.cuda.synchronize()
    assert lens.tolist() == [3, 17] and (k == 3).all() and (v == 3).all()
