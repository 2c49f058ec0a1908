"""What the calls around normed heads and drafted tokens refuse, before anything touches a GPU: in the library, and tensors that the binding refuses."""
import ctypes
import math

import pytest

import paper_2507_09071_amd as bs
from paper_2507_09071_amd import binding
from test_cache_refusals import BAD_CACHES, EINVAL, EUNSUPPORTED, P, broken, cache, heads, ref

torch = pytest.importorskip("torch")


def norm(w0=P, w1=P, dtype=bs.BS_BF16, eps=1e-6, offset=0.0):
    return bs.Norm((ctypes.c_void_p * 2)(w0, w1), dtype, eps, offset)


BAD_NORMS = [(None, EINVAL), (norm(eps=0.0), EINVAL), (norm(eps=-1.0), EINVAL), (norm(eps=math.nan), EINVAL), (norm(eps=math.inf), EINVAL), (norm(eps=1e-40), EINVAL),
             (norm(offset=math.inf), EINVAL), (norm(offset=math.nan), EINVAL), (norm(dtype=2), EUNSUPPORTED), (norm(dtype=-1), EUNSUPPORTED), (norm(w0=P + 1), EINVAL),
             (norm(w1=P + 2, dtype=bs.BS_F32), EINVAL)]
BAD_ROPES = [(broken(rotary_dim=63), EINVAL), (broken(layout=2), EINVAL), (broken(n_axes=5), EINVAL), (broken(axis=1), EINVAL), (broken(freq=math.nan), EINVAL),
             (bs.bs_rope_init(130), EINVAL)]


def call_norm(**kw):
    f = dict(norm=norm(), rope=bs.bs_rope_init(64), x=heads(), y=heads(), n_tensors=1, dtype=bs.BS_BF16, n=3, d=128, positions=P, axis_stride=3)
    f.update(kw)
    return binding.load_library().bs_norm_rope(ref(f["norm"]), ref(f["rope"]), ref(f["x"]), ref(f["y"]), f["n_tensors"], f["dtype"], f["n"], f["d"], f["positions"],
                                               f["axis_stride"], None)


def call_grad(**kw):
    f = dict(norm=norm(), rope=bs.bs_rope_init(64), x=heads(), dy=heads(), dx=heads(), dweight=P, n_tensors=1, dtype=bs.BS_BF16, n=3, d=128, positions=P, axis_stride=3,
             workspace=P, n_bytes=1 << 30)
    f.update(kw)
    return binding.load_library().bs_norm_rope_grad(ref(f["norm"]), ref(f["rope"]), ref(f["x"]), ref(f["dy"]), ref(f["dx"]), f["dweight"], f["n_tensors"], f["dtype"], f["n"],
                                                    f["d"], f["positions"], f["axis_stride"], f["workspace"], f["n_bytes"], None)


def call_append(**kw):
    f = dict(cache=cache(), k=heads(4), v=heads(4), n=3, token_slot=P, norm=norm(), rope=bs.bs_rope_init(64), positions=P, axis_stride=3, q=None, q_out=None, slots=None)
    f.update(kw)
    return binding.load_library().bs_cache_append_norm(ref(f["cache"]), ref(f["k"]), ref(f["v"]), f["n"], None, f["token_slot"], ref(f["norm"]), ref(f["rope"]), f["positions"],
                                                       f["axis_stride"], ref(f["q"]), ref(f["q_out"]), ref(f["slots"]), None, None)


def call_tree(**kw):
    f = dict(cache=cache(), q=heads(), out=heads(), n=5, first=P, lens=P, most=70, mask=P, words=2, window=0, scale=0.1, cap=0.0, workspace=P, n_bytes=1 << 40)
    f.update(kw)
    return binding.load_library().bs_attn_tree(ref(f["cache"]), ref(f["q"]), ref(f["out"]), f["n"], f["first"], f["lens"], f["most"], f["mask"], f["words"], f["window"],
                                               f["scale"], f["cap"], f["workspace"], f["n_bytes"], None)


def call_accept(**kw):
    f = dict(cache=cache(), lens=P, lens_out=P, path=P + 4096, n_path=P + 8192, most=4, slots=None)
    f.update(kw)
    return binding.load_library().bs_cache_accept(ref(f["cache"]), f["lens"], f["lens_out"], f["path"], f["n_path"], f["most"], ref(f["slots"]), None)


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_caches(bad, code):
    c = cache(**bad)
    assert call_append(cache=c) == code
    assert call_accept(cache=c) == code
    assert call_tree(cache=c) == code
    assert binding.load_library().bs_attn_tree_workspace(ref(c), 8, 5, 4) == code


@pytest.mark.parametrize("bad", [dict(head_stride=0), dict(slot_stride=120), dict(slot_stride=0), dict(page_stride=64)])
def test_caches_whose_rows_overlap_are_not_written(bad):
    assert call_append(cache=cache(**bad)) == EINVAL and call_accept(cache=cache(**bad)) == EINVAL


@pytest.mark.parametrize("bad,code", BAD_NORMS)
def test_norms(bad, code):
    assert call_norm(norm=bad) == code and call_grad(norm=bad) == code and call_append(norm=bad) == code


@pytest.mark.parametrize("bad,code", BAD_ROPES)
def test_ropes(bad, code):
    assert call_norm(rope=bad) == code and call_grad(rope=bad) == code and call_append(rope=bad) == code


COMMON = [(dict(x=None), EINVAL), (dict(n_tensors=0), EINVAL), (dict(n_tensors=3), EINVAL), (dict(dtype=2), EUNSUPPORTED), (dict(n=-1), EINVAL), (dict(d=62), EINVAL),
          (dict(d=0, rope=None), EINVAL), (dict(d=129, rope=None), EINVAL), (dict(d=258, rope=None), EINVAL), (dict(positions=None), EINVAL), (dict(axis_stride=-1), EINVAL),
          (dict(x=heads(data=P + 1)), EINVAL), (dict(x=heads(token=-1)), EINVAL), (dict(x=heads(data=None)), EINVAL), (dict(x=heads(0)), EINVAL), (dict(x=heads(7)), EINVAL)]


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(y=None), EINVAL), (dict(y=heads(head=64)), EINVAL), (dict(y=heads(token=0)), EINVAL), (dict(y=heads(token=1016)), EINVAL), (dict(y=heads(7)), EINVAL)])
def test_norm_rope(change, code):
    assert call_norm(**change) == code


@pytest.mark.parametrize("change,code", COMMON + [
    (dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(dx=heads(head=64)), EINVAL), (dict(dx=heads(token=0)), EINVAL), (dict(dx=heads(7)), EINVAL), (dict(dy=heads(7)), EINVAL),
    (dict(dy=heads(data=P + 1)), EINVAL), (dict(dy=heads(token=-1)), EINVAL), (dict(dweight=P + 2), EINVAL), (dict(workspace=None), EINVAL), (dict(workspace=P + 8), EINVAL),
    (dict(n_bytes=100), EINVAL), (dict(n_bytes=-1), EINVAL)])
def test_norm_rope_grad(change, code):
    assert call_grad(**change) == code


def test_workspace_of_the_gradient():
    f = binding.load_library().bs_norm_rope_grad_workspace
    assert 0 < f(1, bs.BS_BF16, 10, 128) < f(2, bs.BS_F32, 10 ** 9, 256) <= 4 << 20
    assert f(0, 0, 1, 64) == f(3, 0, 1, 64) == f(1, 0, -1, 64) == f(1, 0, 1, 63) == f(1, 0, 1, 258) == EINVAL and f(1, 2, 1, 64) == EUNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(k=None), dict(v=None), dict(k=heads(8)), dict(v=heads(3)), dict(n=-1), dict(token_slot=None), dict(q=heads()), dict(q_out=heads()), dict(q=heads(), q_out=heads(4)),
    dict(q=heads(), q_out=heads(token=512)), dict(positions=None), dict(axis_stride=-1), dict(slots=bs.CacheSlots(P, P, 111)), dict(k=heads(4, P + 1))])
def test_append(change):
    assert call_append(**change) == EINVAL


@pytest.mark.parametrize("change,code", [
    (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q=heads(data=None)), EINVAL), (dict(q=heads(6), out=heads(6)), EINVAL), (dict(out=heads(4)), EINVAL),
    (dict(q=heads(0), out=heads(0)), EINVAL), (dict(first=None), EINVAL), (dict(lens=None), EINVAL), (dict(n=-1), EINVAL), (dict(most=0), EINVAL), (dict(most=257), EINVAL),
    (dict(most=-1), EINVAL), (dict(words=1), EINVAL), (dict(words=-1), EINVAL), (dict(mask=None), EINVAL), (dict(mask=P + 4), EINVAL), (dict(window=-1), EINVAL),
    (dict(scale=0.0), EINVAL), (dict(scale=math.nan), EINVAL), (dict(scale=math.inf), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=3e38), EUNSUPPORTED), (dict(cap=-1.0), EINVAL), (dict(cap=math.nan), EINVAL),
    (dict(cap=math.inf), EINVAL), (dict(cap=3e38), EUNSUPPORTED), (dict(cap=1e-38, scale=1e30), EUNSUPPORTED), (dict(cap=1e30, scale=1e-30), EUNSUPPORTED),
    (dict(workspace=None), EINVAL), (dict(workspace=P + 8), EINVAL), (dict(n_bytes=-1), EINVAL), (dict(q=heads(data=P + 8)), EUNSUPPORTED), (dict(out=heads(head=132)), EUNSUPPORTED),
    (dict(out=heads(head=0)), EINVAL), (dict(out=heads(token=512)), EINVAL), (dict(q=heads(token=-8)), EINVAL), (dict(cache=cache(head_dim=256)), EUNSUPPORTED),
    (dict(cache=cache(head_dim=96)), EUNSUPPORTED)])
def test_tree(change, code):
    assert call_tree(**change) == code


@pytest.mark.parametrize("change", [
    dict(lens=None), dict(lens_out=None), dict(path=None), dict(n_path=None), dict(most=-1), dict(most=257), dict(lens_out=P + 4), dict(lens=P + 4), dict(n_path=P), dict(path=P - 4),
    dict(lens_out=P + 2048, path=P + 2048), dict(slots=bs.CacheSlots(P, P, 111)), dict(slots=bs.CacheSlots(P + 2, P, 112))])
def test_accept(change):
    assert call_accept(**change) == EINVAL


# ---------------------------------------------------------------------------------------- tensors

def rows(h, t, d=64):
    return torch.zeros((h, t, d))


def ints(*shape, t=torch.int32):
    return torch.zeros(shape, dtype=t)


def the_cache():
    k = torch.zeros((4, 2, 16, 64))
    return bs.KVCache.of(k, k.clone(), ints(3, 2), bs.BS_F32)


@pytest.fixture
def nothing_is_launched(monkeypatch):
    lib, reached = binding.load_library(), []

    class Library:
        def __getattr__(self, name):
            return (lambda *a: reached.append(name) or 0) if name in ("bs_norm_rope", "bs_norm_rope_grad", "bs_cache_append_norm", "bs_attn_tree", "bs_cache_accept") else getattr(lib, name)

    monkeypatch.setattr(binding, "load_library", lambda: Library())
    return reached


def py_norm(**kw):
    f = dict(norm=bs.Norm.of([torch.ones(64)] * 2), rope=bs.bs_rope_init(32), xs=[rows(8, 5), rows(2, 5)], ys=[rows(8, 5), rows(2, 5)], dtype=bs.BS_F32, n_tokens=5, head_dim=64,
             positions=ints(1, 5))
    f.update(kw)
    bs.bs_norm_rope(**f)


def py_grad(**kw):
    f = dict(norm=bs.Norm.of([torch.ones(64)] * 2), rope=bs.bs_rope_init(32), xs=[rows(8, 5), rows(2, 5)], dys=[rows(8, 5), rows(2, 5)], dxs=[rows(8, 5), rows(2, 5)],
             dweights=torch.zeros(2, 64), dtype=bs.BS_F32, n_tokens=5, head_dim=64, positions=ints(1, 5), workspace=torch.zeros(1 << 20))
    f.update(kw)
    bs.bs_norm_rope_grad(**f)


def py_append(**kw):
    f = dict(cache=the_cache(), k=rows(2, 5), v=rows(2, 5), n_tokens=5, token_seq=ints(5), token_slot=ints(5), norm=bs.Norm.of([torch.ones(64)] * 2), rope=bs.bs_rope_init(32),
             positions=ints(5), q=rows(8, 5), q_out=rows(8, 5))
    f.update(kw)
    bs.bs_cache_append_norm(**f)


def py_tree(**kw):
    f = dict(cache=the_cache(), q=rows(8, 5), out=rows(8, 5), n_tokens=5, first=ints(4), lens=ints(3), max_tokens=3, scale=0.1, workspace=(4096, 1 << 30), mask=ints(5, 1, t=torch.int64))
    f.update(kw)
    bs.bs_attn_tree(**f)


def py_accept(**kw):
    f = dict(cache=the_cache(), lens=ints(3), lens_out=ints(3), path=ints(3, 4), n_path=ints(3))
    f.update(kw)
    bs.bs_cache_accept(**f)


@pytest.mark.parametrize("call,name", [(py_norm, "bs_norm_rope"), (py_grad, "bs_norm_rope_grad"), (py_append, "bs_cache_append_norm"), (py_tree, "bs_attn_tree"), (py_accept, "bs_cache_accept")])
def test_tensors_that_fit_go_down(nothing_is_launched, call, name):
    call()
    assert nothing_is_launched == [name]


@pytest.mark.parametrize("call,change", [
    (py_norm, dict(xs=[rows(8, 4), rows(2, 5)])), (py_norm, dict(ys=[rows(8, 5)])), (py_norm, dict(ys=[rows(8, 5, 32), rows(2, 5)])), (py_norm, dict(positions=ints(1, 4))),
    (py_norm, dict(positions=ints(1, 5, t=torch.int64))), (py_norm, dict(norm=bs.Norm.of([torch.ones(64)]))), (py_norm, dict(norm=bs.Norm.of([torch.ones(64), torch.ones(63)]))),
    (py_norm, dict(xs=[rows(8, 5).bfloat16(), rows(2, 5)])), (py_norm, dict(rope=None, norm=bs.Norm.of([torch.ones(128)] * 2))),
    (py_grad, dict(dys=[rows(8, 5)])), (py_grad, dict(dxs=[rows(8, 4), rows(2, 5)])), (py_grad, dict(dweights=torch.zeros(64))), (py_grad, dict(dweights=torch.zeros(2, 64).bfloat16())),
    (py_grad, dict(dweights=ints(2, 64))), (py_grad, dict(dweights=torch.zeros(64, 2).T)),
    (py_append, dict(k=rows(2, 4))), (py_append, dict(token_slot=ints(4))), (py_append, dict(token_slot=ints(5, t=torch.int64))), (py_append, dict(q=rows(8, 5, 32))),
    (py_append, dict(norm=bs.Norm.of([torch.ones(32), torch.ones(64)]))), (py_append, dict(norm=bs.Norm.of([torch.ones(64)]))),
    (py_tree, dict(q=rows(8, 4))), (py_tree, dict(out=rows(8, 5, 32))), (py_tree, dict(first=ints(3))), (py_tree, dict(lens=ints(2))), (py_tree, dict(lens=ints(3, t=torch.int64))),
    (py_tree, dict(mask=ints(5, 1))), (py_tree, dict(mask=ints(4, 1, t=torch.int64))), (py_tree, dict(mask=ints(5, t=torch.int64))), (py_tree, dict(mask=ints(2, 5, t=torch.int64).T)),
    (py_tree, dict(mask=torch.zeros(5, 1, dtype=torch.float64))),
    (py_accept, dict(lens=ints(2))), (py_accept, dict(lens_out=ints(2))), (py_accept, dict(n_path=ints(2))), (py_accept, dict(path=ints(2, 4))), (py_accept, dict(path=ints(4, 3).T)),
    (py_accept, dict(path=ints(3, 4, t=torch.int64))), (py_accept, dict(max_path=5)), (py_accept, dict(slots=bs.CacheSlots.of(torch.zeros(2, 2, 32))))])
def test_tensors_that_a_call_would_misread_are_refused(nothing_is_launched, call, change):
    with pytest.raises(ValueError):
        call(**change)
    assert not nothing_is_launched


def test_weights_that_are_refused():
    w = torch.ones(64)
    for bad in ([], [w] * 3, [w, w.bfloat16()], [w.half()], [w.double()], [torch.ones(128)[::2]], [torch.ones(2, 64)], [ints(64)]):
        with pytest.raises(ValueError):
            bs.Norm.of(bad)
    n = bs.Norm.of([None, w.bfloat16()], 1e-5, 1.0)
    assert n.weight[0] is None and n.weight_dtype == bs.BS_BF16 and abs(n.eps - 1e-5) < 1e-12 and n.offset == 1.0
