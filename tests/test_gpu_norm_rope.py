"""Norms of heads with rotary positions, their gradient, and the same into a paged cache, against plain forms in 64 bits.

Tolerance per element, u = 2^-24 a step of fp32, A = |a| + |b| of a pair (a, b):
  r = (mean x^2 + eps)^-1/2: a sum of d squares, all positive, is off by at most d + 1 steps, the mean and eps by two more, the root halves that, and root and
  quotient add two: (d / 2 + 4) u, relatively;
  z = x r (w + offset): three steps more; the rotation: 6 u A magnitude and 3 |angle| 2^-53 A (test_gpu_rope.py);
  back, g = R^T dy: 6 u A magnitude and the angle's; t = g w: two steps; s = sum t x: the errors of t, and d + 2 steps of sum |t x|;
  k = s r r / d: three steps; dx = r (t - x k): three steps of |t| + |x k|, and r's;
  the weights' gradients are sums of g x r over rows: the errors of the terms, and as many steps of the sum of their sizes as a thread adds up one behind
  the other, plus 9 (lanes and waves; the workgroups' parts are added in 64 bits, then rounded).
  Results are rounded once, half a step of their type."""
import numpy as np
import pytest
import torch

import paper_2507_09071_amd as bs
from cache_util import DEV, HALF_STEP, TYPES, Paged, dtype_of, stream

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def turn(rope, x, positions, back=False):
    """x [heads][tokens][d] in 64 bits, rotated; what the rotation may be off."""
    if rope is None:
        return x.copy(), np.zeros(x.shape)
    r, y, tol = rope.rotary_dim, x.copy(), np.zeros(x.shape)
    m = float(np.float32(rope.magnitude))
    for i in range(r // 2):
        lo, hi = (i, i + r // 2) if rope.layout == bs.BS_ROPE_HALF else (2 * i, 2 * i + 1)
        angle = positions[rope.axis[i]].astype(np.float64) * rope.freq[i]
        c, s = np.cos(angle) * m, np.sin(angle) * m * (-1 if back else 1)
        a, b = x[..., lo], x[..., hi]
        y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
        tol[..., lo] = tol[..., hi] = (np.abs(a) + np.abs(b)) * m * (6 * U + 3 * np.abs(angle) * 2.0 ** -53)
    return y, tol


def plain(rope, x, w, eps, positions):
    """x [heads][tokens][d], w [d] with the offset, in 64 bits.  The result and its tolerance without the last rounding."""
    d = x.shape[-1]
    z = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * w
    tz = np.abs(z) * (d / 2 + 7) * U
    y, tol = turn(rope, z, positions)
    if rope is not None:   # errors of z, turned: at most the sum of a pair's
        r, m = rope.rotary_dim, float(np.float32(rope.magnitude))
        for i in range(r // 2):
            lo, hi = (i, i + r // 2) if rope.layout == bs.BS_ROPE_HALF else (2 * i, 2 * i + 1)
            both = (tz[..., lo] + tz[..., hi]) * m
            tz[..., lo] = tz[..., hi] = both
    return y, tol + tz


def plain_grad(rope, x, dy, w, eps, positions):
    """dx and the weight's gradient with their tolerances (the sum's own steps apart), and the sum of its terms' sizes."""
    d = x.shape[-1]
    rel = (d / 2 + 4) * U
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    g, tg = turn(rope, dy, positions, back=True)
    t, v = g * w, x * r
    tt = tg * np.abs(w) + 2 * U * np.abs(t)
    s = (t * x).sum(-1, keepdims=True)
    ts = (tt * np.abs(x)).sum(-1, keepdims=True) + (d + 2) * U * np.abs(t * x).sum(-1, keepdims=True)
    k = s * r * r / d
    tk = ts * r * r / d + np.abs(k) * (2 * rel + 3 * U)
    dx = r * (t - x * k)
    tol = r * (tt + np.abs(x) * tk + 3 * U * (np.abs(t) + np.abs(x * k))) + np.abs(dx) * rel
    dw, size = (g * v).sum((0, 1)), np.abs(g * v).sum((0, 1))
    return dx, tol * 1.01, dw, ((tg * np.abs(v)).sum((0, 1)) + (rel + 3 * U) * size) * 1.01, size


def near(got, want, tol, dtype):
    got = got.double().cpu().numpy()
    worst = np.abs(got - want) - (tol * 1.01 + HALF_STEP[dtype] * (np.abs(want) + tol))
    assert (worst <= 0).all(), (float(worst.max()), np.unravel_index(worst.argmax(), worst.shape))


def draw(h, t, d, dtype, seed=0, spread=True):
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn((h, t, d), generator=g)
    if spread:   # rows of very different size
        x = x * torch.exp(2 * torch.randn((h, t, 1), generator=g))
    return x.to(TYPES[dtype])


def draw_weight(d, dtype, offset, seed):
    g = torch.Generator()
    g.manual_seed(50 + seed)
    return (torch.randn(d, generator=g) * 0.3 + 1 - offset).to(TYPES[dtype])


def full_weight(w, d, offset):
    return np.ones(d) if w is None else w.double().numpy() + offset


def check_forward(xs, ws, rope, positions, dtype, eps=1e-6, offset=0.0, views=None, in_place=False, stride=None, weight_views=None):
    t, d = xs[0].shape[1:]
    dev = [x.to(DEV) for x in xs] if views is None else [v(x.to(DEV)) for v, x in zip(views, xs)]
    ys = dev if in_place else [torch.full_like(x, float("nan")) for x in dev]
    wd = weight_views or [None if w is None else w.to(DEV) for w in ws]
    norm = bs.Norm.of(wd, eps, offset)
    pos = None if rope is None else torch.from_numpy(positions).to(DEV)
    bs.bs_norm_rope(norm, rope, dev, ys, dtype_of(dtype), t, d, pos, axis_stride=stride, stream=stream())
    for x, w, y in zip(xs, ws, ys):
        want, tol = plain(rope, x.double().numpy(), full_weight(w, d, offset), float(np.float32(eps)), positions)
        near(y, want, tol, dtype)
    return ys


def chain(n_heads, n_tokens, lanes):
    """Rows that a thread adds up at most: its heads of each token that it has."""
    items = n_tokens * lanes
    splits = max(1, min(n_heads, -(-131072 // items)))
    workgroups = max(1, min(-(-items // 256), 2048 // (splits + 2)))
    return -(-n_heads // splits) * -(-items // (workgroups * 256))


def check_grad(xs, dys, ws, rope, positions, dtype, eps=1e-6, offset=0.0, views=None, in_place=None, weights=True):
    t, d = xs[0].shape[1:]
    view = lambda i, x: x.to(DEV) if views is None else views[i](x.to(DEV))
    dev, ddev = [view(i, x) for i, x in enumerate(xs)], [view(i, x) for i, x in enumerate(dys)]
    dxs = {"x": dev, "dy": ddev, None: [torch.full_like(x, float("nan")) for x in dev]}[in_place]
    wd = [None if w is None else w.to(DEV) for w in ws]
    norm = bs.Norm.of(wd, eps, offset)
    pos = None if rope is None else torch.from_numpy(positions).to(DEV)
    dw = torch.full((len(xs), d), float("nan"), device=DEV) if weights else None
    ws_ = torch.full((bs.bs_norm_rope_grad_workspace(len(xs), dtype_of(dtype), t, d),), 0xff, dtype=torch.uint8, device=DEV) if weights else None
    bs.bs_norm_rope_grad(norm, rope, dev, ddev, dxs, dw, dtype_of(dtype), t, d, pos, ws_, stream=stream())
    for i, (x, dy, w) in enumerate(zip(xs, dys, ws)):
        dx, tol, g, tg, size = plain_grad(rope, x.double().numpy(), dy.double().numpy(), full_weight(w, d, offset), float(np.float32(eps)), positions)
        near(dxs[i], dx, tol, dtype)
        if weights:
            steps = chain(sum(x.shape[0] for x in xs), t, 64) + 9
            near(dw[i], g, tg + steps * U * size, "f32")
    return dxs, dw


SIZES = [(128, 128), (64, 64), (128, 64), (64, 20), (128, 36), (256, 256), (6, 2), (80, 80), (72, 16), (2, 2), (250, 30), (256, 34), (192, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [bs.BS_ROPE_HALF, bs.BS_ROPE_INTERLEAVED])
@pytest.mark.parametrize("d,r", SIZES)
def test_layouts_and_sizes(dtype, layout, d, r):
    rope = bs.bs_rope_init(r, layout, 1e4, magnitude=1.25)
    xs = [draw(7, 13, d, dtype), draw(2, 13, d, dtype, 1)]
    pos = np.arange(13, dtype=np.int32)[None] * 97 + 3
    for wt, offset in ((dtype, 0.0), ("f32", 1.0), ("bf16", 1.0)):
        check_forward(xs, [draw_weight(d, wt, offset, i) for i in range(2)], rope, pos, dtype, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [bs.BS_ROPE_HALF, bs.BS_ROPE_INTERLEAVED])
@pytest.mark.parametrize("d,r", SIZES)
def test_gradients_of_layouts_and_sizes(dtype, layout, d, r):
    rope = bs.bs_rope_init(r, layout, 1e4, magnitude=1.25)
    xs = [draw(7, 13, d, dtype), draw(2, 13, d, dtype, 1)]
    dys = [draw(7, 13, d, dtype, 2), draw(2, 13, d, dtype, 3)]
    pos = np.arange(13, dtype=np.int32)[None] * 97 + 3
    for wt, offset in ((dtype, 0.0), ("f32", 1.0)):
        check_grad(xs, dys, [draw_weight(d, wt, offset, i) for i in range(2)], rope, pos, dtype, offset=offset)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [2, 64, 80, 128, 256, 254])
def test_without_a_rotation_and_without_weights(dtype, d):
    xs, dys = [draw(3, 9, d, dtype), draw(1, 9, d, dtype, 1)], [draw(3, 9, d, dtype, 2), draw(1, 9, d, dtype, 3)]
    ws = [draw_weight(d, dtype, 0, 0), draw_weight(d, dtype, 0, 1)]
    check_forward(xs, ws, None, None, dtype)
    check_grad(xs, dys, ws, None, None, dtype)
    rope, pos = bs.bs_rope_init(d), np.arange(9, dtype=np.int32)[None]
    for some in ([None, None], [ws[0], None], [None, ws[1]]):   # (a missing weight is one, whatever the offset)
        check_forward(xs, some, rope, pos, dtype)
        check_grad(xs, dys, some, rope, pos, dtype)
    check_grad(xs, dys, ws, rope, pos, dtype, weights=False)
    check_forward(xs[:1], ws[:1], rope, pos, dtype)
    check_grad(xs[1:], dys[1:], ws[1:], rope, pos, dtype)
    with_offset = check_forward(xs[:1], [None], rope, pos, dtype, offset=0.0)[0]
    norm = bs.Norm.of([None], 1e-6, 1.0)
    y = torch.empty_like(xs[0], device=DEV)
    bs.bs_norm_rope(norm, rope, [xs[0].to(DEV)], [y], dtype_of(dtype), 9, d, torch.from_numpy(pos).to(DEV), stream=stream())
    assert torch.equal(y, with_offset)


@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 1000, 20011])
def test_token_counts(tokens):
    rope = bs.bs_rope_init(128, sections=[16, 24, 24], base=1e6)
    x, dy = draw(3, tokens, 128, "bf16"), draw(3, tokens, 128, "bf16", 1)
    w = draw_weight(128, "bf16", 0, 0)
    pos = np.stack([np.arange(tokens), np.arange(tokens) // 60, np.arange(tokens) % 60]).astype(np.int32)
    check_forward([x], [w], rope, pos, "bf16")
    check_grad([x], [dy], [w], rope, pos, "bf16")


@pytest.mark.parametrize("heads", [1, 3, 40, 129])
def test_head_counts(heads):
    rope, pos = bs.bs_rope_init(64), np.arange(300, dtype=np.int32)[None]
    xs, dys = [draw(heads, 300, 64, "f32"), draw(5, 300, 64, "f32", 1)], [draw(heads, 300, 64, "f32", 2), draw(5, 300, 64, "f32", 3)]
    ws = [draw_weight(64, "f32", 0, i) for i in range(2)]
    check_forward(xs, ws, rope, pos, "f32")
    check_grad(xs, dys, ws, rope, pos, "f32")


def test_more_rows_than_the_workgroups_have_threads():
    """A thread takes several tokens, one behind the other."""
    rope, pos = bs.bs_rope_init(16), np.arange(40000, dtype=np.int32)[None]
    xs, dys = [draw(2, 40000, 34, "f32"), draw(1, 40000, 34, "f32", 1)], [draw(2, 40000, 34, "f32", 2), draw(1, 40000, 34, "f32", 3)]
    check_grad(xs, dys, [draw_weight(34, "f32", 0, i) for i in range(2)], rope, pos, "f32")


def apart(extra, lead):
    """A view with other strides: rows `extra` elements longer, from element `lead` of a larger array on, token-major."""
    def view(x):
        h, t, d = x.shape
        base = torch.full((t * h * (d + extra) + lead,), float("nan"), dtype=x.dtype, device=x.device)
        v = base[lead:].view(t, h, d + extra)[..., :d].transpose(0, 1)
        v.copy_(x)
        return v
    return view


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("extra,lead", [(0, 0), (8, 8), (2, 2), (1, 0), (1, 1), (4, 4)])
def test_strides_and_alignments(dtype, extra, lead):
    rope, pos = bs.bs_rope_init(64, bs.BS_ROPE_INTERLEAVED), np.arange(11, dtype=np.int32)[None] + 5
    xs, dys = [draw(5, 11, 128, dtype), draw(2, 11, 128, dtype, 1)], [draw(5, 11, 128, dtype, 2), draw(2, 11, 128, dtype, 3)]
    ws, views = [draw_weight(128, dtype, 0, i) for i in range(2)], [apart(extra, lead)] * 2
    check_forward(xs, ws, rope, pos, dtype, views=views)
    check_forward(xs, ws, rope, pos, dtype, views=views, in_place=True)
    check_grad(xs, dys, ws, rope, pos, dtype, views=views)
    for place in ("x", "dy"):
        check_grad(xs, dys, ws, rope, pos, dtype, views=views, in_place=place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_any_alignment(dtype):
    x, w = draw(5, 11, 128, dtype), draw_weight(128, dtype, 0, 0)
    for lead in (0, 1, 2, 5):
        base = torch.zeros(128 + lead, dtype=w.dtype, device=DEV)
        base[lead:] = w.to(DEV)
        check_forward([x], [w], bs.bs_rope_init(128), np.arange(11, dtype=np.int32)[None], dtype, weight_views=[base[lead:]])


def test_rows_that_are_one():
    """x and dy broadcast over tokens and heads (stride 0); dx has rows of its own."""
    rope, pos = bs.bs_rope_init(64), np.arange(40, dtype=np.int32)[None]
    x, dy, w = draw(1, 1, 64, "f32").expand(6, 40, 64), draw(1, 1, 64, "f32", 1).expand(6, 40, 64), draw_weight(64, "f32", 0, 0)
    xd, dyd = x[:1, :1].contiguous().to(DEV).expand(6, 40, 64), dy[:1, :1].contiguous().to(DEV).expand(6, 40, 64)
    wd = w.to(DEV)
    norm = bs.Norm.of([wd])
    y, dx, dw = torch.empty((6, 40, 64), device=DEV), torch.empty((6, 40, 64), device=DEV), torch.empty((1, 64), device=DEV)
    p = torch.from_numpy(pos).to(DEV)
    bs.bs_norm_rope(norm, rope, [xd], [y], bs.BS_F32, 40, 64, p, stream=stream())
    ws = torch.empty(bs.bs_norm_rope_grad_workspace(1, bs.BS_F32, 40, 64), dtype=torch.uint8, device=DEV)
    bs.bs_norm_rope_grad(norm, rope, [xd], [dyd], [dx], dw, bs.BS_F32, 40, 64, p, ws, stream=stream())
    want, tol = plain(rope, x.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), pos)
    near(y, want, tol, "f32")
    want, tol, g, tg, size = plain_grad(rope, x.double().numpy(), dy.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), pos)
    near(dx, want, tol, "f32")
    near(dw[0], g, tg + (chain(6, 40, 64) + 9) * U * size, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zero_and_of_tiny_and_large_values(dtype):
    x, dy = draw(4, 6, 64, dtype), draw(4, 6, 64, dtype, 1)
    for i, f in enumerate((0.0, 1e-20, 1e-4, 1e15)):
        x[i] = (x[i].float() * f).to(x.dtype)
    w, rope, pos = draw_weight(64, dtype, 0, 0), bs.bs_rope_init(64), np.arange(6, dtype=np.int32)[None]
    for eps in (1e-6, 1e-5, 1.0):
        y = check_forward([x], [w], rope, pos, dtype, eps=eps)[0]
        assert (y[0] == 0).all()
        check_grad([x], [dy], [w], rope, pos, dtype, eps=eps)


def test_a_row_that_is_not_finite_stays_alone():
    x = draw(3, 5, 64, "bf16")
    bad = x.clone()
    bad[1, 2, 7], bad[2, 4, 0] = float("nan"), float("inf")
    rope, pos, w = bs.bs_rope_init(64), torch.arange(5, dtype=torch.int32, device=DEV)[None], draw_weight(64, "bf16", 0, 0).to(DEV)
    ys = [torch.empty_like(x, device=DEV) for _ in range(2)]
    for a, y in zip((x, bad), ys):
        bs.bs_norm_rope(bs.Norm.of([w]), rope, [a.to(DEV)], [y], bs.BS_BF16, 5, 64, pos, stream=stream())
    other = torch.ones((3, 5), dtype=torch.bool, device=DEV)
    other[1, 2] = other[2, 4] = False
    assert torch.equal(ys[0][other], ys[1][other]) and torch.isnan(ys[1][1, 2]).all()


@pytest.mark.parametrize("d,r,layout", [(128, 128, bs.BS_ROPE_HALF), (64, 20, bs.BS_ROPE_INTERLEAVED), (6, 2, bs.BS_ROPE_HALF)])
def test_gradients_against_differences(d, r, layout):
    """The loss sum dy y in 64 bits along random directions; central differences with h = 1e-5 are off by about h^2 times the third derivative (rows have size 1, the
    loss's derivatives are of its own size: 1e-8 of the sum of the terms' sizes, with room) and 2^-52 / h of the loss's terms (3e-11)."""
    rope = bs.bs_rope_init(r, layout)
    pos = np.arange(7, dtype=np.int32)[None] * 31
    x, dy = draw(3, 7, d, "f32", spread=False), draw(3, 7, d, "f32", 1, spread=False)
    w = draw_weight(d, "f32", 0, 0)
    eps = float(np.float32(1e-6))
    dxs, dw = check_grad([x], [dy], [w], rope, pos, "f32")
    X, G, W = x.double().numpy(), dy.double().numpy(), w.double().numpy()
    loss = lambda a, b: float((plain(rope, a, b, eps, pos)[0] * G).sum())
    rng = np.random.default_rng(2)
    _, tol, _, tg, size = plain_grad(rope, X, G, W, eps, pos)
    for _ in range(4):
        e, f = rng.standard_normal(X.shape), rng.standard_normal(W.shape)
        h = 1e-5
        by_x, by_w = (loss(X + h * e, W) - loss(X - h * e, W)) / (2 * h), (loss(X, W + h * f) - loss(X, W - h * f)) / (2 * h)
        got = dxs[0].double().cpu().numpy()
        room = 1e-8 * (np.abs(got * e).sum() + np.abs(plain(rope, X, W, eps, pos)[0] * G).sum())
        assert abs((got * e).sum() - by_x) <= ((tol + U * np.abs(got)) * np.abs(e)).sum() + room
        got = dw[0].double().cpu().numpy()
        assert abs((got * f).sum() - by_w) <= ((tg + (chain(3, 7, 64) + 10) * U * size) * np.abs(f)).sum() + room


def test_axes_apart():
    rope = bs.bs_rope_init(64, sections=[8, 12, 12])
    pos = np.random.default_rng(1).integers(-2 ** 31, 2 ** 31, (3, 50)).astype(np.int32)
    check_forward([draw(2, 20, 64, "f32")], [draw_weight(64, "f32", 0, 0)], rope, pos[:, :20].copy(), "f32")
    x, w = draw(2, 20, 64, "f32"), draw_weight(64, "f32", 0, 0)
    wd, y = w.to(DEV), torch.empty_like(x, device=DEV)
    bs.bs_norm_rope(bs.Norm.of([wd]), rope, [x.to(DEV)], [y], bs.BS_F32, 20, 64, torch.from_numpy(pos).to(DEV), axis_stride=50, stream=stream())
    want, tol = plain(rope, x.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), pos[:, :20])
    near(y, want, tol, "f32")


def test_no_tokens():
    """Nothing is written but the weights' gradients, which are zero."""
    rope, w = bs.bs_rope_init(64), torch.ones(64, device=DEV)
    e = torch.empty((2, 0, 64), device=DEV)
    pos = torch.empty((1, 0), dtype=torch.int32, device=DEV)
    bs.bs_norm_rope(bs.Norm.of([w]), rope, [e], [e], bs.BS_F32, 0, 64, pos, stream=stream())
    dw = torch.full((1, 64), 3.0, device=DEV)
    ws = torch.full((bs.bs_norm_rope_grad_workspace(1, bs.BS_F32, 0, 64),), 0xff, dtype=torch.uint8, device=DEV)
    bs.bs_norm_rope_grad(bs.Norm.of([w]), rope, [e], [e], [e], dw, bs.BS_F32, 0, 64, pos, ws, stream=stream())
    assert (dw == 0).all()


def test_same_bits_again():
    rope, pos = bs.bs_rope_init(128), np.arange(3000, dtype=np.int32)[None]
    xs, dys = [draw(8, 3000, 128, "bf16"), draw(2, 3000, 128, "bf16", 1)], [draw(8, 3000, 128, "bf16", 2), draw(2, 3000, 128, "bf16", 3)]
    ws = [draw_weight(128, "bf16", 0, i) for i in range(2)]
    a = check_grad(xs, dys, ws, rope, pos, "bf16")
    for _ in range(2):
        b = check_grad(xs, dys, ws, rope, pos, "bf16")
        assert all(torch.equal(x, y) for x, y in zip(a[0], b[0])) and torch.equal(a[1], b[1])


def test_offsets_beyond_32_bits():
    """Two heads 3 GB apart."""
    base = torch.empty(3 * 2 ** 30 // 2 + 5 * 64, dtype=torch.bfloat16, device=DEV)
    x, w = draw(2, 5, 64, "bf16"), draw_weight(64, "bf16", 0, 0)
    v = torch.as_strided(base, (2, 5, 64), (3 * 2 ** 30 // 2, 64, 1))
    v.copy_(x.to(DEV))
    rope, pos = bs.bs_rope_init(64), np.arange(5, dtype=np.int32)[None]
    wd = w.to(DEV)
    bs.bs_norm_rope(bs.Norm.of([wd]), rope, [v], [v], bs.BS_BF16, 5, 64, torch.from_numpy(pos).to(DEV), stream=stream())
    want, tol = plain(rope, x.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), pos)
    near(v, want, tol, "bf16")


# ---------------------------------------------------------------------------------------- into the cache

@pytest.mark.parametrize("dtype,hq,hkv,d,r", [("bf16", 28, 4, 128, 128), ("f32", 2, 1, 64, 64), ("bf16", 6, 3, 72, 18), ("f32", 4, 2, 256, 256), ("bf16", 8, 2, 96, 96)])
@pytest.mark.parametrize("page,pool", [(16, "heads"), (48, "slots")])
@pytest.mark.parametrize("with_rope", [True, False])
def test_append(dtype, hq, hkv, d, r, page, pool, with_rope):
    """Ragged new tokens of four sequences, some of which go nowhere."""
    rng = np.random.default_rng(d)
    lens, new = [0, 15, 100, 33], [3, 1, 20, 0]
    c = Paged(dtype, hkv, d, page, lens, pool=pool, more=25, seed=d)
    before = [x.clone() for x in (c.k, c.v)]
    seq, slot = np.repeat(np.arange(4), new), np.concatenate([n + np.arange(m) for n, m in zip(lens, new)])
    seq, slot = np.concatenate([seq, [-1, 2, 4, 1]]), np.concatenate([slot, [3, -1, 0, 10 ** 6]])   # the last four go nowhere
    t = len(seq)
    order = rng.permutation(t)
    seq, slot = seq[order].astype(np.int32), slot[order].astype(np.int32)
    q, k, v = draw(hq, t, d, dtype), draw(hkv, t, d, dtype, 1), draw(hkv, t, d, dtype, 2)
    ws = [draw_weight(d, dtype, 1, i) for i in range(2)]
    rope = bs.bs_rope_init(r) if with_rope else None
    pos = rng.integers(0, 10000, (1, t)).astype(np.int32)
    dev = lambda x: torch.from_numpy(x).to(DEV)
    heads = lambda x: x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1)
    q_out = torch.full_like(heads(q), float("nan"))
    w_rows, o_rows = torch.full((4, hkv, c.slots), 7.0, device=DEV), torch.full((4, hkv, c.slots), -3, dtype=torch.int32, device=DEV)
    token_order = np.arange(t, dtype=np.int32) + 1000
    wd = [w.to(DEV) for w in ws]
    bs.bs_cache_append_norm(c.cache, heads(k), heads(v), t, dev(seq), dev(slot), bs.Norm.of(wd, 1e-5, 1.0), rope=rope,
                            positions=None if rope is None else dev(pos), q=heads(q), q_out=q_out, slots=bs.CacheSlots.of(w_rows, o_rows), token_order=dev(token_order),
                            stream=stream())
    torch.cuda.synchronize()
    eps = float(np.float32(1e-5))
    want, tol = plain(rope, q.double().numpy(), ws[0].double().numpy() + 1, eps, pos)
    near(q_out, want, tol, dtype)
    want, tol = plain(rope, k.double().numpy(), ws[1].double().numpy() + 1, eps, pos)
    keys, values = c.k.double().cpu().numpy(), c.v.cpu()
    written = torch.zeros((c.n_pages, page), dtype=torch.bool)
    w_want, o_want = torch.full((4, hkv, c.slots), 7.0), torch.full((4, hkv, c.slots), -3, dtype=torch.int32)
    for i in range(t):
        if not (0 <= seq[i] < 4 and 0 <= slot[i] < c.slots):
            continue
        p, at = c.table_np[seq[i], slot[i] // page], slot[i] % page
        written[p, at] = True
        lim = tol[:, i] * 1.01 + HALF_STEP[dtype] * (np.abs(want[:, i]) + tol[:, i])
        assert (np.abs(keys[p, :, at] - want[:, i]) <= lim).all()
        assert torch.equal(values[p, :, at], v[:, i])
        w_want[seq[i], :, slot[i]], o_want[seq[i], :, slot[i]] = 0.0, token_order[i]
    for old, now in zip(before, (c.k, c.v)):   # all else as it was, NaN too
        kept = ~written[:, None, :, None].expand(old.shape)
        assert torch.equal(old.cpu().contiguous()[kept].view(torch.uint8), now.cpu().contiguous()[kept].view(torch.uint8))
    assert torch.equal(w_rows.cpu(), w_want) and torch.equal(o_rows.cpu(), o_want)


def test_append_without_q_and_without_sequences():
    c = Paged("bf16", 2, 64, 16, [5, 40, 16], more=1, seed=2)
    k, v, w = draw(2, 3, 64, "bf16"), draw(2, 3, 64, "bf16", 1), draw_weight(64, "bf16", 0, 1)
    v[0, 0, 0] = float("nan")
    slot = torch.tensor([5, 40, 16], dtype=torch.int32, device=DEV)
    pos = np.array([[7, 8, 9]], dtype=np.int32)
    wd = w.to(DEV)
    bs.bs_cache_append_norm(c.cache, k.to(DEV), v.to(DEV), 3, None, slot, bs.Norm.of([None, wd]), rope=bs.bs_rope_init(64), positions=torch.from_numpy(pos).to(DEV),
                            stream=stream())
    want, tol = plain(bs.bs_rope_init(64), k.double().numpy(), w.double().numpy(), float(np.float32(1e-6)), pos)
    for i, j in enumerate([5, 40, 16]):
        p = c.table_np[i, j // 16]
        near(c.k[p, :, j % 16], want[:, i], tol[:, i], "bf16")
        assert torch.equal(c.v[p, :, j % 16].cpu().view(torch.uint8), v[:, i].contiguous().view(torch.uint8))
