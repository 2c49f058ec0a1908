"""Operators around the KV cache, as cases that can be timed and compared: what a program that answers with this library runs per
layer besides the prefill attention.

  op = "rope"     rotary positions of q and k (or, inverse, of their gradients)
  op = "append"   the new tokens' k, rotated, and v go into the pages of a cache; q of the same step is rotated along
  op = "decode"   attention of one new token of every sequence over the paged cache; with `weights` the attention that every slot
                  received is added up per KV head
  op = "evict"    the cache is cut back to `keep` slots per sequence and KV head, those with the most accumulated weight

Fields of a case
  dtype, hq, hkv, d   element type of q, k, v; query heads, KV heads, head dimension
  tokens              rope, append: tokens per sequence
  seqs                append, decode, evict: sequences of the batch
  lo, hi              append, decode, evict: slots in use per sequence, over the logarithm between these (the seed deals them out)
  page, pool          slots per page; order of the axes of a page: "heads" [head][slot][d], "slots" [slot][head][d]
  rotary, layout, axes, base, scaling, factor, far   rope, append: rotated channels, "half" or "pairs" (interleaved), axes of the
                      positions (3: time, height, width of a picture's tokens), base and scaling of the frequencies, first position
  window, weights     decode
  keep, first, last   evict: slots kept, of them the first and last tokens of the sequence in any case
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}


def _rope(name, **kw):
    c = {"name": name, "op": "rope", "dtype": "bf16", "hq": 28, "hkv": 4, "d": 128, "tokens": 1, "rotary": 128, "layout": "half",
         "axes": 1, "base": 1e6, "scaling": "plain", "factor": 1.0, "far": 0, "inverse": False}
    c.update(kw)
    return c


def _append(name, **kw):
    c = _rope(name, op="append", seqs=1, lo=0, hi=0, page=16, pool="heads")
    del c["inverse"]
    c.update(kw)
    return c


def _decode(name, **kw):
    c = {"name": name, "op": "decode", "dtype": "bf16", "hq": 28, "hkv": 4, "d": 128, "seqs": 1, "lo": 1, "hi": 1, "page": 16,
         "pool": "heads", "window": 0, "weights": False}
    c.update(kw)
    return c


def _evict(name, **kw):
    c = {"name": name, "op": "evict", "dtype": "bf16", "hkv": 4, "d": 128, "seqs": 1, "lo": 1, "hi": 1, "page": 16, "pool": "heads",
         "keep": 1, "first": 4, "last": 32}
    c.update(kw)
    return c


def listed():
    return [
        # one decoding step of eight chats about pictures, positions on three axes: launches count
        _rope("rope_step_8", tokens=8, axes=3, far=30011),
        # q and k of the prompt with sixteen pictures that the prefill benchmark is quoted on
        _rope("rope_prompt_39k", tokens=39500, axes=3),
        # fine-tuning in fp32: gradients of interleaved pairs in half of the head, of a long-context model
        _rope("rope_gradient_5k", dtype="f32", hq=32, hkv=16, tokens=5003, rotary=64, layout="pairs", base=1e4, scaling="parts", factor=8.0,
              far=120000, inverse=True),
        # one decoding step of a full batch: rotate q and k, write k and v
        _append("append_step_128", hq=40, hkv=8, tokens=1, seqs=128, lo=200, hi=16384, axes=3),
        # the prompt with sixteen pictures goes into an empty cache behind its prefill
        _append("append_prompt_39k", tokens=39500, page=64, pool="slots", axes=3),
        # the smallest configuration of the repository, in fp32, a sliding-window layer
        _decode("decode_tiny_f32", dtype="f32", hq=2, hkv=1, d=64, seqs=5, lo=1, hi=1136, window=512),
        # one chat behind the prompt with sixteen pictures
        _decode("decode_39k", lo=39501, hi=39501),
        # a batch of chats of very different length
        _decode("decode_batch_48", hq=40, hkv=8, seqs=48, lo=17, hi=16384, page=32, pool="slots"),
        # two of the longest prompts, with the weights that an eviction needs
        _decode("decode_weights_150k", hq=32, hkv=16, seqs=2, lo=149003, hi=151777, page=64, weights=True),
        # the smallest configuration, cut back to a quarter
        _evict("evict_tiny_f32", dtype="f32", hkv=1, d=64, seqs=3, lo=1136, hi=1136, keep=284),
        # a served batch on a fixed budget, after 64 more tokens each
        _evict("evict_step_64", hkv=8, seqs=64, lo=4160, hi=4160, keep=4096, last=256),
        # the prompt with sixteen pictures, cut back to a fifth behind its prefill
        _evict("evict_prompt_39k", lo=39500, hi=39500, page=64, pool="slots", keep=8192, last=1024),
    ]


# ---------------------------------------------------------------------------------------- drawn cases

_SHAPES = ((28, 4, 128), (40, 8, 128), (32, 16, 128), (32, 8, 64), (16, 2, 128), (8, 8, 64), (2, 1, 64), (64, 4, 128))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rotation(rng, d):
    scaling = rng.choice(("plain", "linear", "base", "parts"))
    return {"rotary": rng.choice((d, d, d // 2, d // 4 + 4)), "layout": rng.choice(("half", "pairs")), "axes": rng.choice((1, 1, 3)),
            "base": rng.choice((1e4, 1e6)), "scaling": scaling, "factor": 1.0 if scaling == "plain" else rng.choice((2.0, 4.0, 8.0)),
            "far": rng.choice((0, _log(rng, 1, 1000000)))}


def draw(rng):
    op = rng.choice(("rope", "append", "decode", "decode", "evict"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    hq, hkv, d = rng.choice(_SHAPES)
    common = {"dtype": dtype, "hkv": hkv, "d": d}
    per_slot = 2 * hkv * d * SIZES[dtype]
    if op == "rope":
        return _rope("", hq=hq, tokens=_log(rng, 1, 20000), inverse=rng.random() < 0.3, **common, **_rotation(rng, d))
    paged = {"page": rng.choice((16, 32, 48, 64, 128, 256)), "pool": rng.choice(("heads", "slots"))}
    if op == "append":
        seqs = _log(rng, 1, 200)
        tokens = rng.choice((1, _log(rng, 1, max(2, 16000 // seqs))))
        lo = rng.choice((0, _log(rng, 1, 4000)))
        return _append("", hq=hq, tokens=tokens, seqs=seqs, lo=lo, hi=max(lo, _log(rng, 1, 8000)), **common, **paged, **_rotation(rng, d))
    seqs = _log(rng, 1, 128)
    room = int(1.5e9 / per_slot / seqs)   # slots per sequence: half of what the largest listed call holds
    hi = _log(rng, 1, max(2, min(room, 160000)))
    lo = _log(rng, 1, hi + 1) if rng.random() < 0.7 else hi
    lo = min(lo, hi)
    if op == "decode":
        weights = rng.random() < 0.4
        window = 0 if weights or rng.random() < 0.7 else _log(rng, 1, 4096)
        return _decode("", hq=hq, seqs=seqs, lo=lo, hi=hi, window=window, weights=weights, **common, **paged)
    keep = _log(rng, 1, hi + 1) if rng.random() < 0.7 else max(1, hi - rng.randrange(1, 300))
    first = rng.randrange(0, min(keep, 16) + 1)
    return _evict("", seqs=seqs, lo=lo, hi=hi, keep=keep, first=first, last=rng.randrange(0, min(keep - first, 512) + 1), **common, **paged)


# ---------------------------------------------------------------------------------------- inputs

def _lens(case):
    """Slots in use, ascending; their sum does not depend on the seed."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    if lo == hi:
        return [lo] * n
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [int(round(math.exp(a + (b - a) * (i / (n - 1) if n > 1 else 1.0)))) - 1 for i in range(n)]


def _capacity(case):
    """Pages per sequence."""
    more = case["tokens"] if case["op"] == "append" else 0
    return -(-(max(_lens(case)) + more) // case["page"])


def _visible(case, n):
    return min(n, case["window"]) if case.get("window") else n


def work(case):
    e, d = SIZES[case["dtype"]], case["d"]
    hkv = case["hkv"]
    if case["op"] == "rope":
        n = (case["hq"] + hkv) * case["tokens"]
        return {"bytes": 2 * n * d * e + 4 * case["axes"] * case["tokens"], "flops": 3 * n * case["rotary"]}
    if case["op"] == "append":
        t = case["tokens"] * case["seqs"]
        return {"bytes": (2 * case["hq"] + 4 * hkv) * t * d * e + 8 * hkv * t + 4 * (3 + case["axes"]) * t,
                "flops": 3 * (case["hq"] + hkv) * t * case["rotary"]}
    lens = _lens(case)
    if case["op"] == "decode":
        slots = sum(_visible(case, n) for n in lens)
        b = 2 * slots * hkv * d * e + 2 * case["seqs"] * case["hq"] * d * e + sum(-(-n // case["page"]) for n in lens) * 4
        if case["weights"]:
            b += 8 * slots * hkv
        return {"bytes": b, "flops": (4 * d + (1 if case["weights"] else 0)) * slots * case["hq"]}
    keep, moved, slots, written = case["keep"], 0.0, 0, 0
    for n in lens:
        slots += n
        written += min(n, keep)
        if n > keep:   # kept behind `keep`: the last tokens, and of the others the share that is kept
            last = min(case["last"], n - keep)
            free = max(1, n - case["first"] - case["last"])
            moved += last + (n - keep - last) * (keep - case["first"] - case["last"]) / free
    return {"bytes": int(hkv * (8 * slots + 8 * written + 4 * d * e * moved)), "flops": hkv * slots}


def _frequencies(case):
    r, f = case["rotary"], case["factor"]
    i = np.arange(r // 2, dtype=np.float64)
    base = case["base"]
    if case["scaling"] == "base":
        base = base * f ** (r / (r - 2))
    freq = base ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        freq = freq / f
    if case["scaling"] == "parts":
        turns = 8192 * freq / (2 * math.pi)
        g = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        freq = freq * (g + (1.0 - g) / f)
    magnitude = 1.0 + 0.1 * math.log(f) if case["scaling"] == "parts" else 1.0
    return freq, magnitude


def _sections(case):
    """Pairs per axis of the positions: a quarter of them follows the first one."""
    n = case["rotary"] // 2
    if case["axes"] == 1:
        return [n]
    a = n // 4
    b = (n - a) // 2
    return [a, b, n - a - b]


class _State:
    pass


def _positions(case, n, gen):
    """int32 [axes][n]: text counts on, on all axes alike; pictures have rows and columns."""
    p = torch.arange(n, dtype=torch.int64, device=DEV) + case["far"]
    if case["axes"] == 1:
        return p.to(torch.int32)[None].contiguous()
    inside = (p // 1500) % 2 == 1   # every second stretch of 1500 tokens is a picture, 60 tokens wide
    t = torch.where(inside, p - p % 1500, p)
    h = torch.where(inside, t + (p % 1500) // 60, p)
    w = torch.where(inside, t + p % 60, p)
    return torch.stack([t, h, w]).to(torch.int32).contiguous()


def _pool(case, gen, n_pages):
    shape = (n_pages, case["hkv"], case["page"], case["d"]) if case["pool"] == "heads" else (n_pages, case["page"], case["hkv"], case["d"])
    out = []
    for _ in range(2):
        x = torch.empty(shape, dtype=TYPES[case["dtype"]], device=DEV)
        for i in range(0, n_pages, 4096):
            x[i:i + 4096].normal_(generator=gen)
        out.append(x if case["pool"] == "heads" else x.transpose(1, 2))   # viewed as [page][head][slot][d]
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(7919 * int(seed) + 13)
    rng = np.random.default_rng([911, int(seed)])
    s = _State()
    s.case, dt = case, TYPES[case["dtype"]]
    hkv, d = case["hkv"], case["d"]

    def randn(*shape):
        return torch.empty(shape, dtype=dt, device=DEV).normal_(generator=gen)

    if case["op"] == "rope":
        t = case["tokens"]
        s.q, s.k = randn(case["hq"], t, d), randn(hkv, t, d)
        s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)
        s.positions = _positions(case, t, gen)
    else:
        lens = np.asarray(_lens(case), dtype=np.int64)
        rng.shuffle(lens)
        s.seqs, s.max_pages = len(lens), _capacity(case)
        more = case["tokens"] if case["op"] == "append" else 0
        need = -(-(lens + more) // case["page"])
        n_pages = int(need.sum()) + 3
        ids = rng.permutation(n_pages)[:int(need.sum())]
        table = np.full((s.seqs, s.max_pages), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = ids[at:at + n]
            at += n
        s.table = torch.from_numpy(table).to(DEV)
        s.k_pool, s.v_pool = _pool(case, gen, n_pages)
        s.lens = torch.from_numpy(lens.astype(np.int32)).to(DEV)
        slots = s.max_pages * case["page"]
        if case["op"] == "append":
            t = case["tokens"] * s.seqs
            s.q, s.k, s.v = randn(t, case["hq"], d), randn(t, hkv, d), randn(t, hkv, d)   # as a projection leaves them
            s.q_out = torch.empty_like(s.q)
            seq = np.repeat(np.arange(s.seqs), case["tokens"])
            slot = (lens[:, None] + np.arange(case["tokens"])[None]).reshape(-1)
            s.token_seq = torch.from_numpy(seq.astype(np.int32)).to(DEV)
            s.token_slot = torch.from_numpy(slot.astype(np.int32)).to(DEV)
            s.token_order = s.token_slot + case["far"]   # what was evicted before counts
            s.positions = _positions(case, t, gen)
            s.weights = torch.rand((s.seqs, hkv, slots), generator=gen, device=DEV)
            s.order = torch.full((s.seqs, hkv, slots), -1, dtype=torch.int32, device=DEV)
        elif case["op"] == "decode":
            s.q = randn(s.seqs, case["hq"], d)
            s.out = torch.empty_like(s.q)
            if case["weights"]:
                s.weights = torch.rand((s.seqs, hkv, slots), generator=gen, device=DEV)
                s.weights_out = torch.zeros_like(s.weights)
        else:
            # what a slot has received so far spans orders of magnitude, and a good part has received nothing
            w = torch.empty((s.seqs, hkv, slots), device=DEV).normal_(generator=gen).mul_(2.0).exp_()
            s.weights = torch.where(torch.rand(w.shape, generator=gen, device=DEV) < 0.1, torch.zeros_like(w), w)
            step = torch.randint(1, 4, w.shape, generator=gen, device=DEV)   # what was evicted before leaves gaps
            s.order = (step.cumsum(2) - step).to(torch.int32)
            s.weights_out, s.order_out = torch.zeros_like(s.weights), torch.zeros_like(s.order)
            s.lens_out = torch.zeros_like(s.lens)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    import paper_2507_09071_amd as bs

    case = s.case
    s.dtype = bs.BS_BF16 if case["dtype"] == "bf16" else bs.BS_F32
    if "rotary" in case:
        scaling = {"plain": bs.BS_ROPE_PLAIN, "linear": bs.BS_ROPE_LINEAR, "base": bs.BS_ROPE_BASE, "parts": bs.BS_ROPE_PARTS}[case["scaling"]]
        s.rope = bs.bs_rope_init(case["rotary"], bs.BS_ROPE_HALF if case["layout"] == "half" else bs.BS_ROPE_INTERLEAVED, case["base"], scaling,
                                 case["factor"], 8192, 32.0, 1.0, magnitude=_frequencies(case)[1], sections=_sections(case))
    if case["op"] == "rope":
        return
    s.cache = bs.KVCache.of(s.k_pool, s.v_pool, s.table, s.dtype)
    if case["op"] == "append":
        s.slots = bs.CacheSlots.of(s.weights, s.order)
    if case["op"] == "decode":
        s.slots = bs.CacheSlots.of(s.weights) if case["weights"] else None
        s.slots_out = bs.CacheSlots.of(s.weights_out) if case["weights"] else None
        n = bs.bs_attn_decode_workspace(s.cache, case["hq"], case["weights"])
    if case["op"] == "evict":
        s.slots, s.slots_out = bs.CacheSlots.of(s.weights, s.order), bs.CacheSlots.of(s.weights_out, s.order_out)
        n = bs.bs_cache_evict_workspace(s.cache, case["keep"])
    if case["op"] != "append":
        s.workspace = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------------------------------- plain forms

def _angles(case, positions):
    """cos and sin, times the magnitude, float32 [tokens][pairs]; the angle in 64 bits."""
    freq, magnitude = _frequencies(case)
    axis = torch.cat([torch.full((n,), a, dtype=torch.int64) for a, n in enumerate(_sections(case))]).to(DEV)
    angle = positions.to(torch.float64)[axis].T * torch.from_numpy(freq).to(DEV)
    return (torch.cos(angle) * magnitude).float(), (torch.sin(angle) * magnitude).float()


def _rotate(case, x, cos, sin):
    """x [..., d] in float32; cos, sin broadcast against [..., pairs]."""
    r = case["rotary"]
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], dim=-1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _slots_of(pool, table, page):
    """A pool's slots in the order of the sequences, [seq][head][slot][d], and which of them have a page."""
    n_seqs, max_pages = table.shape
    x = pool.permute(0, 2, 1, 3)[table.clamp(0, pool.shape[0] - 1).long()]   # [seq][page][slot][head][d]
    x = x.reshape(n_seqs, max_pages * page, x.shape[3], x.shape[4]).transpose(1, 2)
    return x, ((table >= 0) & (table < pool.shape[0])).repeat_interleave(page, dim=1)


def _plain_rope(s):
    cos, sin = _angles(s.case, s.positions)
    if s.case["inverse"]:
        sin = -sin
    return [_rotate(s.case, x.float(), cos, sin).to(x.dtype) for x in (s.q, s.k)]


def _plain_append(s):
    case = s.case
    cos, sin = _angles(case, s.positions)
    cos, sin = cos[:, None], sin[:, None]
    q = _rotate(case, s.q.float(), cos, sin).to(s.q.dtype)
    k = _rotate(case, s.k.float(), cos, sin).to(s.k.dtype)
    seq, slot = s.token_seq.long(), s.token_slot.long()
    page, at = s.table[seq, slot // case["page"]].long(), slot % case["page"]
    s.k_pool[page, :, at] = k
    s.v_pool[page, :, at] = s.v
    s.weights[seq, :, slot] = 0.0
    s.order[seq, :, slot] = s.token_order[:, None].expand(-1, case["hkv"])
    return [q, s.k_pool, s.v_pool, s.weights, s.order]


def _plain_decode(s):
    case = s.case
    k, there = _slots_of(s.k_pool, s.table, case["page"])
    v, _ = _slots_of(s.v_pool, s.table, case["page"])
    j = torch.arange(k.shape[2], device=DEV)
    seen = (j[None] < s.lens[:, None]) & there
    if case["window"]:
        seen = seen & (j[None] >= s.lens[:, None] - case["window"])
    g = case["hq"] // case["hkv"]
    q = s.q.float().reshape(s.seqs, case["hkv"], g, case["d"])
    score = torch.matmul(q, k.float().transpose(2, 3)) * (case["d"] ** -0.5)
    score = torch.where(seen[:, None, None], score, -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.matmul(p, torch.where(seen[:, None, :, None], v.float(), torch.zeros((), device=DEV)))
    out = out.reshape(s.seqs, case["hq"], case["d"]).to(s.q.dtype)
    if not case["weights"]:
        return [out]
    used = (j[None] < s.lens[:, None])[:, None]
    return [out, torch.where(used, s.weights + p.sum(2), s.weights_out)]


def _plain_evict(s):
    case, keep = s.case, s.case["keep"]
    slots = s.weights.shape[2]
    j = torch.arange(slots, device=DEV)
    used = (j[None] < s.lens[:, None])[:, None].expand_as(s.weights)
    newest = torch.where(used, s.order, torch.full_like(s.order, -2 ** 31)).amax(2, keepdim=True).to(torch.int64)
    safe = (s.order < case["first"]) | (s.order > newest - case["last"])
    value = torch.where(safe, math.inf, s.weights)
    value = torch.where(used, value, -math.inf)
    ranked = torch.sort(value, dim=2, descending=True, stable=True).indices   # ties: the lowest slot first
    kept = torch.zeros_like(used).scatter(2, ranked[..., :keep], True) & used
    hole = ~kept & (j < keep) & used                # evicted in front
    late = kept & (j >= keep)                       # kept behind: the i-th of them moves into the i-th hole
    source = torch.zeros((s.seqs, case["hkv"], slots + 1), dtype=torch.int64, device=DEV)
    rank = torch.where(late, late.cumsum(2) - 1, torch.full_like(ranked, slots))
    source.scatter_(2, rank, j.expand_as(ranked))
    n = min(keep, slots)
    src = torch.where(hole, source.gather(2, (hole.cumsum(2) - 1).clamp(min=0)), j.expand_as(ranked))[..., :n]
    front = used[..., :n]
    weights = s.weights_out.clone()
    order = s.order_out.clone()
    weights[..., :n] = torch.where(front, s.weights.gather(2, src), weights[..., :n])
    order[..., :n] = torch.where(front, s.order.gather(2, src), order[..., :n])
    page_of = lambda x: s.table.long()[:, None].expand(-1, case["hkv"], -1).gather(2, x // case["page"])
    head = torch.arange(case["hkv"], device=DEV)[None, :, None].expand_as(src)
    # every slot in front takes the row it keeps or the one that moves there; behind the last one, the first slot's once more
    to = torch.where(front, j[:n].expand_as(src), torch.zeros_like(src))
    src = torch.where(front, src, src[..., :1])
    for pool in (s.k_pool, s.v_pool):
        pool[page_of(to), head, to % case["page"]] = pool[page_of(src), head, src % case["page"]]
    return [s.k_pool, s.v_pool, weights, order, torch.clamp(s.lens, max=keep)]


# ---------------------------------------------------------------------------------------- the framework's calls

def _own_rope(s, bs, stream):
    bs.bs_rope_apply(s.rope, [s.q, s.k], [s.q_out, s.k_out], s.dtype, s.case["tokens"], s.case["d"], s.positions, inverse=s.case["inverse"],
                     stream=stream)
    return [s.q_out, s.k_out]


def _own_append(s, bs, stream):
    heads = lambda x: x.transpose(0, 1)   # [token][head][d], viewed as [head][token][d]
    bs.bs_cache_append(s.cache, heads(s.k), heads(s.v), s.k.shape[0], s.token_seq, s.token_slot, rope=s.rope, positions=s.positions, q=heads(s.q),
                       q_out=heads(s.q_out), slots=s.slots, token_order=s.token_order, stream=stream)
    return [s.q_out, s.k_pool, s.v_pool, s.weights, s.order]


def _own_decode(s, bs, stream):
    bs.bs_attn_decode(s.cache, s.q.transpose(0, 1), s.out.transpose(0, 1), s.lens, s.case["d"] ** -0.5, s.workspace, window=s.case["window"],
                      slots=s.slots, slots_out=s.slots_out, stream=stream)
    return [s.out, s.weights_out] if s.case["weights"] else [s.out]


def _own_evict(s, bs, stream):
    bs.bs_cache_evict(s.cache, s.lens, s.lens_out, s.case["keep"], s.case["first"], s.case["last"], s.slots, s.slots_out, s.workspace, stream=stream)
    return [s.k_pool, s.v_pool, s.weights_out, s.order_out, s.lens_out]


def run(state):
    op = state.case["op"]
    if own:
        import paper_2507_09071_amd as bs
        call = {"rope": _own_rope, "append": _own_append, "decode": _own_decode, "evict": _own_evict}[op]
        return call(state, bs, torch.cuda.current_stream().cuda_stream)
    return {"rope": _plain_rope, "append": _plain_append, "decode": _plain_decode, "evict": _plain_evict}[op](state)


# ---------------------------------------------------------------------------------------- in 64 bits, from the definitions

def _exact_rotation(case, x, positions, sign):
    """A complex number per pair, times exp(i angle)."""
    x = x.double()
    r = case["rotary"]
    freq, magnitude = _frequencies(case)
    counts = np.cumsum([0] + _sections(case))
    out = x.clone()
    for axis in range(case["axes"]):
        for i in range(counts[axis], counts[axis + 1]):
            lo, hi = (i, i + r // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
            a = positions[axis].double() * float(freq[i]) * sign
            z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.full_like(a, magnitude), a)
            out[..., lo], out[..., hi] = z.real, z.imag
    return out


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    page = case.get("page")
    if case["op"] == "rope":
        return [_exact_rotation(case, x, s.positions, -1.0 if case["inverse"] else 1.0) for x in (s.q, s.k)]
    table = s.table.cpu().numpy()
    lens = s.lens.cpu().numpy()
    if case["op"] == "append":
        rotated = [_exact_rotation(case, x.transpose(0, 1), s.positions, 1.0).transpose(0, 1) for x in (s.q, s.k)]
        k, v = s.k_pool.double(), s.v_pool.double()
        weights, order = s.weights.double(), s.order.clone()
        t = case["tokens"]
        for i in range(s.seqs):
            mine = slice(i * t, (i + 1) * t)
            slots = lens[i] + np.arange(t)
            pages = torch.from_numpy(table[i, slots // page].astype(np.int64)).to(DEV)
            at = torch.from_numpy(slots % page).to(DEV)
            k[pages, :, at], v[pages, :, at] = rotated[1][mine], s.v[mine].double()
            weights[i, :, lens[i]:lens[i] + t] = 0.0
            order[i, :, lens[i]:lens[i] + t] = s.token_order[mine]
        return [rotated[0], k, v, weights, order]
    if case["op"] == "decode":
        g = case["hq"] // case["hkv"]
        out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEV)
        weights = s.weights_out.double() if case["weights"] else None
        for i in range(s.seqs):
            n = int(lens[i])
            begin = max(0, n - case["window"]) if case["window"] else 0
            pages = torch.from_numpy(table[i, :-(-n // page)].astype(np.int64)).to(DEV)
            for h in range(case["hkv"]):
                k = s.k_pool[pages, h].reshape(-1, case["d"])[begin:n].double()
                v = s.v_pool[pages, h].reshape(-1, case["d"])[begin:n].double()
                if len(k):
                    p = torch.softmax(torch.mm(s.q[i, h * g:(h + 1) * g].double(), k.T.contiguous()) / math.sqrt(case["d"]), dim=1)
                    out[i, h * g:(h + 1) * g] = torch.mm(p, v)
                    if case["weights"]:
                        weights[i, h, begin:n] = s.weights[i, h, begin:n].double() + p.sum(0)
        return [out] + ([weights] if case["weights"] else [])
    k, v = s.k_pool.double(), s.v_pool.double()
    w, o = s.weights.cpu().numpy(), s.order.cpu().numpy()
    weights, order = s.weights_out.cpu().numpy().astype(np.float64), s.order_out.cpu().numpy()
    keep = case["keep"]
    for i in range(s.seqs):
        n = int(lens[i])
        for h in range(case["hkv"]):
            if n <= keep:
                weights[i, h, :n], order[i, h, :n] = w[i, h, :n], o[i, h, :n]
                continue
            value = w[i, h, :n].astype(np.float64)
            value[(o[i, h, :n] < case["first"]) | (o[i, h, :n].astype(np.int64) > int(o[i, h, :n].max()) - case["last"])] = np.inf
            stay = np.zeros(n, dtype=bool)
            stay[np.lexsort((np.arange(n), -value))[:keep]] = True
            to, src = np.flatnonzero(~stay[:keep]), keep + np.flatnonzero(stay[keep:])
            weights[i, h, :keep], order[i, h, :keep] = w[i, h, :keep], o[i, h, :keep]
            weights[i, h, to], order[i, h, to] = w[i, h, src], o[i, h, src]
            at = [torch.from_numpy(x).to(DEV) for x in (table[i, to // page].astype(np.int64), to % page, table[i, src // page].astype(np.int64), src % page)]
            for pool in (k, v):
                pool[at[0], h, at[1]] = pool[at[2], h, at[3]]
    return [k, v, torch.from_numpy(weights).to(DEV), torch.from_numpy(order).to(DEV), torch.from_numpy(np.minimum(lens, keep)).to(DEV)]
