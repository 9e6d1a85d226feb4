"""A grouped-head decoder's way through a cache held in 8 bits, as operators that can be timed and compared.

A case is a dict of plain values; `op` says which operator it is:
  attend   causal attention of a batch of prompts packed one behind the other, query heads sharing key/value heads;
           returns the output and the log of every row's sum
  weights  the attention weight that every token of those prompts has received, summed over the query heads that share
           its key/value head and over all queries, or over the last `window` queries of its sequence
  store    rows of keys and values into the cache: 8-bit codes, one scale for each block of 64 tokens of a head.  A whole
           prompt (`held` 0), or rows behind those that are held already
  decode   one query for each head over the cache, optionally adding the weights it gives to those accumulated so far
  evict    the cache cut to `keep` rows a head: the last `recent` tokens and, of the others, those with the largest
           accumulated weight (ties: the earlier token).  The rows that go leave holes, which rows from the end fill

The scale of a block is the smallest power of two 2^e, -60 <= e <= 60, with max|x| <= 127 * 2^e; a code is x / 2^e rounded to
the nearest integer, half to even, within [-127, 127].  A block that already holds rows keeps the larger of its own and
the new rows' scale, and its codes are rounded to it.  A block that receives rows from an eviction gets the scale of the rows
it then holds; other blocks stay as they are.
"""
import math
import random

import torch

own = False

BLOCK = 64
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------- the cases
def _ragged(n, lo, hi, mix):
    """`n` lengths in [lo, hi], the same for the same `mix`, as text."""
    r = random.Random(mix)
    return ",".join(str(r.randint(lo, hi)) for _ in range(n))


def _prompts(name, op, **kw):
    c = dict(name=name, op=op, dtype="bf16", lens="", heads=32, kv_heads=8, dim=128, fused=True)
    if op == "weights":
        c["window"] = 0
    c.update(kw)
    return c


def _cache(name, op, **kw):
    c = dict(name=name, op=op, dtype="bf16", held="", kv_heads=8, dim=128)
    if op == "store":
        c["new"] = ""
    if op == "decode":
        c.update(heads=32, weights=True)
    if op == "evict":
        c.update(keep=1024, recent=64)
    c.update(kw)
    return c


def listed():
    images = _ragged(16, 640, 739, 1)
    long_prompts = "12000,3043"
    users = _ragged(32, 600, 4000, 2)
    return [
        # A word, a sentence and a paragraph in front of a small model: latency is all there is.
        _prompts("attend_small", "attend", lens="1,37,130", heads=8, kv_heads=2, dim=64, fused=False),
        # A batch of questions about one image each, packed as they come out of a fused projection.
        _prompts("attend_images", "attend", lens=images),
        # A long document and a high-resolution image.
        _prompts("attend_long", "attend", lens=long_prompts),
        # What each token of the image batch has received, ahead of its first eviction.
        _prompts("weights_images", "weights", lens=images),
        # The same over the last 32 queries of long prompts only.
        _prompts("weights_window", "weights", lens=long_prompts, window=32),
        # The prompts of eight high-resolution images go into the cache.
        _cache("store_prompt", "store", held=",".join(["0"] * 8), new=_ragged(8, 2950, 3043, 3)),
        # One generated token of each of 32 sequences goes into the cache.
        _cache("store_step", "store", held=_ragged(32, 100, 1000, 4), new=",".join(["1"] * 32)),
        # The smallest model, in fp32, every query head with its own keys.
        _cache("decode_f32_small", "decode", dtype="f32", held="211,305", heads=8, kv_heads=8, dim=64),
        # A server's batch of users with conversations of different lengths, which keeps accumulated weights.
        _cache("decode_users", "decode", held=users),
        # Four very long conversations, five query heads to a key/value head, without weights.
        _cache("decode_long", "decode", held="65536,65001,64000,65537", heads=40, weights=False),
        # A few generated tokens past the budget: as many rows go as came.
        _cache("evict_step", "evict", held=_ragged(32, 1025, 1040, 5)),
        # Prompts of high-resolution images cut to a third.
        _cache("evict_prompt", "evict", held=",".join(["3043"] * 8), recent=128),
    ]


def _ints(text):
    return [int(x) for x in text.split(",")]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _seconds(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 1e15


def _plain_elements(case):
    """What the plain form holds in 32 bits at its largest."""
    if case["op"] in ("attend", "weights"):
        lens = _ints(case["lens"])
        rows = max(lens) if case["op"] == "attend" or not case["window"] else min(case["window"], max(lens))
        return len(lens) * case["heads"] * rows * max(lens)
    held = _ints(case["held"])
    rows = max(a + b for a, b in zip(held, _ints(case["new"]))) if case["op"] == "store" else max(held)
    return 2 * len(held) * case["kv_heads"] * rows * case["dim"]


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), _seconds(c))
    while True:
        c = _draw(rng)
        c.pop("name", None)
        if _seconds(c) <= most[c["op"]] and _plain_elements(c) <= 9.3e9:
            return c


def _draw(rng):
    op = rng.choice(["attend", "weights", "store", "decode", "decode", "evict"])
    kv_heads, group = rng.choice([1, 2, 4, 8, 8, 10]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 12, 16])
    dim = rng.choice([64, 128, 128])
    if op in ("attend", "weights"):
        n, top = _log(rng, 1, 24), _log(rng, 1, 12000)
        lens = ",".join(str(_log(rng, 1, top)) for _ in range(n))
        kw = dict(lens=lens, heads=kv_heads * group, kv_heads=kv_heads, dim=dim, fused=rng.random() < 0.6)
        if op == "weights":
            kw["window"] = rng.choice([0, 0, 1, _log(rng, 2, 700)])
        return _prompts("", op, **kw)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    n = _log(rng, 1, 48)
    if op == "store":
        new, start = _log(rng, 1, 6000), rng.choice([0, _log(rng, 1, 3000)])
        held = [rng.randint(start // 2, start) for _ in range(n)]
        step = rng.random() < 0.3
        rows = [1 if step else rng.randint((new + 1) // 2, new) for _ in range(n)]
        return _cache("", op, dtype=dtype, held=",".join(map(str, held)), new=",".join(map(str, rows)), kv_heads=kv_heads, dim=dim)
    if op == "decode":
        top = _log(rng, 1, 100000)
        held = ",".join(str(rng.randint(max(1, top // rng.choice([1, 4, 40])), top)) for _ in range(n))
        return _cache("", op, dtype=dtype, held=held, heads=kv_heads * group, kv_heads=kv_heads, dim=dim, weights=rng.random() < 0.6)
    keep = _log(rng, 1, 4000)
    over = rng.choice([1, rng.randint(1, 64), _log(rng, 1, 8000)])
    held = ",".join(str(rng.randint(max(1, keep // 2) if rng.random() < 0.15 else keep, keep + over)) for _ in range(n))
    return _cache("", op, held=held, kv_heads=kv_heads, dim=dim, keep=keep, recent=rng.choice([0, 1, rng.randint(0, min(256, keep))]) if keep > 1 else 1)


def work(case):
    """Each input read once, each output written once: 2 or 4 bytes an element, 1 a code, 4 a scale, sum, weight or id."""
    e, dim, kv = 2 if case["dtype"] == "bf16" else 4, case["dim"], case["kv_heads"]
    if case["op"] in ("attend", "weights"):
        lens, h = _ints(case["lens"]), case["heads"]
        total = sum(lens)
        if case["op"] == "attend":
            pairs = sum(t * (t + 1) // 2 for t in lens) * h
            return {"bytes": total * (2 * h + 2 * kv) * dim * e + total * h * 4, "flops": 4 * dim * pairs}
        rows = [min(t, case["window"] or t) for t in lens]
        pairs = sum(r * t - r * (r - 1) // 2 for r, t in zip(rows, lens)) * h
        return {"bytes": sum(rows) * h * (dim * e + 4) + total * kv * (dim * e + 4), "flops": 2 * dim * pairs}
    held = _ints(case["held"])
    if case["op"] == "store":
        new = _ints(case["new"])
        # the rows in, their codes out; and what comes back: the rows of the blocks that were written, as bf16
        rows = sum(n + h % BLOCK for h, n in zip(held, new))
        return {"bytes": kv * dim * 2 * (sum(new) * (e + 1) + rows * 3) + kv * sum(new) * 8, "flops": 0}
    if case["op"] == "decode":
        rows = sum(held) * kv
        return {"bytes": rows * (2 * dim + 8 / BLOCK + (8 if case["weights"] else 0)) + 2 * len(held) * case["heads"] * dim * e,
                "flops": 4 * dim * sum(held) * case["heads"]}
    # weights and ids of all rows in; the rows that stay: codes in and out, and out once more as bf16
    kept = sum(min(case["keep"], t) for t in held) * kv
    return {"bytes": sum(held) * kv * 8 + kept * (2 * dim * 2 + 8 + 2 * dim * 3), "flops": 0}


# ------------------------------------------------------------------------------------------------- inputs and handles
def _rows(g, n, kv_heads, dim, dtype):
    """Keys and values of `n` tokens, [n, heads, dim]: a tenth of the tokens lie towards the queries' direction, which is
    the first axis here; some channels of the keys are larger than others, as in trained models."""
    k = torch.randn(n, kv_heads, dim, generator=g, device="cuda")
    v = torch.randn(n, kv_heads, dim, generator=g, device="cuda")
    k[..., 0] += 2.0 * (torch.rand(n, kv_heads, generator=g, device="cuda") < 0.1)
    k[..., 3::16] *= 3.0
    return k.to(dtype), v.to(dtype)


def _queries(g, *shape, dtype):
    q = torch.randn(*shape, generator=g, device="cuda")
    q[..., 0] += math.sqrt(shape[-1])
    q[..., 3::16] /= 3.0
    return q.to(dtype)


def _starts(lens):
    t = torch.zeros(len(lens) + 1, dtype=torch.int32)
    t[1:] = torch.tensor(lens, dtype=torch.int64).cumsum(0)
    return t.cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype, dim, kv = _TORCH[case["dtype"]], case["dim"], case["kv_heads"]
    s = {"case": case}
    if case["op"] in ("attend", "weights"):
        lens, h = _ints(case["lens"]), case["heads"]
        total = sum(lens)
        q = _queries(g, total, h, dim, dtype=dtype)
        k, v = _rows(g, total, kv, dim, dtype)
        if case["fused"]:   # slices of one projection's output
            q, k, v = torch.cat([q, k, v], 1).split([h, kv, kv], 1)
        s.update(q=q, k=k, v=v, cu=_starts(lens), lens=torch.tensor(lens, device="cuda"), longest=max(lens))
        if case["op"] == "weights":
            s["lse"] = _prompt_lse(s)
            s["v"] = None
            s["capacity"] = -(-max(lens) // BLOCK) * BLOCK
            s["weights"] = torch.zeros(len(lens), kv, s["capacity"], device="cuda")
        return s
    held = _ints(case["held"])
    n, new = len(held), _ints(case["new"]) if case["op"] == "store" else [0] * len(held)
    rows = max(a + b for a, b in zip(held, new))
    cap = -(-rows // BLOCK) * BLOCK
    s["held"], s["capacity"] = torch.tensor(held, dtype=torch.int32, device="cuda"), cap
    s.update(_cache_of(g, n, kv, cap, dim, s["held"], empty=max(held) == 0))
    if case["op"] == "store":
        total = sum(new)
        s["k"], s["v"] = _rows(g, total, kv, dim, dtype)
        s["cu"] = _starts(new)
        s["total"] = s["held"] + torch.tensor(new, dtype=torch.int32, device="cuda")
        s["first"] = s["held"] // BLOCK * BLOCK
        s["window"] = max(-(-(a % BLOCK + b) // BLOCK) * BLOCK for a, b in zip(held, new))
        s["most_new"] = max(new)
    if case["op"] == "decode":
        s["q"] = _queries(g, n, case["heads"], dim, dtype=dtype)
        s["weights_out"] = torch.zeros_like(s["weights"])
    if case["op"] == "evict":
        keep_cap = -(-case["keep"] // BLOCK) * BLOCK
        # positions: the sequence has lost tokens before, and its rows stand in any order
        s["seen"] = s["held"] * 2
        some = torch.rand(n, kv, 2 * cap, generator=g, device="cuda")
        some.masked_fill_(torch.arange(2 * cap, device="cuda") >= s["seen"][:, None, None], -1.0)
        s["ids"] = some.topk(cap, dim=2).indices.to(torch.int32).contiguous()
        # many tokens have received nothing yet, and share their weight
        s["weights"] *= torch.rand(n, kv, cap, generator=g, device="cuda") < 0.8
        s["into"] = {"k": torch.zeros(n, kv, keep_cap, dim, dtype=torch.int8, device="cuda"),
                     "v": torch.zeros(n, kv, keep_cap, dim, dtype=torch.int8, device="cuda"),
                     "k_scale": torch.zeros(n, kv, keep_cap // BLOCK, device="cuda"),
                     "v_scale": torch.zeros(n, kv, keep_cap // BLOCK, device="cuda"),
                     "ids": torch.zeros(n, kv, keep_cap, dtype=torch.int32, device="cuda"),
                     "weights": torch.zeros(n, kv, keep_cap, device="cuda")}
    if own:   # the library's handles over these same tensors, and their workspaces
        from paper_2412_20105_b200 import binding as B
        names = ("k", "v", "k_scale", "v_scale", "ids", "weights")
        s["cache"] = B.Cache(*(s["codes_" + x] if x in "kv" else s[x] for x in names))
        if case["op"] == "evict":
            s["into_cache"] = B.Cache(*(s["into"][x] for x in names))
    return s


def _cache_of(g, n, kv, cap, dim, held, empty):
    """A cache that holds the first `held` rows of each sequence; what lies behind them is left over from earlier use."""
    s = {"ids": torch.arange(cap, dtype=torch.int32, device="cuda").repeat(n, kv, 1),
         "weights": torch.randn(n, kv, cap, generator=g, device="cuda").exp_().mul_(0.5)}
    if empty:
        for x in "kv":
            s["codes_" + x] = torch.zeros(n, kv, cap, dim, dtype=torch.int8, device="cuda")
            s[x + "_scale"] = torch.zeros(n, kv, cap // BLOCK, device="cuda")
        return s
    held = held[:, None, None]
    for x, rows in zip("kv", _rows(g, n * kv * cap, 1, dim, torch.bfloat16)):
        rows = rows.view(n, kv, cap, dim)
        valid = (torch.arange(cap, device="cuda") < held)[..., None]
        s["codes_" + x], s[x + "_scale"] = _quantise(rows, valid)
        left = torch.randint(-127, 128, (1, 1, cap, dim), generator=g, device="cuda", dtype=torch.int8)
        s["codes_" + x] = torch.where(valid, s["codes_" + x], left)
    return s


# --------------------------------------------------------------------------------------------------- the plain forms
def _scale_of(amax):
    """The smallest power of two 2^e, -60 <= e <= 60, with amax <= 127 * 2^e."""
    f, x = torch.frexp(amax)
    e = torch.where(f <= 127 / 128, x - 7, x - 6)
    e = torch.where(amax > 0, e, torch.full_like(e, -60)).clamp(-60, 60)
    return torch.ldexp(torch.ones_like(amax), e)


def _by_block(x):
    return x.unflatten(-2, (-1, BLOCK))


def _codes(x, scale):
    """x [..., rows, dim] as the nearest multiples of its block's scale."""
    return (_by_block(x) / scale[..., None, None]).round_().clamp_(-127, 127).flatten(-3, -2)


def _quantise(rows, valid):
    x = rows.float().masked_fill_(~valid, 0.0)
    scale = _scale_of(_by_block(x).abs().amax((-1, -2)))
    return _codes(x, scale).to(torch.int8), scale


def _values(codes, scale):
    return (_by_block(codes.float()) * scale[..., None, None]).flatten(-3, -2)


def _padded(s, x, rows):
    """[total, heads, dim] -> [sequences, heads, rows, dim] in 32 bits; places past a sequence's end hold its last row."""
    at = torch.arange(rows, device="cuda").minimum(s["lens"][:, None] - 1) + s["cu"][:-1, None]
    return x[at].float().transpose(1, 2)


def _prompt_logits(s, rows):
    """Scaled logits [sequences, kv heads, group, queries, keys] of the last `rows` queries of each sequence (all of them
    where rows is the longest length), and each query's position, negative where the sequence has no such query."""
    c = s["case"]
    t = s["longest"]
    if rows == t:
        pos = torch.arange(t, device="cuda").expand(len(s["lens"]), t)
        pos = pos.masked_fill(pos >= s["lens"][:, None], -1)
    else:
        pos = s["lens"][:, None] - rows + torch.arange(rows, device="cuda")
    q = s["q"][pos.clamp(min=0) + s["cu"][:-1, None]].float().transpose(1, 2)
    q = q.unflatten(1, (c["kv_heads"], -1)) * (1.0 / math.sqrt(c["dim"]))
    k = _padded(s, s["k"], t)
    x = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).unflatten(2, (-1, rows))
    x.masked_fill_((torch.arange(t, device="cuda") > pos[..., None])[:, None, None], -math.inf)
    return x, pos


def _prompt_lse(s):
    """The log of each row's sum, [heads, total], of the rows that the case's window asks for."""
    c = s["case"]
    rows = min(c["window"] or s["longest"], s["longest"])
    x, pos = _prompt_logits(s, rows)
    seq, i = (pos >= 0).nonzero(as_tuple=True)
    top = x.amax(-1, keepdim=True).clamp_(min=-1e30)
    lse = x.sub_(top).exp_().sum(-1, dtype=torch.float64).log_().add_(top[..., 0]).flatten(1, 2)
    out = torch.zeros(c["heads"], s["q"].shape[0], device="cuda")
    out[:, pos[seq, i] + s["cu"][seq]] = lse[seq, :, i].t().float()
    return out


def _attend_plain(s):
    c, t = s["case"], s["longest"]
    x, pos = _prompt_logits(s, t)
    top = x.amax(-1, keepdim=True).clamp_(min=-1e30)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x.flatten(2, 3), _padded(s, s["v"], t)).unflatten(2, (-1, t)).div_(total).flatten(1, 2)
    lse = total.log_().add_(top)[..., 0].flatten(1, 2)
    seq, i = (pos >= 0).nonzero(as_tuple=True)
    return {"out": out[seq, :, i].to(s["q"].dtype), "lse": lse[seq, :, i].t().contiguous()}


def _weights_plain(s):
    c, t = s["case"], s["longest"]
    rows = min(c["window"] or t, t)
    x, pos = _prompt_logits(s, rows)
    lse = s["lse"][:, pos.clamp(min=0) + s["cu"][:-1, None]].transpose(0, 1)
    got = x.sub_(lse.unflatten(1, (c["kv_heads"], -1))[..., None]).exp_().sum((2, 3))
    out = torch.zeros_like(s["weights"])
    out[..., :t] = got
    return {"weights": out}


def _store_plain(s):
    """The blocks that the new rows touch: those that stand there, moved to the block's new scale, and the new ones."""
    first, held, width, kv = s["first"][:, None], s["held"][:, None], s["window"], s["case"]["kv_heads"]
    at = first + torch.arange(width, device="cuda")                       # rows of the cache, [sequences, width]
    old, new = at < held, (at >= held) & (at < s["total"][:, None])
    inside = at.clamp(max=s["capacity"] - 1)
    blocks = inside[:, ::BLOCK] // BLOCK
    had = old[:, None, ::BLOCK]                                           # a block with rows holds them from its first place
    src = (s["cu"][:-1, None] + at - held).clamp(0, s["k"].shape[0] - 1)
    ids = torch.where((old | new)[:, None], torch.where(new[:, None], at[:, None], _at(s["ids"], inside)), 0)
    weights = torch.where(old[:, None], _at(s["weights"], inside), 0.0)
    return {"k": _store_side(s, "k", inside, blocks, src, old, new, had), "v": _store_side(s, "v", inside, blocks, src, old, new, had),
            "ids": ids.expand(-1, kv, -1).to(torch.int32), "weights": weights}


def _at(x, rows):
    return torch.gather(x, 2, rows[:, None].expand(-1, x.shape[1], -1).long())


def _store_side(s, x, inside, blocks, src, old, new, had):
    codes, scale = s["codes_" + x], _at(s[x + "_scale"], blocks)
    seq = torch.arange(len(inside), device="cuda")[:, None]
    there = codes.transpose(1, 2)[seq, inside].transpose(1, 2)            # [sequences, heads, width, dim]
    there = _values(there, scale).masked_fill_(~old[:, None, :, None], 0.0)
    come = s[x][src].float().transpose(1, 2).masked_fill(~new[:, None, :, None], 0.0)
    need = _scale_of(_by_block(come).abs().amax((-1, -2)))
    scale = torch.where(had, torch.maximum(scale, need), need)
    return _values(_codes(there + come, scale), scale).to(torch.bfloat16)


def _decode_plain(s):
    c = s["case"]
    held = s["held"][:, None, None]
    live = torch.arange(s["capacity"], device="cuda") < held
    q = s["q"].float().unflatten(1, (c["kv_heads"], -1)) * (1.0 / math.sqrt(c["dim"]))
    x = torch.matmul(q, _values(s["codes_k"], s["k_scale"]).transpose(-1, -2)).masked_fill_(~live[:, :, None], -math.inf)
    p = x.sub_(x.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    v = _values(s["codes_v"], s["v_scale"]).masked_fill_(~live[..., None], 0.0)
    out = {"out": torch.matmul(p, v).flatten(1, 2).to(s["q"].dtype)}
    if c["weights"]:
        out["weights"] = torch.where(live, s["weights"] + p.sum(2), 0.0)
    return out


def _evict_plain(s):
    c, cap = s["case"], s["capacity"]
    held, at = s["held"][:, None, None], torch.arange(cap, device="cuda")
    live = at < held
    n = held.clamp(max=c["keep"])                                         # rows that stay
    # order: the most recent tokens, then by weight, ties by position
    key = s["weights"].masked_fill(s["ids"] >= s["seen"][:, None, None] - c["recent"], math.inf).masked_fill_(~live, -math.inf)
    place = s["ids"].masked_fill(~live, 2 ** 31 - 1)
    by_id = place.argsort(dim=-1, stable=True)
    order = by_id.gather(-1, key.gather(-1, by_id).argsort(dim=-1, descending=True, stable=True))
    kept = torch.zeros_like(live.expand_as(key)).scatter_(-1, order, (at < n).expand_as(order))
    hole, mover = ~kept & (at < n), kept & (at >= n)
    movers = mover.to(torch.int8).argsort(dim=-1, descending=True, stable=True)
    src = torch.where(hole, movers.gather(-1, (hole.cumsum(-1) - 1).clamp_(min=0)), at)
    width = s["into"]["ids"].shape[2]
    src, hole = src[..., : min(width, cap)], hole[..., : min(width, cap)]
    if width > cap:
        src, hole = (torch.nn.functional.pad(x, (0, width - cap)) for x in (src, hole))
    stays = torch.arange(width, device="cuda") < n
    changed = hole.unflatten(-1, (-1, BLOCK)).any(-1)
    out = {x: _evict_side(s, x, src, stays, changed) for x in "kv"}
    out["ids"] = s["ids"].gather(-1, src).masked_fill_(~stays, 0)
    out["weights"] = s["weights"].gather(-1, src).masked_fill_(~stays, 0.0)
    out["held"] = n[:, 0, 0]
    return out


def _evict_side(s, x, src, stays, changed):
    dim = s["codes_" + x].shape[-1]
    scale = s[x + "_scale"]
    rows = s["codes_" + x].gather(2, src[..., None].expand(*src.shape, dim)).float()
    rows = rows.mul_(scale.gather(2, src // BLOCK)[..., None]).masked_fill_(~stays[..., None], 0.0)
    there = torch.nn.functional.pad(scale, (0, max(0, changed.shape[-1] - scale.shape[-1])), value=1.0)[..., : changed.shape[-1]]
    scale = torch.where(changed, _scale_of(_by_block(rows).abs().amax((-1, -2))), there)
    return _values(_codes(rows, scale), scale).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if not own:
        return {"attend": _attend_plain, "weights": _weights_plain, "store": _store_plain, "decode": _decode_plain,
                "evict": _evict_plain}[op](s)
    from paper_2412_20105_b200 import binding as B
    c = s["case"]
    if op == "attend":
        out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        lse = torch.empty(c["heads"], s["q"].shape[0], device="cuda")
        B.packed_attend(s["q"], s["k"], s["v"], s["cu"], out, lse)
        return {"out": out, "lse": lse}
    if op == "weights":
        B.packed_weights(s["q"], s["k"], s["lse"], s["cu"], s["weights"], window=c["window"])
        return {"weights": s["weights"]}
    if op == "store":
        s["cache"].store(s["k"], s["v"], s["cu"], start=s["held"])
        k, v, ids, weights = s["cache"].rows(s["total"], s["window"], first=s["first"])
        return {"k": k, "v": v, "ids": ids, "weights": weights}
    if op == "decode":
        out = torch.empty_like(s["q"])
        s["cache"].attend(s["q"], s["held"], out, weights_out=s["weights_out"] if c["weights"] else None)
        return {"out": out, "weights": s["weights_out"]} if c["weights"] else {"out": out}
    held = s["cache"].evict(s["held"], s["seen"], c["keep"], recent=c["recent"], into=s["into_cache"])
    k, v, ids, weights = s["into_cache"].rows(held, s["into"]["ids"].shape[2])
    return {"k": k, "v": v, "ids": ids, "weights": weights, "held": held}


# ------------------------------------------------------------------------------------- the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_prompts, "weights": _exact_prompts, "store": _exact_store, "decode": _exact_decode, "evict": _exact_evict}[case["op"]](s)


def _exact_prompts(s):
    c = s["case"]
    total, h, dim = s["q"].shape
    group = h // c["kv_heads"]
    weights = c["op"] == "weights"
    out = torch.zeros_like(s["weights"], dtype=torch.float64) if weights else torch.empty(total, h, dim, dtype=torch.float64, device="cuda")
    lse = torch.empty(h, total, dtype=torch.float64, device="cuda")
    cu = s["cu"].tolist()
    for b, (lo, hi) in enumerate(zip(cu, cu[1:])):
        begin = max(0, hi - lo - c["window"]) if weights and c["window"] else 0
        for head in range(h):
            k = s["k"][lo:hi, head // group].double()
            for i in range(begin, hi - lo, 2048):
                j = min(i + 2048, hi - lo)
                x = s["q"][lo + i:lo + j, head].double() @ k[:j].t() / math.sqrt(dim)
                x.masked_fill_(torch.ones(j - i, j, dtype=torch.bool, device="cuda").triu(i + 1), -math.inf)
                if weights:
                    out[b, head // group, :j] += torch.exp(x - s["lse"][head, lo + i:lo + j, None].double()).sum(0)
                else:
                    lse[head, lo + i:lo + j] = torch.logsumexp(x, 1)
                    out[lo + i:lo + j, head] = torch.softmax(x, 1) @ s["v"][lo:lo + j, head // group].double()
    return {"weights": out} if weights else {"out": out, "lse": lse}


def _exact_scale(top):
    """top: list of floats, the largest magnitude of each block."""
    got = []
    for x in top:
        e = -60
        if x > 0:
            e = max(-60, min(60, math.ceil(math.log2(x / 127.0)) - 1))
            while e < 60 and 127.0 * 2.0 ** e < x:
                e += 1
        got.append(2.0 ** e)
    return got


def _exact_store(s):
    c = s["case"]
    n, kv, cap, dim = s["codes_k"].shape
    held, total, first, cu = (s[x].tolist() for x in ("held", "total", "first", "cu"))
    got = {x: torch.zeros(n, kv, s["window"], dim, dtype=torch.float64, device="cuda") for x in "kv"}
    for b in range(n):
        for r in range(first[b], total[b], BLOCK):
            old, end = max(0, min(held[b] - r, BLOCK)), min(total[b] - r, BLOCK)
            for x in "kv":
                was = s[x + "_scale"][b, :, r // BLOCK].double()
                rows = torch.cat([s["codes_" + x][b, :, r:r + old].double() * was[:, None, None],
                                  s[x][cu[b] + r + old - held[b]:cu[b] + r + end - held[b]].double().transpose(0, 1)], 1)
                need = _exact_scale(rows[:, old:].abs().amax((1, 2)).tolist())
                scale = torch.tensor([max(a, w) if old else a for a, w in zip(need, was.tolist())], dtype=torch.float64, device="cuda")[:, None, None]
                got[x][b, :, r - first[b]:r - first[b] + end] = (rows / scale).round().clamp(-127, 127) * scale
    return {"k": got["k"], "v": got["v"], "ids": None, "weights": None}


def _exact_decode(s):
    c = s["case"]
    n, kv, cap, dim = s["codes_k"].shape
    out = torch.empty(n, c["heads"], dim, dtype=torch.float64, device="cuda")
    weights = torch.zeros(n, kv, cap, dtype=torch.float64, device="cuda")
    for b, t in enumerate(s["held"].tolist()):
        of = (torch.arange(t, device="cuda") // BLOCK)
        k, v = (s["codes_" + x][b, :, :t].double() * s[x + "_scale"][b][:, of, None].double() for x in "kv")
        x = torch.einsum("hgd,htd->hgt", s["q"][b].double().view(kv, -1, dim), k) / math.sqrt(dim)
        p = torch.softmax(x, -1)
        out[b] = torch.einsum("hgt,htd->hgd", p, v).reshape(-1, dim)
        weights[b, :, :t] = s["weights"][b, :, :t].double() + p.sum(1)
    return {"out": out, "weights": weights} if c["weights"] else {"out": out}


def _exact_evict(s):
    """The rows that stay, one head at a time, from the definition."""
    c = s["case"]
    n, kv, cap, dim = s["codes_k"].shape
    if n * kv * cap > 2e6:
        return None
    width = s["into"]["ids"].shape[2]
    got = {x: torch.zeros(n, kv, width, dim, dtype=torch.float64, device="cuda") for x in "kv"}
    w_out = torch.zeros(n, kv, width, dtype=torch.float64, device="cuda")
    ids, weights, held, seen = s["ids"].tolist(), s["weights"].double().tolist(), s["held"].tolist(), s["seen"].tolist()
    top = {}
    for b in range(n):
        keep = min(held[b], c["keep"])
        for h in range(kv):
            i, w = ids[b][h], weights[b][h]
            order = sorted(range(held[b]), key=lambda r: (i[r] < seen[b] - c["recent"], -w[r] if i[r] < seen[b] - c["recent"] else 0.0, i[r]))
            stay = set(order[:keep])
            moved = iter(sorted(r for r in stay if r >= keep))
            src = [r if r in stay else next(moved) for r in range(keep)]
            at = torch.tensor(src, device="cuda")
            w_out[b, h, :keep] = s["weights"][b, h, at].double()
            new = {r // BLOCK for r, x in enumerate(src) if x != r}
            for x in "kv":
                scale = s[x + "_scale"][b, h].double()
                rows = s["codes_" + x][b, h, at].double() * scale[at // BLOCK][:, None]
                tops = torch.nn.functional.pad(rows.abs().amax(1), (0, -keep % BLOCK)).view(-1, BLOCK).amax(1)
                need = torch.tensor(_exact_scale(tops.tolist()), dtype=torch.float64, device="cuda")
                fresh = torch.tensor([r in new for r in range(len(need))], device="cuda")
                there = torch.nn.functional.pad(scale, (0, max(0, len(need) - len(scale))))[: len(need)]
                scale = torch.where(fresh, need, there)[torch.arange(keep, device="cuda") // BLOCK][:, None]
                got[x][b, h, :keep] = (rows / scale).round().clamp(-127, 127) * scale
    return {"k": got["k"], "v": got["v"], "ids": None, "weights": w_out, "held": None}
