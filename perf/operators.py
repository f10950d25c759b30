"""Attention with a paged key/value cache, as timed cases: rotary embedding with the write into the cache, attention over
whole prompts, attention of single tokens over the cache (with a prefix that the batch shares), and copies of pages.

`listed()` names the cases, `draw()` gives more of the same ranges; `prepare()` makes what a user's program holds before the
call, `run()` is one pass through an operator, `work()` states what the pass cannot do without and `exact()` what it returns
in 64 bits.  With `own` false `run()` computes the operators from elementary torch operations, in 32 bits; with `own` true it
calls the entry points of `paper_2505_14638_amd`.

Shapes: a QKV layer's output row is H query heads, then HK key heads, then HK value heads, of D channels each; a cache holds
pages [HK, P, D] of P tokens, in bf16 or as E4M3 bytes with one static scale for the keys and one for the values.
"""
import math

import torch

own = False

E4M3 = torch.float8_e4m3fn


def _write(name, tokens, hq, hk, d, cache, page, rope="halves", keep_k=False):
    """The QKV rows of `tokens` tokens: queries and keys rotated by their positions, keys and values written into pages.
    keep_k: the rotated keys are kept as rows too, as attention over a prompt reads them."""
    return {"name": name, "kind": "write", "tokens": tokens, "hq": hq, "hk": hk, "d": d, "cache": cache, "page": page, "rope": rope,
            "keep_k": keep_k}


def _prompt(name, seqs, lo, hi, hq, hk, d, out="bf16", causal=True):
    """Attention inside each of `seqs` packed prompts of lo to hi tokens."""
    return {"name": name, "kind": "prompt", "seqs": seqs, "lo": lo, "hi": hi, "hq": hq, "hk": hk, "d": d, "out": out, "causal": causal}


def _decode(name, seqs, lo, hi, hq, hk, d, cache, page, prefix=0, out="bf16"):
    """One token of each of `seqs` sequences against its own lo to hi cached tokens, behind `prefix` tokens that all share."""
    return {"name": name, "kind": "decode", "seqs": seqs, "lo": lo, "hi": hi, "hq": hq, "hk": hk, "d": d, "cache": cache, "page": page,
            "prefix": prefix, "out": out}


def _copy(name, copies, pages, planes, hk, d, cache, page):
    """`copies` of `pages` pages copied within each of `planes` planes (keys and values of every layer)."""
    return {"name": name, "kind": "copy", "copies": copies, "pages": pages, "planes": planes, "hk": hk, "d": d, "cache": cache, "page": page}


def listed():
    return [
        # a decode step of a batch of users: one token each, the smallest write
        _write("write_decode_32", 32, 32, 8, 128, "bf16", 16),
        # the prompts of a step, 64 query heads, into an 8-bit cache
        _write("write_prompt_8192_e4m3", 8192, 64, 8, 128, "e4m3", 64, keep_k=True),
        # the smallest prompt: a few words
        _prompt("prompt_17", 1, 17, 17, 32, 8, 128),
        # a packed batch of short prompts of unequal lengths, output quantized for the O layer
        _prompt("prompt_packed_13_e4m3", 13, 1, 1531, 32, 8, 128, out="e4m3"),
        # an encoder's pass: both directions, 64 channels a head, no shared heads
        _prompt("prompt_both_ways_d64", 3, 700, 1500, 16, 16, 64, causal=False),
        # one long prompt, the largest case
        _prompt("prompt_8192", 1, 8192, 8192, 32, 8, 128),
        # one user's token, where launches count
        _decode("decode_1", 1, 1000, 1000, 32, 8, 128, "bf16", 16),
        # a decode batch of unequal lengths on 64 query heads, 8-bit cache, output quantized for the O layer
        _decode("decode_64_e4m3", 64, 200, 8192, 64, 8, 128, "e4m3", 64, out="e4m3"),
        # users of one assistant: a common instruction of 4096 tokens and a short conversation each
        _decode("prefix_4096_batch_32", 32, 1, 512, 32, 8, 128, "bf16", 16, prefix=4096),
        # the same at a large batch, the prefix ending inside a page
        _decode("prefix_8191_batch_256_e4m3", 256, 30, 1000, 64, 8, 128, "e4m3", 32, prefix=8191),
        # the last pages of sixteen sequences copied for their forks, all layers of a 32-layer model
        _copy("fork_16", 16, 128, 64, 8, 128, "bf16", 16),
        # a pool made dense after many sequences ended
        _copy("compact_400", 400, 1024, 64, 8, 128, "bf16", 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(("write", "prompt", "prompt", "prompt", "decode", "decode", "decode", "copy"))
    d, hk = rng.choice((128, 128, 64)), rng.choice((1, 2, 4, 8, 8))
    hq = hk * rng.choice((1, 3, 4, 4, 8))
    cache, page, out = rng.choice(("bf16", "e4m3")), rng.choice((16, 32, 64, 128)), rng.choice(("bf16", "e4m3"))
    if kind == "write":
        case = _write("", _log_int(rng, 1, 8192), hq, hk, d, cache, page, rng.choice(("halves", "pairs")), rng.random() < 0.5)
    elif kind == "prompt":
        seqs, hi = _log_int(rng, 1, 16), _log_int(rng, 1, 8192)
        while seqs * hi > 8192 or seqs * hq * hi * hi > 32 * 8192 * 8192 // 2:
            seqs, hi = max(1, seqs // 2), hi if seqs > 1 else hi // 2
        case = _prompt("", seqs, rng.randint(0, hi), hi, hq, hk, d, out, rng.random() < 0.8)
    elif kind == "decode":
        seqs, hi = _log_int(rng, 1, 256), _log_int(rng, 1, 16384)
        while seqs * hi * hk * d > 256 * 1024 * 8 * 128:
            hi //= 2
        case = _decode("", seqs, rng.randint(0, hi), hi, hq, hk, d, cache, page, rng.choice((0, _log_int(rng, 1, 8192))), out)
    else:
        copies, planes = _log_int(rng, 1, 400), rng.choice((1, 16, 64))
        case = _copy("", copies, 2 * copies + rng.randint(1, 200), planes, hk, d, cache, rng.choice((16, 32)))
    return dict(case, name=None)


def _lengths(case):
    """Lengths from lo to hi in a fixed irregular order; the first is the longest."""
    lo, hi, n = case["lo"], case["hi"], case["seqs"]
    return [hi - int((hi - lo) * (i * 0.6180339887498949 % 1.0) + 0.5) for i in range(n)]


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _filled_cache(gen, case, pages):
    """Keys and values as a cache holds them: [pages, HK, P, D], bf16, or E4M3 bytes (uint8) that stand for value / scale."""
    shape = (pages, case["hk"], case["page"], case["d"])
    k, v = _randn(gen, *shape), _randn(gen, *shape)
    if case["cache"] == "bf16":
        return k.bfloat16(), v.bfloat16(), None
    scales = torch.tensor([0.011, 0.013], device="cuda")
    return _to_e4m3(k / scales[0]).view(torch.uint8), _to_e4m3(v / scales[1]).view(torch.uint8), scales


def _prepare_write(case, gen):
    t, hq, hk, d, page = case["tokens"], case["hq"], case["hk"], case["d"], case["page"]
    pages = -(-t // page) + 16 if t > 512 else t + 16           # few tokens: every one is the next of a sequence of its own
    limit = 16384
    angle = torch.arange(limit, device="cuda", dtype=torch.float64)[:, None] * 5e5 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    order = torch.randperm(pages, generator=gen, device="cuda")
    if t > 512:
        slots = order[torch.arange(t, device="cuda") // page] * page + torch.arange(t, device="cuda") % page
        positions = torch.arange(t, device="cuda")
    else:
        positions = torch.randint(0, limit, (t,), generator=gen, device="cuda")
        slots = order[:t] * page + positions % page
    k_cache, v_cache, scales = _filled_cache(gen, case, pages)
    return {"case": case, "qkv": _randn(gen, t, (hq + 2 * hk) * d).bfloat16(), "cos_sin": torch.cat([angle.cos(), angle.sin()], dim=1).float(),
            "positions": positions.int(), "slots": slots.int(), "k_cache": k_cache, "v_cache": v_cache, "scales": scales,
            "q_out": torch.empty((t, hq * d), dtype=torch.bfloat16, device="cuda"),
            "k_out": torch.empty((t, hk * d), dtype=torch.bfloat16, device="cuda") if case["keep_k"] else None}


def _prepare_prompt(case, gen):
    hq, hk, d = case["hq"], case["hk"], case["d"]
    lengths = _lengths(case)
    total = sum(lengths)
    starts = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    v = _randn(gen, max(total, 1), (hq + 2 * hk) * d).bfloat16()[:total, (hq + hk) * d:]   # where the QKV layer left them
    out8 = case["out"] == "e4m3"
    return {"case": case, "q": _randn(gen, total, hq * d).bfloat16(), "k": _randn(gen, total, hk * d).bfloat16(), "v": v,
            "starts": _ints(starts), "longest": max(lengths), "y_scale": torch.tensor([0.01], device="cuda") if out8 else None,
            "y": torch.empty((total, hq * d), dtype=torch.uint8 if out8 else torch.bfloat16, device="cuda")}


def _prepare_decode(case, gen):
    hq, hk, d, page, prefix = case["hq"], case["hk"], case["d"], case["page"], case["prefix"]
    lengths = _lengths(case)
    width = max(1, -(-max(lengths) // page))
    used = [-(-n // page) for n in lengths]
    shared = -(-prefix // page)
    pages = sum(used) + shared + 8
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    tables = torch.zeros((len(lengths), width), dtype=torch.int32, device="cuda")
    at = shared
    for b, n in enumerate(used):
        tables[b, :n] = order[at:at + n]
        at += n
    k_cache, v_cache, scales = _filled_cache(gen, case, pages)
    return {"case": case, "q": _randn(gen, len(lengths), hq * d).bfloat16(), "k_cache": k_cache, "v_cache": v_cache, "scales": scales,
            "tables": tables, "lengths": _ints(lengths), "prefix_pages": order[:shared].contiguous() if prefix else None,
            "y_scale": torch.tensor([0.01], device="cuda") if case["out"] == "e4m3" else None,
            "y": torch.empty((len(lengths), hq * d), dtype=torch.uint8 if case["out"] == "e4m3" else torch.bfloat16, device="cuda")}


def _prepare_copy(case, gen):
    shape = (case["planes"], case["pages"], case["hk"], case["page"], case["d"])
    cache = torch.empty(shape, dtype=torch.bfloat16 if case["cache"] == "bf16" else torch.uint8, device="cuda")
    for plane in cache:
        x = _randn(gen, *shape[1:])
        plane.copy_(x.bfloat16() if case["cache"] == "bf16" else (50 * x).to(E4M3).view(torch.uint8))
    order = torch.randperm(case["pages"], generator=gen, device="cuda").int()
    n = case["copies"]
    return {"case": case, "cache": cache, "src": order[:n].contiguous(), "dst": order[n:2 * n].contiguous()}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"write": _prepare_write, "prompt": _prepare_prompt, "decode": _prepare_decode, "copy": _prepare_copy}[case["kind"]](case, gen)


def _values(cache):
    """A cache as the values it holds."""
    return cache.view(E4M3) if cache.dtype == torch.uint8 else cache


def _to_e4m3(x):
    return x.clamp(-448.0, 448.0).to(E4M3)


def _rotated(x, cos, sin, rope):
    """x [T, heads, D] with channel pairs (i, i + D/2) or (2i, 2i + 1) turned by the angle whose cosine and sine are given."""
    if rope == "halves":
        a, b = x.chunk(2, dim=2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=2)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=3).flatten(2)


def _run_write(st):
    case, k_cache, v_cache, scales = st["case"], st["k_cache"], st["v_cache"], st["scales"]
    hq, hk, d, page = case["hq"], case["hk"], case["d"], case["page"]
    if own:
        from paper_2505_14638_amd import binding as B
        B.rope_cache_write(st["qkv"], st["cos_sin"], st["positions"], st["slots"], k_cache, v_cache, kv_scales=scales,
                           rope=B.ROPE_HALVES if case["rope"] == "halves" else B.ROPE_PAIRS, q_out=st["q_out"], k_out=st["k_out"])
        return st["q_out"], st["k_out"], _values(k_cache), _values(v_cache)
    x = st["qkv"].view(-1, hq + 2 * hk, d).float()
    cos, sin = st["cos_sin"][st["positions"].long()][:, None].chunk(2, dim=2)
    turned, v = _rotated(x[:, :hq + hk], cos, sin, case["rope"]), x[:, hq + hk:]
    q, k = turned[:, :hq], turned[:, hq:]
    slots = st["slots"].long()
    if scales is None:
        k_cache[slots // page, :, slots % page] = k.bfloat16()
        v_cache[slots // page, :, slots % page] = v.bfloat16()
    else:
        k_cache[slots // page, :, slots % page] = _to_e4m3(k / scales[0]).view(torch.uint8)
        v_cache[slots // page, :, slots % page] = _to_e4m3(v / scales[1]).view(torch.uint8)
    return q.bfloat16().flatten(1), k.bfloat16().flatten(1) if case["keep_k"] else None, _values(k_cache), _values(v_cache)


def _finished(y, y_scale):
    """The output rows as the O layer reads them."""
    return y.bfloat16() if y_scale is None else _to_e4m3(y / y_scale)


def _run_prompt(st):
    case = st["case"]
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if own:
        from paper_2505_14638_amd import binding as B
        B.attention_prompt(st["q"].view(-1, hq, d), st["k"].view(-1, hk, d), st["v"].unflatten(1, (hk, d)), st["starts"],
                           causal=case["causal"], out=st["y"], y_scale=st["y_scale"])
        return _values(st["y"])
    # sequences padded to the longest one
    at = torch.arange(st["longest"], device="cuda")
    starts = st["starts"].long()
    there = at < (starts[1:] - starts[:-1])[:, None]
    rows = torch.where(there, starts[:-1, None] + at, 0)
    n, length = rows.shape
    q = st["q"].float()[rows].view(n, length, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, hq // hk * length, d)
    k, v = (x.float()[rows].view(n, length, hk, d).transpose(1, 2) for x in (st["k"], st["v"]))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n, hk, hq // hk, length, length) * d ** -0.5
    seen = there[:, None, None, None, :]
    if case["causal"]:
        seen = seen & (at[None, :] <= at[:, None])
    s.masked_fill_(~seen, -math.inf)
    p = torch.exp(s - s.amax(dim=4, keepdim=True))
    p = p / p.sum(dim=4, keepdim=True)
    y = torch.matmul(p.view(n, hk, hq // hk * length, length), v.contiguous()).view(n, hq, length, d).transpose(1, 2).reshape(n, length, hq * d)
    return _finished(y[there], st["y_scale"])


def _own_keys(st, cache, scale):
    """The cached tokens of each sequence as its table lists them: float32 [sequences, HK, tokens, D]."""
    x = _values(cache[st["tables"].long()]).float().transpose(1, 2).flatten(2, 3)
    return x if scale is None else x * scale


def _shared_keys(st, cache, scale):
    x = _values(cache[st["prefix_pages"].long()]).float().transpose(0, 1).flatten(1, 2)[:, :st["case"]["prefix"]]
    return x if scale is None else x * scale


def _run_decode(st):
    case = st["case"]
    n, hq, hk, d = case["seqs"], case["hq"], case["hk"], case["d"]
    if own:
        from paper_2505_14638_amd import binding as B
        B.attention_decode(st["q"].view(n, hq, d), st["k_cache"], st["v_cache"], st["tables"], st["lengths"], prefix_pages=st["prefix_pages"],
                           prefix_length=case["prefix"], kv_scales=st["scales"], out=st["y"], y_scale=st["y_scale"])
        return _values(st["y"])
    k_scale, v_scale = (None, None) if st["scales"] is None else (st["scales"][0], st["scales"][1])
    q = st["q"].float().view(n, hk, hq // hk, d) * d ** -0.5
    k, v = _own_keys(st, st["k_cache"], k_scale), _own_keys(st, st["v_cache"], v_scale)
    s = torch.matmul(q, k.transpose(2, 3).contiguous())
    there = torch.arange(k.shape[2], device="cuda") < st["lengths"][:, None, None, None]
    s.masked_fill_(~there, -math.inf)
    if case["prefix"]:
        k1, v1 = _shared_keys(st, st["k_cache"], k_scale), _shared_keys(st, st["v_cache"], v_scale)
        rows = q.transpose(0, 1).reshape(hk, n * (hq // hk), d)
        s1 = torch.matmul(rows, k1.transpose(1, 2).contiguous()).view(hk, n, hq // hk, -1).transpose(0, 1)
        s = torch.cat([s1, s], dim=3)
    p = torch.exp(s - s.amax(dim=3, keepdim=True).clamp(min=-3e38))
    total = p.sum(dim=3, keepdim=True)
    y = torch.matmul(p[..., case["prefix"]:].contiguous(), v.contiguous())
    if case["prefix"]:
        p1 = p[..., :case["prefix"]].transpose(0, 1).reshape(hk, n * (hq // hk), -1)
        y = y + torch.matmul(p1, v1.contiguous()).view(hk, n, hq // hk, d).transpose(0, 1)
    y = torch.where(total > 0, y / total, 0.0)
    return _finished(y.reshape(n, hq * d), st["y_scale"])


def _run_copy(st):
    cache = st["cache"]
    if own:
        from paper_2505_14638_amd import binding as B
        B.cache_copy_pages(cache, st["src"], st["dst"])
    else:
        cache[:, st["dst"].long()] = cache[:, st["src"].long()]
    return _values(cache)


def run(state):
    return {"write": _run_write, "prompt": _run_prompt, "decode": _run_decode, "copy": _run_copy}[state["case"]["kind"]](state)


def work(case):
    size = 2 if case.get("cache") == "bf16" else 1
    hk, d = case["hk"], case["d"]
    if case["kind"] == "write":
        t, hq = case["tokens"], case["hq"]
        # the QKV rows, a table row, a position and a slot for every token; the rotated queries (and keys), the cache's entries
        return {"bytes": t * ((hq + 2 * hk) * d * 2 + d * 4 + 8 + (hq + (hk if case["keep_k"] else 0)) * d * 2 + 2 * hk * d * size),
                "flops": 3 * t * (hq + hk) * d}
    if case["kind"] == "copy":
        return {"bytes": case["copies"] * (2 * case["planes"] * hk * case["page"] * d * size + 8), "flops": 0}
    hq, lengths = case["hq"], _lengths(case)
    out = 2 if case["out"] == "bf16" else 1
    if case["kind"] == "prompt":
        t = sum(lengths)
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)
        return {"bytes": max(1, t) * (hq * (2 + out) + 4 * hk) * d, "flops": 4 * d * hq * pairs}
    tokens = sum(lengths) + case["prefix"]
    return {"bytes": 2 * size * tokens * hk * d + case["seqs"] * hq * d * (2 + out), "flops": 4 * d * hq * (sum(lengths) + case["seqs"] * case["prefix"])}


def _softmax_rows(q, k, v, hidden=None):
    """Attention of rows q [HK, rows, D] to keys k [HK, keys, D] in 64 bits; a row that sees no key gives zeros."""
    if k.shape[1] == 0:
        return torch.zeros_like(q)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(q.shape[2])
    if hidden is not None:
        s = s.masked_fill(hidden, -math.inf)
    return torch.matmul(torch.softmax(s, dim=2), v)


def _exact_write(st):
    case, t = st["case"], st["case"]["tokens"]
    hq, hk, d, page = case["hq"], case["hk"], case["d"], case["page"]
    x = st["qkv"].double().view(t, hq + 2 * hk, d)
    table = st["cos_sin"].double()[st["positions"].long()].view(t, 1, d)
    turn = torch.complex(table[..., :d // 2], table[..., d // 2:])
    if case["rope"] == "halves":
        z = torch.complex(x[:, :hq + hk, :d // 2], x[:, :hq + hk, d // 2:]) * turn
        z = torch.cat([z.real, z.imag], dim=2)
    else:
        z = torch.view_as_real(torch.view_as_complex(x[:, :hq + hk].unflatten(2, (d // 2, 2)).contiguous()) * turn).flatten(2)
    caches = []
    for i, (cache, rows) in enumerate(((st["k_cache"], z[:, hq:]), (st["v_cache"], x[:, hq + hk:]))):
        full = _values(cache).double()
        rows = rows if st["scales"] is None else (rows / st["scales"][i].double()).clamp(-448.0, 448.0)
        full.view(-1, hk, page, d).transpose(1, 2)[st["slots"].long() // page, st["slots"].long() % page] = rows
        caches.append(full)
    return z[:, :hq].flatten(1), z[:, hq:].flatten(1) if case["keep_k"] else None, caches[0], caches[1]


def _exact_prompt(st):
    case = st["case"]
    hq, hk, d = case["hq"], case["hk"], case["d"]
    y = torch.zeros((st["q"].shape[0], hq, d), dtype=torch.float64, device="cuda")
    starts = st["starts"].tolist()
    for a, b in zip(starts, starts[1:]):
        k, v = (st[x][a:b].double().view(b - a, hk, d).transpose(0, 1).contiguous() for x in ("k", "v"))
        for lo in range(a, b, 1024):                            # rows in chunks, one query head of each shared head at a time
            hi = min(b, lo + 1024)
            hidden = None
            if case["causal"]:
                hidden = torch.arange(b - a, device="cuda")[None, :] > torch.arange(lo - a, hi - a, device="cuda")[:, None]
            for g in range(hq // hk):
                rows = st["q"][lo:hi].double().view(hi - lo, hk, hq // hk, d)[:, :, g].transpose(0, 1).contiguous()
                y.view(-1, hk, hq // hk, d)[lo:hi, :, g] = _softmax_rows(rows, k, v, hidden).transpose(0, 1)
    return y.flatten(1)


def _exact_decode(st):
    case = st["case"]
    hq, hk, d, prefix = case["hq"], case["hk"], case["d"], case["prefix"]
    shared = st["prefix_pages"].long() if prefix else torch.zeros(0, dtype=torch.long, device="cuda")

    def tokens(cache, i, pages, count):
        x = _values(cache[pages]).double().transpose(0, 1).reshape(hk, -1, d)[:, :count]
        return x if st["scales"] is None else x * st["scales"][i].double()

    front = [tokens(st[c], i, shared, prefix) for i, c in enumerate(("k_cache", "v_cache"))]
    y = []
    for b, count in enumerate(st["lengths"].tolist()):
        k, v = (torch.cat([front[i], tokens(st[c], i, st["tables"][b].long(), count)], dim=1) for i, c in enumerate(("k_cache", "v_cache")))
        y.append(_softmax_rows(st["q"][b].double().view(hk, hq // hk, d), k, v).reshape(hq * d))
    return torch.stack(y)


def _exact_copy(st):
    # a permutation of whole pages, one plane at a time
    source = torch.arange(st["case"]["pages"], device="cuda").index_copy(0, st["dst"].long(), st["src"].long())
    moved = torch.empty_like(st["cache"])
    for i, plane in enumerate(st["cache"]):
        torch.index_select(plane, 0, source, out=moved[i])
    return _values(moved)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("write", "copy"):
        return {"write": _exact_write, "copy": _exact_copy}[case["kind"]](st)
    y = {"prompt": _exact_prompt, "decode": _exact_decode}[case["kind"]](st)
    return y if st["y_scale"] is None else (y / st["y_scale"].double()).clamp(-448.0, 448.0)
