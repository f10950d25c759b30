"""Attention and its cache against their definitions in 64 bits, at the sizes and masks where they can go wrong."""
import math

import pytest
import torch

import attention_reference as R
from paper_2505_14638_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = math.nan


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DEV)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def e4m3_bytes(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def prompt_inputs(seed, t, hq, hk, d):
    """As a block has them: queries and keys rows of their own, values a part of the QKV rows."""
    qkv = randn(seed, t, (hq + 2 * hk) * d).bfloat16()
    q, k = randn(seed + 1, t, hq, d).bfloat16(), randn(seed + 2, t, hk, d).bfloat16()
    return q, k, qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,hq,hk,d", [
    ([1], 4, 1, 128), ([17], 32, 8, 128), ([64], 2, 2, 64), ([65, 0, 1, 129, 31], 6, 2, 128), ([127, 128, 1], 8, 8, 64),
    ([0, 0, 300], 3, 1, 128), ([513, 2], 16, 8, 64), ([700], 8, 8, 128), ([33, 1025], 9, 3, 64),
])
def test_prompt(gpu_lib, lengths, hq, hk, d, causal):
    t = sum(lengths)
    starts = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    q, k, v = prompt_inputs(7 * t + hq, t, hq, hk, d)
    y = B.attention_prompt(q, k, v, ints(starts), causal=causal)
    torch.cuda.synchronize()
    out, size = R.prompt(q, k, v, starts, d, causal)
    assert R.worst(y, out, size) <= 1.0
    scale = torch.tensor([0.013], device=DEV)
    y8 = B.attention_prompt(q, k, v, ints(starts), causal=causal, y_scale=scale)
    assert torch.equal(y8, B.quantize_act(y, scale))


def test_prompt_of_many_sequences(gpu_lib):
    """More sequences than a wavefront has lanes, empty ones among them; rows around them stay as they were."""
    lengths = [(37 * i) % 23 for i in range(150)]
    lead, hq, hk, d = 5, 4, 2, 64
    starts = [lead + sum(lengths[:i]) for i in range(len(lengths) + 1)]
    t = starts[-1] + 9
    q, k, v = prompt_inputs(3, t, hq, hk, d)
    y = torch.full((t, hq * d), 7.0, dtype=torch.bfloat16, device=DEV)
    B.attention_prompt(q, k, v, ints(starts), out=y)
    out, size = R.prompt(q, k, v, starts, d, True)
    assert R.worst(y[lead:starts[-1]], out[lead:starts[-1]], size[lead:starts[-1]]) <= 1.0
    assert (y[:lead] == 7).all() and (y[starts[-1]:] == 7).all()


def test_prompt_scale_and_large_scores(gpu_lib):
    """Scores of hundreds, a running maximum that moves, and another softmax scale."""
    t, hq, hk, d = 400, 4, 2, 128
    q, k, v = prompt_inputs(11, t, hq, hk, d)
    k = (k.float() * torch.linspace(0.1, 30, t, device=DEV)[:, None, None]).bfloat16()
    for scale in (d ** -0.5, 0.5, 1e-3):
        y = B.attention_prompt(q, k, v, ints([0, t]), softmax_scale=scale)
        out, size = R.prompt(q, k, v, [0, t], d, True, scale)
        # scores of up to 30 * 128 * scale carry float32 errors of 2^-24 of the sums behind them: up to 128 * 2^-24 * 3000 * scale of the weights
        slack = 128 * 2.0 ** -24 * 30 * 12 * 128 * scale
        error = (y.cpu().double() - out).abs()
        assert (error <= 2.0 ** -8 * (out.abs() + size) + (2.0 ** -10 + slack) * size).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, NAN])
def test_prompt_hidden_keys_have_no_effect(gpu_lib, d, bad):
    """Infinities and NaN in keys and values that a row does not see, inside its tile too."""
    t, hq, hk = 200, 4, 2
    q, k, v = prompt_inputs(23, t, hq, hk, d)
    y = B.attention_prompt(q, k, v, ints([0, 150]))
    k2, v2 = k.clone(), v.clone()
    for at in (40, 75, 149, 150, 199):
        k2[at, :, 3] = bad
        v2[at, :, 5] = bad
    y2 = B.attention_prompt(q, k2, v2, ints([0, 150]))
    torch.cuda.synchronize()
    assert torch.equal(y[:40], y2[:40])
    # the values alone: rows from the bad one on carry it in its channel, the others are as they were
    v3 = v.clone()
    v3[77, 0, 5] = bad
    y3 = B.attention_prompt(q, k, v3, ints([0, 150])).view(t, hq, d)
    out, size = R.prompt(q, k, v3, [0, 150], d, True)
    out = out.view(t, hq, d)
    assert torch.equal(y3[:77], y.view(t, hq, d)[:77])
    assert torch.equal(y3[:, 2:], y.view(t, hq, d)[:, 2:])
    got = y3[77:150, :2, 5].cpu().double()
    assert torch.isnan(got).all() if math.isnan(bad) else torch.equal(got, out[77:150, :2, 5])
    rest = [c for c in range(d) if c != 5]
    assert torch.equal(y3[:150, :2][:, :, rest], y.view(t, hq, d)[:150, :2][:, :, rest])


def paged(seed, lengths, prefix, hk, d, page, cache, spare=3, fill=None):
    """Caches with `lengths` own tokens and a prefix in pages of random order; tokens behind a length hold `fill`."""
    gen = torch.Generator().manual_seed(seed)
    used, shared = [-(-n // page) for n in lengths], -(-prefix // page)
    pages = sum(used) + shared + spare
    order = torch.randperm(pages, generator=gen).tolist()
    width = max(1, max(used, default=1))
    tables, at = [], shared
    for n in used:
        tables.append(order[at:at + n] + [order[-1]] * (width - n))
        at += n
    k, v = (torch.randn((pages, hk, page, d), generator=gen) for _ in range(2))
    if fill is not None:
        live = torch.zeros((pages, page), dtype=torch.bool)
        for j in range(prefix):
            live[order[j // page], j % page] = True
        for b, n in enumerate(lengths):
            for j in range(n):
                live[tables[b][j // page], j % page] = True
        k, v = (torch.where(live[:, None, :, None], x, fill) for x in (k, v))
    scales = None
    if cache == "e4m3":
        scales = torch.tensor([0.011, 0.017], device=DEV)
        k, v = ((x / s).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x, s in ((k, 0.011), (v, 0.017)))
    else:
        k, v = k.bfloat16(), v.bfloat16()
    return k.to(DEV), v.to(DEV), scales, tables, order[:shared]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("lengths,prefix,hq,hk,d,page", [
    ([1], 0, 4, 1, 128, 16), ([1000], 0, 32, 8, 128, 16), ([0, 5, 64, 33], 0, 8, 2, 64, 32), ([300, 1, 0], 40, 6, 2, 128, 16),
    ([0], 1, 2, 2, 64, 16), ([0, 0], 513, 8, 8, 128, 128), ([90] * 5, 777, 40, 2, 128, 64), ([16, 17, 15], 0, 33, 1, 64, 16),
    ([2000, 31], 95, 24, 8, 64, 128), ([7] * 40, 300, 8, 2, 128, 16), ([20, 0, 3] * 3, 130, 8, 2, 128, 32), ([5] * 17, 1000, 4, 2, 64, 16),
    ([1] * 70, 2049, 6, 2, 64, 64),
])
def test_decode(gpu_lib, lengths, prefix, hq, hk, d, page, cache):
    n = len(lengths)
    k, v, scales, tables, prefix_pages = paged(n + prefix, lengths, prefix, hk, d, page, cache, fill=NAN if cache == "bf16" else None)
    q = randn(5, n, hq, d).bfloat16()
    args = dict(prefix_pages=ints(prefix_pages) if prefix else None, prefix_length=prefix, kv_scales=scales)
    y = B.attention_decode(q, k, v, ints(tables), ints(lengths), **args)
    torch.cuda.synchronize()
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q, R.cache_values(k, k_scale), R.cache_values(v, v_scale), tables, lengths, d, prefix_pages, prefix)
    assert R.worst(y, out, size) <= 1.0
    for b, length in enumerate(lengths):
        if length + prefix == 0:
            assert (y[b] == 0).all()
    y_scale = torch.tensor([0.013], device=DEV)
    y8 = B.attention_decode(q, k, v, ints(tables), ints(lengths), y_scale=y_scale, **args)
    assert torch.equal(y8, B.quantize_act(y, y_scale))


def test_decode_lengths_and_pages_out_of_range(gpu_lib):
    """Lengths beyond the table count up to its end, negative ones as zero; pages that are none hold no tokens."""
    lengths, hk, d, page = [100, 60, 48, 20], 2, 128, 16
    k, v, _, tables, _ = paged(9, lengths, 0, hk, d, page, "bf16")
    tables[1][1], tables[1][3], tables[2] = -1, 1 << 30, [-5] * len(tables[2])
    q = randn(6, 4, 4, d).bfloat16()
    told = [1 << 30, 60, 48, -7]
    y = B.attention_decode(q, k, v, ints(tables), ints(told))
    out, size = R.decode(q, R.cache_values(k), R.cache_values(v), tables, told, d)
    assert R.worst(y, out, size) <= 1.0 and (y[2] == 0).all() and (y[3] == 0).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,d", [(3, 128), (10, 64), (10, 128), (40, 64), (40, 128)])
def test_prefix_pages_out_of_range(gpu_lib, n, d, cache):
    """In each kernel that reads a prefix: by 16 rows and by 128."""
    hq, hk, page, prefix = 8, 2, 16, 500
    k, v, scales, tables, prefix_pages = paged(9, [3] * n, prefix, hk, d, page, cache, fill=NAN if cache == "bf16" else None)
    for i, bad in ((0, -1), (5, 1 << 30), (6, k.shape[0]), (7, -1), (8, -9), (31, -1)):
        prefix_pages[i] = bad
    q = randn(6, n, hq, d).bfloat16()
    y = B.attention_decode(q, k, v, ints(tables), ints([3] * n), ints(prefix_pages), prefix, scales)
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q, R.cache_values(k, k_scale), R.cache_values(v, v_scale), tables, [3] * n, d, prefix_pages, prefix)
    assert R.worst(y, out, size) <= 1.0
    y = B.attention_decode(q, k, v, ints(tables), ints([0] * n), ints([-1] * len(prefix_pages)), prefix, scales)
    assert (y == 0).all()


def test_decode_strides(gpu_lib):
    """Queries that are columns of wider rows, pages of several layers side by side, tables and outputs that are parts of larger ones."""
    lengths, hq, hk, d, page = [50, 130, 7], 8, 2, 64, 32
    k, v, _, tables, _ = paged(4, lengths, 0, hk, d, page, "bf16")
    both = torch.stack([k, v, k * 0 + NAN], dim=1)
    q = randn(8, 3, hq + 4, d).bfloat16()[:, :hq]
    wide = torch.full((3, len(tables[0]) + 3), -1, dtype=torch.int32, device=DEV)
    wide[:, :len(tables[0])] = ints(tables)
    y = torch.full((3, hq * d + 64), 3.0, dtype=torch.bfloat16, device=DEV)
    B.attention_decode(q, both[:, 0], both[:, 1], wide[:, :len(tables[0])], ints(lengths), out=y[:, :hq * d])
    assert torch.equal(y[:, :hq * d], B.attention_decode(q.contiguous(), k, v, ints(tables), ints(lengths)))
    assert (y[:, hq * d:] == 3).all()


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("t,hq,hk,d,page,cache,keep", [
    (1, 4, 1, 128, 16, "bf16", True), (37, 32, 8, 128, 16, "bf16", False), (130, 6, 2, 64, 32, "e4m3", True), (3000, 16, 8, 128, 128, "e4m3", True),
])
def test_rope_cache_write(gpu_lib, t, hq, hk, d, page, cache, keep, pairs):
    limit, n_pages = 5000, -(-t // page) + 3
    gen = torch.Generator().manual_seed(t)
    angle = torch.arange(limit, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    cos_sin = torch.cat([angle.cos(), angle.sin()], dim=1).float().to(DEV)
    positions = torch.randint(0, limit, (t,), generator=gen)
    slots = torch.randperm(n_pages * page, generator=gen)[:t]
    skipped = [i for i in range(t) if i % 7 == 5]                # padding tokens on either side of the cache
    told = slots.clone()
    told[skipped] = torch.tensor([-1, n_pages * page] * t, dtype=torch.long)[:len(skipped)]
    qkv = randn(t + 1, t, (hq + 2 * hk) * d).bfloat16()
    scales = torch.tensor([0.011, 0.017], device=DEV) if cache == "e4m3" else None
    empty = torch.zeros((n_pages, hk, page, d), dtype=torch.uint8 if scales is not None else torch.bfloat16, device=DEV)
    k_cache, v_cache = empty.clone(), empty.clone()
    q_out, k_out = (torch.full((t, h * d), 9.0, dtype=torch.bfloat16, device=DEV) for h in (hq, hk))
    B.rope_cache_write(qkv, cos_sin, positions.int().to(DEV), told.int().to(DEV), k_cache, v_cache, kv_scales=scales,
                       rope=B.ROPE_PAIRS if pairs else B.ROPE_HALVES, q_out=q_out, k_out=k_out if keep else None)
    torch.cuda.synchronize()
    x = R.heads(qkv, d)
    turned = R.rotated(x[:, :hq + hk], cos_sin, positions, pairs)
    live = [i for i in range(t) if i not in set(skipped)]
    # one rounding to bf16 of two products and a sum in float32: 2^-8 of the value and 2^-22 of the products
    ref = turned.flatten(1)
    a = torch.cat([q_out, k_out], dim=1).cpu().double() if keep else q_out.cpu().double()
    bound = 2.0 ** -8 * ref.abs() + 2.0 ** -21 * 8
    n = a.shape[1]
    assert ((a - ref[:, :n]).abs() <= bound[:, :n])[live].all()
    assert (a[skipped] == 9).all()
    if not keep:
        assert (k_out == 9).all()
    at = slots[live] // page, slots[live] % page
    for cached, rows, scale in ((k_cache, turned[:, hq:], 0 if scales is None else float(scales[0])), (v_cache, x[:, hq + hk:], 0 if scales is None else float(scales[1]))):
        full = R.cache_values(cached) if scales is None else cached.cpu().view(R.E4M3).double()
        got = full.permute(0, 2, 1, 3)[at]
        want = rows[live] if scales is None else (rows[live] / scale).clamp(-448, 448)
        # half a step: 2^-8 (bf16), 2^-4 (E4M3; below 2^-6 the step is 2^-9), and the float32 products behind it
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -18 if scales is None else 2.0 ** -4 * want.abs().clamp(min=2.0 ** -6) + 2.0 ** -18 / scale
        assert ((got - want).abs() <= bound).all()
        rest = torch.ones(n_pages, page, dtype=torch.bool)
        rest[at] = False
        assert (full.permute(0, 2, 1, 3)[rest] == 0).all()


def test_rope_in_place_and_positions_out_of_range(gpu_lib):
    t, hq, hk, d, page = 20, 4, 2, 128, 16
    cos_sin = torch.randn((50, d), generator=torch.Generator().manual_seed(1)).to(DEV)
    positions, slots = torch.arange(t).int().to(DEV), torch.arange(t).int().to(DEV)
    positions[3], positions[4] = -1, 50
    qkv = randn(2, t, (hq + 2 * hk) * d).bfloat16()
    caches = [torch.zeros((2, hk, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    k_out = torch.empty((t, hk * d), dtype=torch.bfloat16, device=DEV)
    q = B.rope_cache_write(qkv, cos_sin, positions, slots, caches[0], caches[1], k_out=k_out)
    x = qkv.clone()
    B.rope_cache_write(x, cos_sin, positions, slots, caches[2], caches[3], q_out=x[:, :hq * d], k_out=x[:, hq * d:(hq + hk) * d])
    fine = [i for i in range(t) if i not in (3, 4)]
    assert torch.equal(x[fine][:, :hq * d], q[fine]) and torch.equal(x[fine][:, hq * d:(hq + hk) * d], k_out[fine])
    assert torch.equal(x[:, (hq + hk) * d:], qkv[:, (hq + hk) * d:]) and torch.equal(caches[1], caches[3])
    assert torch.isnan(q[3:5]).all() and torch.isnan(k_out[3:5]).all()


@pytest.mark.parametrize("planes,pages,shape,dtype,copies", [
    (1, 2, (1, 16, 64), torch.uint8, 1), (4, 60, (8, 16, 128), torch.bfloat16, 20), (3, 40, (2, 128, 128), torch.bfloat16, 17), (64, 9, (3, 16, 64), torch.uint8, 4),
])
def test_copy_pages(gpu_lib, planes, pages, shape, dtype, copies):
    wide = (100 * randn(planes, planes, pages + 1, *shape)).to(dtype)
    cache = wide[:, :pages]                                      # planes further apart than their pages reach
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(pages))
    src, dst = order[:copies].tolist(), order[copies:2 * copies].tolist()
    want = wide.clone()
    want[:, dst] = want[:, src]
    B.cache_copy_pages(cache, ints(src), ints(dst))
    assert torch.equal(wide, want)
    B.cache_copy_pages(cache, ints([-1, pages, src[0]][:pages]), ints([dst[0], dst[0], pages][:pages]))   # skipped
    assert torch.equal(wide, want)
