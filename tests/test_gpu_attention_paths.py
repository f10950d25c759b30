"""Attention and its cache where calls are large or far apart: the kernels that only many rows reach, tensors beyond 32 bits of bytes, other
streams, calls at the same time, captured calls."""
import math

import pytest
import torch

import attention_reference as R
from paper_2505_14638_amd import binding as B
from test_gpu_attention import DEV, ints, paged, prompt_inputs, randn

pytestmark = pytest.mark.gpu


def bounds(lengths, lead=0):
    return [lead + sum(lengths[:i]) for i in range(len(lengths) + 1)]


# Many rows (tiles of 128 times heads above a few hundred) have four wavefronts on rows of their own, few have pairs on the same rows.
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,hq,hk,d", [
    ([600], 96, 8, 128), ([100, 0, 1, 260, 64], 128, 16, 64), ([129, 127, 128, 33], 112, 7, 128), ([321, 320], 90, 1, 64),
    ([(37 * i) % 23 for i in range(90)], 64, 4, 64),
])
def test_prompt_of_many_rows(gpu_lib, lengths, hq, hk, d, causal):
    starts = bounds(lengths)
    t = starts[-1]
    assert -(-t // 128) * hq > 384
    q, k, v = prompt_inputs(5 * t + hq, t, hq, hk, d)
    y = B.attention_prompt(q, k, v, ints(starts), causal=causal)
    out, size = R.prompt(q, k, v, starts, d, causal)
    assert R.worst(y, out, size) <= 1.0
    scale = torch.tensor([0.013], device=DEV)
    assert torch.equal(B.attention_prompt(q, k, v, ints(starts), causal=causal, y_scale=scale), B.quantize_act(y, scale))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("t,hq,hk,d", [(900, 64, 2, 128), (900, 64, 2, 64), (400, 4, 2, 128), (400, 4, 2, 64)])
def test_values_that_are_no_numbers(gpu_lib, t, hq, hk, d, causal):
    """Infinities of both signs and NaN among the values reach the rows that see them, in their channel and their heads, and nothing else."""
    q, k, v = prompt_inputs(31, t, hq, hk, d)
    v = v.clone()
    y = B.attention_prompt(q, k, v, ints([0, t]), causal=causal).view(t, hk, hq // hk, d)
    plus, minus, none, lone = 100, 230, 333, 65
    bad = v.clone()
    bad[plus, 1, 5], bad[minus, 1, 5] = math.inf, -math.inf      # NaN where both are seen
    bad[none, 1, 6], bad[lone, 1, d - 1] = math.nan, -math.inf
    want = y.clone()
    at = (lambda i: i) if causal else (lambda i: 0)              # the first row that sees key i
    want[at(plus):, 1, :, 5] = math.inf
    want[max(at(plus), at(minus)):, 1, :, 5] = math.nan
    want[at(none):, 1, :, 6] = math.nan
    want[at(lone):, 1, :, d - 1] = -math.inf
    got = B.attention_prompt(q, k, bad, ints([0, t]), causal=causal)
    same = got.view_as(want)
    assert torch.equal(torch.isnan(same), torch.isnan(want))
    assert torch.equal(same.nan_to_num(7.0, math.inf, -math.inf), want.nan_to_num(7.0, math.inf, -math.inf))
    scale = torch.tensor([0.02], device=DEV)
    assert torch.equal(B.attention_prompt(q, k, bad, ints([0, t]), causal=causal, y_scale=scale), B.quantize_act(got, scale))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_decode_of_sequences_of_very_different_lengths(gpu_lib, cache):
    """One workgroup on thousands of tokens, whose page numbers it lists more than once, beside others on a few or none."""
    lengths, hq, hk, d, page = [9000, 4097, 0, 4096] + [(11 * i) % 50 for i in range(60)], 8, 8, 64, 16
    k, v, scales, tables, _ = paged(2, lengths, 0, hk, d, page, cache, fill=math.nan if cache == "bf16" else None)
    q = randn(5, len(lengths), hq, d).bfloat16()
    y = B.attention_decode(q, k, v, ints(tables), ints(lengths), kv_scales=scales)
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q, R.cache_values(k, k_scale), R.cache_values(v, v_scale), tables, lengths, d)
    assert R.worst(y, out, size) <= 1.0


@pytest.mark.parametrize("n", [2, 20])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_cache_beyond_32_bits(gpu_lib, kind, n):
    """Pages 2^27 elements apart, forty of them: written, copied and read where an offset in 32 bits would end elsewhere."""
    hq, hk, d, page, n_pages, far = 8, 2, 128, 16, 40, 1 << 27
    dtype = torch.bfloat16 if kind == "bf16" else torch.uint8
    pool = torch.empty(n_pages * far, dtype=dtype, device=DEV)
    k, v = (pool.as_strided((n_pages, hk, page, d), (far, page * d, d, 1), o) for o in (0, hk * page * d))
    k.zero_(), v.zero_()
    scales = torch.tensor([0.011, 0.017], device=DEV) if kind == "e4m3" else None
    prefix, own = 64, 40                                         # tokens: pages 39 .. 36, then pages 35, 3, 34 of the first sequence
    prefix_pages, table = [39, 38, 37, 36], [35, 3, 34]
    t = prefix + own
    qkv = randn(3, t, (hq + 2 * hk) * d).bfloat16()
    places = [p * page + i for p in prefix_pages + table for i in range(page)][:t]
    cos_sin = torch.cat([torch.ones(1, d // 2), torch.zeros(1, d // 2)], dim=1).to(DEV)   # no turn: the cache holds the rows
    q = B.rope_cache_write(qkv, cos_sin, ints([0] * t), ints(places), k, v, kv_scales=scales)
    rows = R.heads(qkv, d)
    assert torch.equal(q, qkv[:, :hq * d])
    near = {p: i for i, p in enumerate(prefix_pages + table)}
    kk, vv = (torch.stack([x[p] for p in prefix_pages + table]) for x in (k, v))
    if kind == "bf16":
        written = kk.permute(0, 2, 1, 3).flatten(0, 1)[:t].cpu().double()
        assert torch.equal(written, rows[:, hq:hq + hk])
    q = randn(4, n, hq, d).bfloat16()
    tables = [table] + [[table[i % 3]] * 3 for i in range(n - 1)]
    lengths = [own] + [(7 * i) % 48 for i in range(n - 1)]
    args = dict(prefix_pages=ints(prefix_pages), prefix_length=prefix, kv_scales=scales)
    y = B.attention_decode(q, k, v, ints(tables), ints(lengths), **args)
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q, R.cache_values(kk, k_scale), R.cache_values(vv, v_scale), [[near[p] for p in x] for x in tables], lengths, d,
                         [near[p] for p in prefix_pages], prefix)
    assert R.worst(y, out, size) <= 1.0
    # each page of the prefix and of the first sequence to a page near the start
    src, dst = prefix_pages + table, [0, 1, 2, 4, 5, 6, 7]
    B.cache_copy_pages(pool.as_strided((1, n_pages, 2 * hk, page, d), (0, far, page * d, d, 1)), ints(src), ints(dst))
    args["prefix_pages"] = ints(dst[:4])
    moved = [[dst[src.index(p)] for p in x] for x in tables]
    assert torch.equal(B.attention_decode(q, k, v, ints(moved), ints(lengths), **args), y)
    assert (k[8:34] == 0).all() and (v[8:34] == 0).all()


def test_prompt_rows_beyond_32_bits(gpu_lib):
    t, hq, hk, d, wide = 2200, 2, 1, 64, (1 << 20) - 8
    x = torch.empty((t, wide), dtype=torch.bfloat16, device=DEV)     # 4.6 GB
    q, k, v = prompt_inputs(6, t, hq, hk, d)
    far = [x[:, 0:128].unflatten(1, (hq, d)), x[:, 128:192].unflatten(1, (hk, d)), x[:, wide - 64:].unflatten(1, (hk, d))]
    for a, b in zip(far, (q, k, v)):
        a.copy_(b)
    y = B.attention_prompt(*far, ints([0, 9, t]), out=x[:, 512:640])
    assert torch.equal(y, B.attention_prompt(q, k, v, ints([0, 9, t])))


def test_calls_at_the_same_time_on_two_streams(gpu_lib):
    """Each with its own workspace; the tensors were made on another stream."""
    hq, hk, d, page = 32, 8, 128, 16
    calls = []
    for seed, lengths, prefix in ((1, [900, 40], 0), (2, [70] * 30, 500)):
        k, v, _, tables, prefix_pages = paged(seed, lengths, prefix, hk, d, page, "bf16")
        q = randn(seed, len(lengths), hq, d).bfloat16()
        size = B.attention_decode_workspace_bytes(len(lengths), hq, hk, d, page, len(tables[0]), prefix)
        assert size > 0
        calls.append((q, k, v, ints(tables), ints(lengths), dict(
            prefix_pages=ints(prefix_pages) if prefix else None, prefix_length=prefix,
            workspace=torch.empty(size, dtype=torch.uint8, device=DEV), out=torch.zeros((len(lengths), hq * d), dtype=torch.bfloat16, device=DEV))))
    q, k, v = prompt_inputs(8, 300, 4, 2, 64)
    want_prompt = B.attention_prompt(q, k, v, ints([0, 300]))
    starts = ints([0, 300])
    want = [B.attention_decode(*c[:5], **c[5]).clone() for c in calls]
    for c in calls:
        c[5]["out"].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(8):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                B.attention_decode(*c[:5], **c[5])
                y = B.attention_prompt(q, k, v, starts)
    torch.cuda.synchronize()
    assert all(torch.equal(c[5]["out"], w) for c, w in zip(calls, want)) and torch.equal(y, want_prompt)


def test_two_graphs_share_a_workspace(gpu_lib):
    """Replayed one after the other, in any order: nothing of a call is left for the next."""
    hq, hk, d, page, graphs = 8, 2, 128, 16, []
    sets = []
    for seed, lengths, prefix in ((1, [900, 40], 0), (2, [70, 0] * 10, 500)):
        k, v, _, tables, prefix_pages = paged(seed, lengths, prefix, hk, d, page, "bf16")
        sets.append((randn(seed, len(lengths), hq, d).bfloat16(), k, v, ints(tables), ints(lengths), ints(prefix_pages) if prefix else None, prefix))
    need = [B.attention_decode_workspace_bytes(len(s[4]), hq, hk, d, page, s[3].shape[1], s[6]) for s in sets]
    work = torch.full((max(need),), 255, dtype=torch.uint8, device=DEV)  # NaN, were it read
    want = [B.attention_decode(*s) for s in sets]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for s, y in zip(sets, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.attention_decode(*s, workspace=work, out=y)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        outs[i].zero_()
        work.fill_(255)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i], want[i])


def test_captured_prompt_follows_its_inputs(gpu_lib):
    """Rotation, cache write and attention in one graph; rows, starts, positions and slots change between the replays."""
    t, hq, hk, d, page = 200, 8, 2, 64, 16
    qkv, starts = torch.zeros((t, (hq + 2 * hk) * d), dtype=torch.bfloat16, device=DEV), ints([0, 0, 0, 0])
    positions, slots = ints([0] * t), ints([-1] * t)
    cos_sin = torch.randn((512, d), generator=torch.Generator().manual_seed(1)).to(DEV)
    k_cache, v_cache = (torch.zeros((16, hk, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k_rows, q_rows = (torch.zeros((t, h * d), dtype=torch.bfloat16, device=DEV) for h in (hk, hq))
    y = torch.zeros((t, hq * d), dtype=torch.bfloat16, device=DEV)

    def run():
        B.rope_cache_write(qkv, cos_sin, positions, slots, k_cache, v_cache, q_out=q_rows, k_out=k_rows)
        B.attention_prompt(q_rows.view(t, hq, d), k_rows.view(t, hk, d), qkv[:, (hq + hk) * d:].unflatten(1, (hk, d)), starts, out=y)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed, cuts in enumerate(([0, 200, 200, 200], [0, 64, 65, 130], [0, 0, 0, 199], [10, 80, 90, 200])):
        qkv.copy_(randn(seed, *qkv.shape))
        starts.copy_(ints(cuts))
        positions.copy_(torch.arange(t) + 7 * seed)
        slots.copy_(torch.randperm(256, generator=torch.Generator().manual_seed(seed))[:t])
        results = []
        for call in (graph.replay, run):
            for x in (k_cache, v_cache, y):
                x.zero_()
            call()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (k_cache, v_cache, y)])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        assert results[0][2][cuts[0]:cuts[-1]].any() and not results[0][2][:cuts[0]].any() and not results[0][2][cuts[-1]:].any()


@pytest.mark.parametrize("scale", [0.01, 0.013, 1 / 448, 1 / 3, 2.0 ** -7, 2.0 ** -7 * (1 - 2.0 ** -24), 2.0 ** -7 * (1 + 2.0 ** -23), -0.02, 1e-12, 1e12, 0.0, math.inf, math.nan])
def test_quantized_outputs_of_every_value(gpu_lib, scale):
    """Sequences of one token give its values, all 65536 bf16 patterns; their bytes are those of the activation quantization."""
    v = torch.arange(-32768, 32768, dtype=torch.int32, device=DEV).short().view(torch.bfloat16).view(1024, 1, 64)
    q = torch.zeros_like(v)
    s = torch.tensor([scale], device=DEV)
    y = B.attention_prompt(q, q, v, ints(list(range(1025))))
    finite = torch.isfinite(v).view_as(y)
    assert ((y - v.view_as(y))[finite].abs() <= 2.0 ** -126).all()   # values below the normal ones may count as zero
    assert torch.equal(B.attention_prompt(q, q, v, ints(list(range(1025))), y_scale=s), B.quantize_act(y, s))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("lengths,prefix,hq,hk,d", [([5000], 0, 4, 2, 128), ([8300, 3], 0, 6, 1, 64), ([8192], 8192, 4, 1, 64), ([40] * 30, 3000, 8, 1, 128), ([300] * 40, 2500, 16, 2, 64)])
def test_decode_in_many_parts(gpu_lib, lengths, prefix, hq, hk, d, cache):
    """More partial results than a wavefront joins at once, up to 128, with few rows and with many."""
    k, v, scales, tables, prefix_pages = paged(prefix + 1, lengths, prefix, hk, d, 16, cache)
    q = randn(7, len(lengths), hq, d).bfloat16()
    args = dict(prefix_pages=ints(prefix_pages) if prefix else None, prefix_length=prefix, kv_scales=scales)
    y = B.attention_decode(q, k, v, ints(tables), ints(lengths), **args)
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q, R.cache_values(k, k_scale), R.cache_values(v, v_scale), tables, lengths, d, prefix_pages, prefix)
    assert R.worst(y, out, size) <= 1.0
    y_scale = torch.tensor([0.013], device=DEV)
    assert torch.equal(B.attention_decode(q, k, v, ints(tables), ints(lengths), y_scale=y_scale, **args), B.quantize_act(y, y_scale))


def test_calls_without_tokens(gpu_lib):
    hq, hk, d = 4, 2, 64
    q, k, v = prompt_inputs(1, 0, hq, hk, d)
    assert B.attention_prompt(q, k, v, ints([0])).shape == (0, hq * d) and B.attention_prompt(q, k, v, ints([0, 0, 0])).shape == (0, hq * d)
    q, k, v = prompt_inputs(1, 3, hq, hk, d)
    assert (B.attention_prompt(q, k, v, ints([2])) == 0).all() and (B.attention_prompt(q, k, v, ints([1, 1, 1])) == 0).all()
    cache = torch.full((4, hk, 16, d), 5.0, dtype=torch.bfloat16, device=DEV)
    assert B.attention_decode(q[:0], cache, cache, ints([]).view(0, 1), ints([])).shape == (0, hq * d)
    assert (B.attention_decode(q, cache, cache, ints([]).view(3, 0), ints([7, 0, -1])) == 0).all()
    cos_sin = torch.ones((8, d), device=DEV)
    assert B.rope_cache_write(randn(1, 0, (hq + 2 * hk) * d).bfloat16(), cos_sin, ints([]), ints([]), cache, cache).shape == (0, hq * d)
    B.cache_copy_pages(cache.unsqueeze(0), ints([]), ints([]))
    torch.cuda.synchronize()
    assert (cache == 5).all()


@pytest.mark.parametrize("causal", [True, False])
def test_a_long_prompt(gpu_lib, causal):
    """30000 tokens: some rows against 64 bits.  The longest chain of float32 sums is 7500 long: 7500 * 2^-24 < 2^-11 of the result, within the bound's 2^-10."""
    t, hq, hk, d = 30000, 2, 1, 64
    q, k, v = prompt_inputs(12, t, hq, hk, d)
    y = B.attention_prompt(q, k, v, ints([0, t]), causal=causal).view(t, hq, d)
    kk, vv = R.heads(k, d)[:, 0], R.heads(v, d)[:, 0]
    rows = [0, 1, 63, 64, 127, 128, 4095, 14999, 15000, 29951, 29952, 29999]
    hidden = torch.arange(t)[None] > torch.tensor(rows)[:, None] if causal else None
    for h in range(hq):
        out, size = R.attend(R.heads(q, d)[rows, h], kk, vv, d ** -0.5, hidden)
        assert R.worst(y[rows, h], out, size) <= 1.0


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("length,prefix,n", [(150000, 0, 1), (100, 100001, 20)])
def test_long_caches(gpu_lib, length, prefix, n, cache):
    hq, hk, d, page = 2, 1, 64, 128
    k, v, scales, tables, prefix_pages = paged(3, [length] * n, prefix, hk, d, page, cache)
    q = randn(9, n, hq, d).bfloat16()
    y = B.attention_decode(q, k, v, ints(tables), ints([length] * n), ints(prefix_pages) if prefix else None, prefix, scales)
    k_scale, v_scale = (None, None) if scales is None else scales.tolist()
    out, size = R.decode(q[-1:], R.cache_values(k, k_scale), R.cache_values(v, v_scale), tables[-1:], [length], d, prefix_pages, prefix)
    assert R.worst(y[-1:], out, size) <= 1.0


@pytest.mark.parametrize("n", [2, 20])
@pytest.mark.parametrize("cache,d", [("bf16", 64), ("bf16", 128), ("e4m3", 64), ("e4m3", 128)])
def test_decode_with_values_that_are_no_numbers(gpu_lib, cache, d, n):
    """NaN behind the lengths and the prefix's end changes nothing; seen, in one channel of one key head, it reaches that channel of the rows that see it."""
    hq, hk, page, prefix = 8, 2, 32, 150                         # the prefix ends inside a page, the lengths too
    lengths = [45 + i for i in range(n)]
    k, v, scales, tables, prefix_pages = paged(5, lengths, prefix, hk, d, page, cache)
    q = randn(9, n, hq, d).bfloat16()
    none = math.nan if cache == "bf16" else 0x7F

    def run(k, v):
        y = B.attention_decode(q, k, v, ints(tables), ints(lengths), ints(prefix_pages), prefix, scales)
        return y.view(n, hk, hq // hk, d)

    y = run(k, v)
    k2, v2 = k.clone(), v.clone()
    for x in (k2, v2):
        x[prefix_pages[-1], :, prefix % page:] = none
        for b, length in enumerate(lengths):
            if length % page:
                x[tables[b][length // page], :, length % page:] = none
        x[[p for p in range(len(x)) if p not in prefix_pages and not any(p in t[:-(-m // page)] for t, m in zip(tables, lengths))]] = none
    assert torch.equal(run(k2, v2), y) and not torch.isnan(y).any()
    v3 = v2.clone()
    v3[tables[1][1], 1, 3, 7] = none                             # token 35 of sequence 1
    want = y.clone()
    want[1, 1, :, 7] = math.nan
    assert torch.equal(run(k2, v3).nan_to_num(1e30), want.nan_to_num(1e30))
    v3 = v2.clone()
    v3[prefix_pages[4], 0, 21, 3] = none                         # token 149 of the prefix, its last one
    want = y.clone()
    want[:, 0, :, 3] = math.nan
    assert torch.equal(run(k2, v3).nan_to_num(1e30), want.nan_to_num(1e30))
    k3 = k2.clone()
    k3[prefix_pages[0], 1, 0, 0] = none                          # a key: all that its head's rows become
    want = y.clone()
    want[:, 1] = math.nan
    assert torch.equal(run(k3, v2).nan_to_num(1e30), want.nan_to_num(1e30))


@pytest.mark.parametrize("hk,d", [(1, 64), (1024, 128), (4096, 64)])
def test_as_many_heads_as_there_may_be(gpu_lib, hk, d):
    hq = 4096
    starts = [0, 5, 5, 8]
    q, k, v = (randn(i, 8, h, d).bfloat16() for i, h in enumerate((hq, hk, hk)))
    y = B.attention_prompt(q, k, v, ints(starts))
    out, size = R.prompt(q, k, v, starts, d, True)
    assert R.worst(y, out, size) <= 1.0
    lengths = [20, 0, 3]
    for prefix in (0, 40):
        kc, vc, _, tables, prefix_pages = paged(prefix, lengths, prefix, hk, d, 16, "bf16", spare=1)
        y = B.attention_decode(q[:3], kc, vc, ints(tables), ints(lengths), ints(prefix_pages) if prefix else None, prefix)
        out, size = R.decode(q[:3], R.cache_values(kc), R.cache_values(vc), tables, lengths, d, prefix_pages, prefix)
        assert R.worst(y, out, size) <= 1.0
    cos_sin = torch.randn((64, d), generator=torch.Generator().manual_seed(1)).to(DEV)
    qkv = randn(3, 4, (hq + 2 * hk) * d).bfloat16()
    turned = B.rope_cache_write(qkv, cos_sin, ints([0, 63, 7, 9]), ints([0, 17, 3, 18]), kc, vc)
    want = R.rotated(R.heads(qkv, d)[:, :hq], cos_sin, torch.tensor([0, 63, 7, 9]), False).flatten(1)
    # one rounding to bf16 of two products of up to 6 and 5, and their sum, in float32
    assert ((turned.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
    at = kc[[0, 1, 0, 1], :, [0, 1, 3, 2]], vc[[0, 1, 0, 1], :, [0, 1, 3, 2]]
    assert torch.equal(at[1].flatten(1), qkv[:, (hq + hk) * d:])
    want = R.rotated(R.heads(qkv, d)[:, hq:hq + hk], cos_sin, torch.tensor([0, 63, 7, 9]), False)
    assert ((at[0].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
