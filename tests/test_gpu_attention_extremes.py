"""Attention where scores or values are infinities or NaN, where a row's weights have to come to exactly one, and where rows see nothing, against
the definition in 64 bits: the softmax of the visible scores, and the sum over the visible values alone."""
import math

import pytest
import torch

import attention_reference as R
from paper_2505_14638_amd import binding as B
from test_gpu_attention import DEV, ints, paged, prompt_inputs, randn

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def defined(q, k, v, scale, hidden=None):
    """One query head's rows q [n, D] against keys k, v [m, D], float64: (output, sum of the weights times |v|)."""
    s = (q @ k.t()) * scale
    hidden = torch.zeros_like(s, dtype=torch.bool) if hidden is None else hidden
    w = torch.softmax(torch.where(hidden, -INF, s), dim=1)
    parts = torch.where(hidden[:, :, None], 0.0, w[:, :, None] * v[None])
    return parts.sum(dim=1), parts.abs().sum(dim=1)


def agrees(y, out, size):
    """NaN where it is NaN, infinities with their signs, and within the bound of the other tests elsewhere."""
    y = y.detach().cpu().double()
    plain = torch.isfinite(out)
    assert torch.equal(torch.isnan(y), torch.isnan(out))
    assert torch.equal(y[torch.isinf(out)], out[torch.isinf(out)]) and torch.isfinite(y[plain]).all()
    assert R.worst(y[plain], out[plain], size[plain]) <= 1.0


def check_prompt(q, k, v, causal, heads):
    """The rows of some heads against the definition; E4M3 output against the quantization of the bf16 one."""
    t, hq, d = q.shape
    group = hq // k.shape[1]
    y = B.attention_prompt(q, k, v, ints([0, t]), causal=causal)
    hidden = torch.ones((t, t), dtype=torch.bool).triu(1) if causal else None
    x = [R.heads(a.reshape(t, -1), d) for a in (q, k, v)]
    for h in heads:
        agrees(y.view(t, hq, d)[:, h], *defined(x[0][:, h], x[1][:, h // group], x[2][:, h // group], d ** -0.5, hidden))
    scale = torch.tensor([0.02], device=DEV)
    assert torch.equal(B.attention_prompt(q, k, v, ints([0, t]), causal=causal, y_scale=scale), B.quantize_act(y, scale))


# tiles of 128 rows times heads: few (two wavefronts on the same rows) and many
SIZES = [(200, 4, 2, 64), (200, 4, 2, 128), (200, 200, 2, 64), (200, 200, 2, 128)]


def heads_of(hq):
    return sorted({0, hq // 2 - 1, hq // 2, hq - 1})


def infinite_values(v, at):
    """Both infinities, apart and together, and NaN among the values of one key head, a channel each."""
    v = v.clone()
    v[at, 0, 5], v[at, 0, 6], v[at, 0, 8] = INF, -INF, NAN
    v[at, 0, 7], v[at + 5, 0, 7] = INF, -INF
    return v


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("t,hq,hk,d", SIZES)
def test_scores_that_are_nan_beside_infinite_values(gpu_lib, t, hq, hk, d, causal):
    """A NaN in a query, or in a key that a row sees, makes all of the row's outputs NaN, whatever its values are."""
    q, k, v = prompt_inputs(41, t, hq, hk, d)
    v = infinite_values(v, 30)
    q[90, :, 3] = NAN
    check_prompt(q, k, v, causal, heads_of(hq))
    q[90, :, 3] = 0.5
    k[70, 0, 3] = NAN
    check_prompt(q, k, v, causal, heads_of(hq))


@pytest.mark.parametrize("prefix", [145, 150, 159, 160])
@pytest.mark.parametrize("n", [2, 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_infinite_values_at_the_end_of_a_prefix(gpu_lib, d, n, prefix, bad):
    """In the last token of a prefix, which may end inside sixteen keys or not: they reach every row that sees it as they are."""
    hq, hk, page = 8, 2, 32
    lengths = [45 + i for i in range(n)]
    k, v, _, tables, prefix_pages = paged(5, lengths, prefix, hk, d, page, "bf16", fill=NAN)
    q = randn(9, n, hq, d).bfloat16()
    args = ints(tables), ints(lengths), ints(prefix_pages), prefix
    want = B.attention_decode(q, k, v, *args).view(n, hk, hq // hk, d)
    assert torch.isfinite(want).all()
    v[prefix_pages[-1], 0, (prefix - 1) % page, 3] = bad
    want[:, 0, :, 3] = bad
    y = B.attention_decode(q, k, v, *args).view_as(want)
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(7.0, INF, -INF), want.nan_to_num(7.0, INF, -INF))


@pytest.mark.parametrize("spread", [1.0, 3.0, 8.0])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_a_row_come_to_one(gpu_lib, d, spread):
    """Where every value is one, so is every output: the sum that divides is that of the weights as they enter the product, rounded to bf16.  Both are
    float32 sums in chains of less than 512 additions, so at most 2^-14 apart, and what is within 2^-9 of one rounds to it."""
    hq, hk, t = 8, 2, 700
    q, k, _ = prompt_inputs(51, t, hq, hk, d)
    q = (q.float() * spread).bfloat16()
    one = torch.ones_like(k)
    for causal in (True, False):
        assert (B.attention_prompt(q, k, one, ints([0, t]), causal=causal) == 1).all()
        many = q.repeat(1, 12, 1)
        assert (B.attention_prompt(many, k, one, ints([0, t]), causal=causal) == 1).all()
    for cache in ("bf16", "e4m3"):
        for lengths, prefix in (([300, 1, 17] * 5, 0), ([700], 0), ([60] * 3, 0), ([30] * 100, 0), ([40] * 2, 200), ([40] * 40, 200), ([700] * 256, 0), ([1] * 4, 40000)):
            k, v, scales, tables, prefix_pages = paged(3, lengths, prefix, hk, d, 16, cache)
            v.fill_(1.0 if cache == "bf16" else 0x30)            # E4M3: 0.5 times a scale of 2
            if scales is not None:
                scales[1] = 2.0
            y = B.attention_decode(q[:len(lengths)], k, v, ints(tables), ints(lengths), ints(prefix_pages) if prefix else None, prefix, scales)
            assert (y == 1).all(), (cache, lengths, prefix)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("t,hq,hk,d", SIZES)
def test_infinite_values_under_infinite_scores(gpu_lib, t, hq, hk, d, causal):
    """A weight of exactly zero, that of a score of -infinity, makes NaN of an infinite value; a weight that is only small does not."""
    q, k, v = prompt_inputs(47, t, hq, hk, d)
    q[..., 0] = q[..., 0].abs() + 0.1
    k[..., 0] = 0.25
    v = infinite_values(v, 30)
    for at in (30, 35, 33):                                      # under both, one of a pair, neither
        bad = k.clone()
        bad[at, 0, 0] = -INF
        check_prompt(q, bad, v, causal, heads_of(hq))
    far = k.clone()
    far[30, 0, 0] = -1500.0                                      # a weight of about e^-200 or less: zero in 32 bits, not in 64
    far_q = q.clone()
    far_q[..., 0] = 2.0 if d == 128 else 1.25
    check_prompt(far_q, far, v, causal, heads_of(hq))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("t,hq,hk,d", SIZES)
def test_infinite_scores(gpu_lib, t, hq, hk, d, causal):
    """Keys with an infinity: scores of +infinity make a row NaN; those of -infinity count nothing, unless a row has no others (NaN, as 0 / 0 is)."""
    q, k, v = prompt_inputs(43, t, hq, hk, d)
    q[::3, :, 0], k[0:40, 0, 0], k[40:, 1, 0] = q[::3, :, 0].abs(), -INF, INF
    check_prompt(q, k, v, causal, heads_of(hq))
    k[:, :, 0] = -INF
    check_prompt(q, k, infinite_values(v, 30), causal, heads_of(hq))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,prefix,hq,hk", [
    ([40, 0, 5], 0, 4, 2), ([700, 0, 33], 0, 4, 2), ([20] * 300, 0, 4, 4), ([600, 0, 3], 50, 4, 2), ([5, 0] * 15, 330, 8, 2), ([0] * 30, 330, 8, 2),
])
def test_decode_of_rows_without_a_weight(gpu_lib, lengths, prefix, hq, hk, d, cache):
    """Rows with tokens whose scores are all -infinity give NaN, those without any token zeros; in each kernel, with one part and with several."""
    n = len(lengths)
    k, v, scales, tables, prefix_pages = paged(17, lengths, prefix, hk, d, 16, cache)
    one = 1.0 if cache == "bf16" else 0x38
    k[..., 0] = one
    q = randn(5, n, hq, d).bfloat16()
    args = dict(prefix_pages=ints(prefix_pages) if prefix else None, prefix_length=prefix, kv_scales=scales)
    usual = B.attention_decode(q, k, v, ints(tables), ints(lengths), **args)
    told = q.clone()
    told[:, 1, 3] = 0.0                                          # (its neighbour is changed too, and stays finite)
    told[:, 0, 0] = -INF
    y = B.attention_decode(told, k, v, ints(tables), ints(lengths), **args).view(n, hq, d)
    seen = torch.tensor([x + prefix > 0 for x in lengths])
    assert torch.isnan(y[seen, 0]).all() and (y[~seen] == 0).all() and torch.isfinite(y[:, 1:]).all()
    assert torch.equal(y[:, max(2, hq // hk):], usual.view(n, hq, d)[:, max(2, hq // hk):])
    # tokens on pages that are none: as if there were no tokens
    none = [[-1] * len(x) for x in tables]
    args["prefix_pages"] = ints([-1] * len(prefix_pages)) if prefix else None
    assert (B.attention_decode(told, k, v, ints(none), ints(lengths), **args) == 0).all()


@pytest.mark.parametrize("prefix,n", [(0, 1), (50, 1), (150, 20)])
def test_decode_of_some_infinite_scores(gpu_lib, prefix, n):
    """A whole part, and a whole wavefront's keys, of scores of -infinity count nothing beside others."""
    hq, hk, d = 4, 2, 64
    lengths = [700] * n
    k, v, _, tables, prefix_pages = paged(19, lengths, prefix, hk, d, 16, "bf16")
    q = randn(5, n, hq, d).bfloat16()
    q[..., 0] = q[..., 0].abs() + 0.1
    k[[p for x in tables for p in x[:40]], :, :, 0] = -INF       # the first 640 own tokens
    k[[p for x in tables for p in x[40:]] + prefix_pages, :, :, 0] = 0.25
    y = B.attention_decode(q, k, v, ints(tables), ints(lengths), ints(prefix_pages) if prefix else None, prefix)
    places = [prefix_pages[j // 16] * 16 + j % 16 for j in range(prefix)] + [p * 16 + j for p in tables[0] for j in range(16)][:700]
    kk, vv = (R.cache_values(x).transpose(1, 2).reshape(-1, hk, d)[places] for x in (k, v))
    for h in range(hq):
        agrees(y.view(n, hq, d)[:1, h], *defined(R.heads(q[:1].reshape(1, -1), d)[:, h], kk[:, h // 2], vv[:, h // 2], d ** -0.5))
