"""The attention operators in 64 bits on the CPU, from their definitions; shared by their tests."""
import math

import torch

E4M3 = torch.float8_e4m3fn


def heads(x, d):
    """Rows of heads as float64 [tokens, heads, D] on the CPU."""
    return x.detach().cpu().double().reshape(x.shape[0], -1, d)


def attend(q, k, v, scale, hidden=None):
    """One query head's rows q [n, D] against keys k, v [m, D]: (output, sum of the weights times |v|).  hidden: bool [n, m]; hidden keys are left out
    whatever they hold; a row without keys gives zeros."""
    n, m = q.shape[0], k.shape[0]
    if m == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    s = (q @ k.t()) * scale
    if hidden is not None:
        s = torch.where(hidden, -math.inf, s)
    top = s.max(dim=1, keepdim=True).values
    p = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    if hidden is not None:
        p = torch.where(hidden, 0.0, p)
    total = p.sum(dim=1, keepdim=True)
    w = torch.where(total > 0, p / total, 0.0)
    if torch.isfinite(v).all():
        return w @ v, w @ v.abs()
    out = torch.zeros((n, v.shape[1]), dtype=torch.float64)
    for i in range(n):                                           # only what the row sees enters its sum
        seen = torch.ones(m, dtype=torch.bool) if hidden is None else ~hidden[i]
        out[i] = (w[i, seen, None] * v[seen]).sum(dim=0)
    return out, out.abs()


def prompt(q, k, v, starts, d, causal, scale=None):
    """(output, weights times |v|), float64 [T, H * D]; rows of no sequence are NaN."""
    q, k, v = heads(q, d), heads(k, d), heads(v, d)
    group = q.shape[1] // k.shape[1]
    out, size = torch.full_like(q, math.nan), torch.full_like(q, math.nan)
    for a, b in zip(starts, starts[1:]):
        hidden = torch.ones((b - a, b - a), dtype=torch.bool).triu(1) if causal else None
        for h in range(q.shape[1]):
            out[a:b, h], size[a:b, h] = attend(q[a:b, h], k[a:b, h // group], v[a:b, h // group], scale or d ** -0.5, hidden)
    return out.flatten(1), size.flatten(1)


def cache_values(cache, scale=None):
    """float64 [pages, HK, P, D] on the CPU."""
    x = cache.detach().cpu()
    return x.double() if scale is None else x.view(E4M3).double() * float(scale)


def decode(q, k, v, tables, lengths, d, prefix_pages=(), prefix_length=0, scale=None):
    """k, v: float64 [pages, HK, P, D].  (output, weights times |v|), float64 [sequences, H * D]."""
    q = heads(q, d)
    pages, hk, page, _ = k.shape
    group = q.shape[1] // hk
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    for b, length in enumerate(lengths):
        places = [(prefix_pages[j // page], j % page) for j in range(prefix_length)]
        places += [(tables[b][j // page], j % page) for j in range(max(0, min(length, len(tables[b]) * page)))]
        places = [x for x in places if 0 <= x[0] < pages]
        at = torch.tensor(places, dtype=torch.long).reshape(-1, 2)
        kk, vv = k[at[:, 0], :, at[:, 1]], v[at[:, 0], :, at[:, 1]]
        for h in range(q.shape[1]):
            out[b, h], size[b, h] = (x[0] for x in attend(q[b, h][None], kk[:, h // group], vv[:, h // group], scale or d ** -0.5))
    return out.flatten(1), size.flatten(1)


def worst(y, out, size):
    """Largest error of a bf16 output against its bound.  Bound: half a step of the output's rounding, 2^-8 |out|; the same of every weight's
    rounding to bf16 for the second product, 2^-8 sum w |v|; and 2^-10 of that for what is float32 (scores of up to 128 products, whose
    error of 128 * 2^-24 * sum |q k| scale, about 1e-4 here, is the weights' relative error, the exponential, the sums)."""
    error = (y.detach().cpu().double() - out).abs()
    bound = 2.0 ** -8 * (out.abs() + size) + 2.0 ** -10 * size + 1e-30
    return float((error / bound).max()) if error.numel() else 0.0


def rotated(x, cos_sin, positions, pairs):
    """x float64 [T, heads, D]: the heads turned by their tokens' angles."""
    d = x.shape[2]
    row = cos_sin.detach().cpu().double()[positions]
    cos, sin = row[:, None, :d // 2], row[:, None, d // 2:]
    out = torch.empty_like(x)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if pairs else (slice(0, d // 2), slice(d // 2, None))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    return out
