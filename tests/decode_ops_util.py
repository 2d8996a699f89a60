"""The decoding step's operators in 64 bits on the CPU, written from their definitions, and how far a kernel's result may
be from them.

The bounds count roundings (u = 2^-24), of results that are rounded once to their type:
  rms_norm   the factor to 16 u (blocks of up to 16 squares may be summed in 32 bits, the rest in 64; then its own rounding),
             two products; a scale the same, and its own rounding.  8-bit integers are equal, not near.
  linear_i8  the sum is exact, its conversion one rounding, two products, two sums; activations have slopes below 1.2 and are
             evaluated to 4 u of their argument
  paged_attention  as attention of packed sequences
"""
import math

import torch

import block_ops_util as ref
from block_ops_util import U, activation, half_ulp


def smallest(dtype):
    """The step between subnormal numbers."""
    return 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149


def rows_i8(t):
    """Integers of the rows of t (64 bits) and the largest value of each; rows that are not finite: zeros, NaN."""
    most = t.abs().amax(1)
    fine = torch.isfinite(most)
    q = torch.round(127 * t / torch.where(fine & (most > 0), most, 1.0)[:, None])
    return torch.where(fine[:, None], q, 0.0).to(torch.int8), torch.where(fine, most, math.nan)


def quantize(x):
    q, most = rows_i8(x.double())
    return q, most / 127


def stream(x, res):
    return x if res is None else (x.float() + res.float()).to(x.dtype)


def rms_norm(x, res, gamma, eps, i8):
    """(h, y, bound) or (h, q, scales)."""
    h = stream(x, res)
    t = h.double() * (gamma.double() if gamma is not None else 1.0)
    factor = 1 / torch.sqrt(h.double().square().mean(1) + eps)
    if i8:
        q, most = rows_i8(t)
        bad = torch.isnan(most) | ~torch.isfinite(h.double()).all(1)
        return h, torch.where(bad[:, None], 0, q), torch.where(bad, math.nan, most * factor / 127)
    y = t * factor[:, None]
    size = 1 + gamma.double().abs() if gamma is not None else 2.0  # a product below 2^-126 is off by 2^-150, and that times gamma
    return h, y, (20 * U + 1.01 * half_ulp(x.dtype)) * y.abs() + size * 2.0 ** -149 + smallest(x.dtype)


def linear_i8(x, sx, w, sw, bias, res, act, residual_first, dtype):
    z = x.double() @ w.double().t()
    for s, at in ((sx, (slice(None), None)), (sw, (None, slice(None)))):
        if s is not None:
            z = z * s.double()[at]
    size = z.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    r = res.double() if res is not None else torch.zeros_like(z)
    if residual_first:
        y, size = activation(z + r, act), size + r.abs()
    else:
        y = activation(z, act) + r
    return y, 1.2 * 8 * U * size + 4 * U * (z.abs() + r.abs()) + 1.01 * half_ulp(dtype) * y.abs() + smallest(dtype)


def visible(n, window, sinks):
    first = max(0, n - window) if window else 0
    return list(range(min(sinks, first))) + list(range(first, n))


def paged_attention(q, k_cache, v_cache, table, kv_lens, window, sinks, scale):
    """q [seqs][heads][dim], caches [pages][positions][kv_heads][dim]."""
    y, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    page = k_cache.shape[1]
    for s, n in enumerate(kv_lens):
        n = min(max(n, 0), table.shape[1] * page)
        if n == 0:
            continue
        at = torch.tensor(visible(n, window, sinks))
        rows = table[s].long()[at // page], at % page
        y[s:s + 1], bound[s:s + 1] = ref.attention(q[s:s + 1], k_cache[rows], v_cache[rows], [1], [len(at)], False, scale)
    return y, bound


def paged_append(k, v, offsets, table, kv_lens, k_cache, v_cache):
    k_cache, v_cache = k_cache.clone(), v_cache.clone()
    pages, page = k_cache.shape[:2]
    offsets = range(len(kv_lens) + 1) if offsets is None else offsets
    for s, n in enumerate(kv_lens):
        n = min(max(n, 0), table.shape[1] * page)
        for token in range(offsets[s], offsets[s + 1]):
            p = n - (offsets[s + 1] - token)
            if p >= 0 and 0 <= int(table[s, p // page]) < pages:
                k_cache[int(table[s, p // page]), p % page] = k[token]
                v_cache[int(table[s, p // page]), p % page] = v[token]
    return k_cache, v_cache
