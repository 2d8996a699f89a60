"""The attention-block operators in 64 bits on the CPU, written from their definitions, and how far a
kernel's result may be from them.

The bounds count roundings of a kernel with fp32 sums (u = 2^-24, any order of summation) whose result is
rounded once to its type (bf16: 8 significant bits, so half a unit in the last place is up to 2^-8 of the value):
  linear     a sum of k products loses at most (k + 16) u sum|x w|; activations have slopes below 1.2 and
             are evaluated to 4 u of their argument
  norm       statistics to 64 u of the largest |x| and 128 u of the deviation
  attention  a score's error e gives a weight's relative error e, numerator and denominator: 2 e; the
             weights go into the product with v as bf16 (a relative 2^-8 each, 2^-7 with the normaliser)
"""
import math

import torch

U = 2.0 ** -24


def half_ulp(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def activation(z, act):
    if act == 1:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == 2:
        return 0.5 * z * (1 + torch.special.erf(z / math.sqrt(2)))
    if act == 3:
        return z * torch.sigmoid(z)
    return z


def linear(x, w, bias, res, act, residual_first):
    """Result and bound, for tensors as the kernel gets them."""
    dtype, k = x.dtype, x.shape[1]
    x, w = x.double(), w.double()
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    r = res.double() if res is not None else torch.zeros_like(z)
    if residual_first:
        y, size = activation(z + r, act), size + r.abs()
    else:
        y = activation(z, act) + r
    bound = 1.2 * (k + 16) * U * size + 4 * U * (z.abs() + r.abs()) + 1.01 * half_ulp(dtype) * y.abs()
    return y, bound


def group_norm(x, gamma, beta, res, n, hw, groups, eps, act):
    """x: [n * hw][c]."""
    dtype, c = x.dtype, x.shape[1]
    per = c // groups
    t = x.double().reshape(n, hw, groups, per)
    dev = t - t.mean(dim=(1, 3), keepdim=True)
    inv = 1 / torch.sqrt((dev * dev).mean(dim=(1, 3), keepdim=True) + eps)
    g = gamma.double() if gamma is not None else torch.ones(c, dtype=torch.float64)
    b = beta.double() if beta is not None else torch.zeros(c, dtype=torch.float64)
    hat = (dev * inv).reshape(n * hw, c)
    largest = (t.abs().amax(dim=(1, 3), keepdim=True) * inv).expand(n, hw, groups, per).reshape(n * hw, c)
    r = res.double() if res is not None else torch.zeros_like(hat)
    z = hat * g + b
    y = activation(z + r, act)
    size = (hat * g).abs() + b.abs() + r.abs()
    bound = 1.2 * (64 * U * largest * g.abs() + 128 * U * (hat * g).abs()) + 8 * U * size + 1.01 * half_ulp(dtype) * y.abs()
    return y, bound


def attention(q, k, v, q_lens, kv_lens, causal, scale):
    """q [tokens][heads][dim], k and v [tokens][kv_heads][dim]."""
    dtype, (_, heads, dim) = q.dtype, q.shape
    group = heads // k.shape[1]
    scale = 1 / math.sqrt(dim) if scale == 0 else scale
    y = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros_like(y)
    weights = 2.0 ** -7 if dtype == torch.bfloat16 else 0.0
    at_q = at_k = 0
    for nq, nk in zip(q_lens, kv_lens):
        for i in range(nq):
            seen = min(nk, i + nk - nq + 1) if causal else nk
            if seen <= 0:
                continue
            qi = q[at_q + i].double().reshape(-1, group, dim)                                     # [kv_heads][group][dim]
            kj, vj = (t[at_k:at_k + seen].double().transpose(0, 1) for t in (k, v))                # [kv_heads][seen][dim]
            s = scale * torch.matmul(qi, kj.transpose(1, 2).contiguous())
            size = abs(scale) * torch.matmul(qi.abs(), kj.abs().transpose(1, 2).contiguous()).amax(2, keepdim=True)
            p = torch.softmax(s, dim=2)
            o, spread = torch.matmul(p, vj), torch.matmul(p, vj.abs())
            y[at_q + i] = o.reshape(heads, dim)
            b = ((4 * (dim + 8) * size + seen + 256) * U + weights) * spread + 1.01 * half_ulp(dtype) * o.abs()
            bound[at_q + i] = b.reshape(heads, dim)
        at_q, at_k = at_q + nq, at_k + nk
    return y, bound


def assert_within(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere than in the definition"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), f"{what}: infinities differ"
    err = (got - want).abs()[finite]
    over = err - bound[finite]
    if over.numel() and not bool((over <= 0).all()):
        at = int(torch.argmax(over))
        raise AssertionError(f"{what}: off by {float(err[at]):.3e}, allowed {float(bound[finite][at]):.3e} "
                             f"({int((over > 0).sum())} of {over.numel()} values)")
