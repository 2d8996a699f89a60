"""Host logic of the attention-block operators: what their descriptors may say, and that the oracles in
block_ops_util agree with brute force."""
import math

import pytest
import torch

import paper_2406_09425_amd as S
import block_ops_util as ref

LINEAR = dict(m=4, n=8, k=16, dtype=S.SGPRS_F32)
NORM = dict(n=2, hw=9, c=32, groups=4, dtype=S.SGPRS_BF16, eps=1e-5)
ATTENTION = dict(n_seqs=2, total_q=7, total_kv=20, max_q=5, max_kv=12, heads=4, kv_heads=2, head_dim=64, dtype=S.SGPRS_BF16)


def need(kind, **change):
    if kind == "linear":
        return S.sgprs_linear_workspace(S.LinearDesc(**{**LINEAR, **change}), 256)
    if kind == "norm":
        return S.sgprs_group_norm_workspace(S.GroupNormDesc(**{**NORM, **change}), 256)
    return S.sgprs_attention_workspace(S.AttentionDesc(**{**ATTENTION, **change}), 256)


def test_descriptors_that_are_fine():
    for kind, change in [("linear", {}), ("linear", dict(m=0)), ("linear", dict(ldx=17, ldw=16, ldr=9, ldy=8, act=3, residual_first=1)), ("norm", {}),
                         ("norm", dict(n=0)), ("norm", dict(eps=0.0, act=1, ldx=33)), ("attention", {}), ("attention", dict(total_kv=0, max_kv=0)),
                         ("attention", dict(total_q=0, max_q=0)), ("attention", dict(ldq=512, hq=128, causal=1, scale=-0.5))]:
        assert need(kind, **change) >= 0


@pytest.mark.parametrize("kind,change,status", [
    ("linear", dict(dtype=7), -5), ("linear", dict(act=4), -5), ("linear", dict(act=-1), -5), ("linear", dict(m=-1), -1), ("linear", dict(n=0), -1),
    ("linear", dict(k=0), -1), ("linear", dict(residual_first=2), -1), ("linear", dict(ldx=15), -1), ("linear", dict(ldw=-16), -1),
    ("linear", dict(ldr=7), -1), ("linear", dict(ldy=7), -1), ("linear", dict(ldx=(1 << 20) + 1), -5), ("linear", dict(ldy=1 << 40), -5),
    ("norm", dict(dtype=2), -5), ("norm", dict(act=9), -5), ("norm", dict(n=-1), -1), ("norm", dict(hw=0), -1), ("norm", dict(c=0), -1),
    ("norm", dict(groups=0), -1), ("norm", dict(groups=5), -1), ("norm", dict(eps=-1.0), -1), ("norm", dict(eps=math.nan), -1),
    ("norm", dict(eps=math.inf), -1), ("norm", dict(ldx=31), -1), ("norm", dict(ldr=1), -1), ("norm", dict(ldy=1 << 21), -5),
    ("attention", dict(dtype=5), -5), ("attention", dict(n_seqs=0), -1), ("attention", dict(heads=0), -1), ("attention", dict(heads=3), -1),
    ("attention", dict(kv_heads=0), -1), ("attention", dict(head_dim=0), -1), ("attention", dict(head_dim=12), -5), ("attention", dict(head_dim=136), -5),
    ("attention", dict(total_q=-1), -1), ("attention", dict(max_q=8), -1), ("attention", dict(max_q=0), -1), ("attention", dict(max_kv=21), -1),
    ("attention", dict(max_kv=0), -1), ("attention", dict(causal=2), -1), ("attention", dict(scale=math.inf), -1), ("attention", dict(scale=math.nan), -1),
    ("attention", dict(ldq=252), -5), ("attention", dict(hk=68), -5), ("attention", dict(ldv=56), -1), ("attention", dict(ho=-64), -1),
    ("attention", dict(ldo=1 << 21), -5), ("attention", dict(total_q=(1 << 30) + 1, max_q=1), -5)])
def test_descriptors_that_are_refused(kind, change, status):
    with pytest.raises(S.SgprsError) as e:
        need(kind, **change)
    assert e.value.status == status, str(e.value)


def test_null_and_partition_arguments_are_refused():
    lib = S.lib()
    assert lib.sgprs_linear(None, None, None, None, None, None, None, 0, None, 0) == -1
    assert lib.sgprs_group_norm(None, None, None, None, None, None, None, 0, None, 0) == -1
    assert lib.sgprs_attention(None, None, None, None, None, None, None, None, 0, None, 0) == -1
    for cus in (0, -3, 513):
        with pytest.raises(S.SgprsError):
            S.sgprs_linear_workspace(S.LinearDesc(**LINEAR), cus)
    with pytest.raises(S.SgprsError):
        S.sgprs_linear(S.LinearDesc(**LINEAR), 16, 16, None, None, 32, None, 0, None, 0)


def test_the_definitions_agree_with_brute_force():
    g = torch.Generator().manual_seed(1)
    x, w, b, r = (torch.randn(*s, generator=g) for s in ((3, 5), (4, 5), (4,), (3, 4)))
    y, bound = ref.linear(x, w, b, r, 3, 1)
    for i in range(3):
        for j in range(4):
            z = sum(float(x[i, t]) * float(w[j, t]) for t in range(5)) + float(b[j]) + float(r[i, j])
            assert abs(float(y[i, j]) - z / (1 + math.exp(-z))) < 1e-12 and float(bound[i, j]) > 0
    x, ga, be = torch.randn(2 * 3, 4, generator=g), torch.randn(4, generator=g), torch.randn(4, generator=g)
    y, _ = ref.group_norm(x, ga, be, None, 2, 3, 2, 1e-3, 1)
    for n in range(2):
        for grp in range(2):
            vals = [float(x[n * 3 + p, grp * 2 + c]) for p in range(3) for c in range(2)]
            mean = sum(vals) / 6
            var = sum((v - mean) ** 2 for v in vals) / 6
            for p in range(3):
                for c in range(2):
                    ch = grp * 2 + c
                    z = (float(x[n * 3 + p, ch]) - mean) / math.sqrt(var + 1e-3) * float(ga[ch]) + float(be[ch])
                    assert abs(float(y[n * 3 + p, ch]) - max(z, 0.0)) < 1e-12
    q, k, v = torch.randn(5, 2, 8, generator=g), torch.randn(4, 1, 8, generator=g), torch.randn(4, 1, 8, generator=g)
    y, _ = ref.attention(q, k, v, [4, 1], [3, 1], True, 0.5)
    assert bool((y[0] == 0).all())  # four queries, three keys: the first sees none
    for i, seen, at in ((1, 1, 0), (2, 2, 0), (3, 3, 0), (4, 1, 3)):
        for h in range(2):
            s = [0.5 * sum(float(q[i, h, c]) * float(k[at + j, 0, c]) for c in range(8)) for j in range(seen)]
            p = [math.exp(t - max(s)) for t in s]
            for c in range(8):
                assert abs(float(y[i, h, c]) - sum(pj * float(v[at + j, 0, c]) for j, pj in enumerate(p)) / sum(p)) < 1e-12


def test_the_bounds_allow_the_correctly_rounded_result():
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(40, 96, generator=g).bfloat16(), torch.randn(50, 96, generator=g).bfloat16()
    y, bound = ref.linear(x, w, None, None, 2, 0)
    assert bool(((y.bfloat16().double() - y).abs() <= bound).all())
    y, bound = ref.group_norm(x, None, None, None, 4, 10, 8, 1e-5, 0)
    assert bool(((y.bfloat16().double() - y).abs() <= bound).all())
    y, bound = ref.attention(x.view(40, 4, 24), w.view(50, 4, 24), w.view(50, 4, 24), [40], [50], True, 0.0)
    assert bool(((y.bfloat16().double() - y).abs() <= bound).all())
