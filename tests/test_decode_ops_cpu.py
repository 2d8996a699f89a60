"""Host logic of the decoding step's operators: what their descriptors and calls may say, both routes into the library,
and that the oracles in decode_ops_util agree with brute force."""
import ctypes
import math
from ctypes import c_void_p

import pytest
import torch

import decode_ops_util as ref
import paper_2406_09425_amd as S

INT_MAX = 2 ** 31 - 1
NORM = dict(m=4, c=64, dtype=S.SGPRS_BF16, out_dtype=S.SGPRS_I8, eps=1e-6)
QUANTIZE = dict(m=4, c=64, dtype=S.SGPRS_F32)
LINEAR = dict(m=4, n=8, k=16, dtype=S.SGPRS_F32)
CACHE = dict(n_seqs=3, kv_heads=2, head_dim=64, dtype=S.SGPRS_BF16, n_pages=9, page_size=16, table_width=4)
APPEND = dict(total=3, **CACHE)
ATTENTION = dict(heads=4, **CACHE)
P = 1 << 20  # a pointer that no call may follow


def call(kind, pool=None, **change):
    """The call with fitting pointers and no pool: INVALID_ARG "pool is NULL" where its descriptor is fine."""
    if kind == "rms_norm":
        S.sgprs_rms_norm(S.RmsNormDesc(**{**NORM, **change}), P, None, None, None, 2 * P, 3 * P, pool, 0)
    elif kind == "quantize":
        S.sgprs_quantize_i8(S.QuantizeDesc(**{**QUANTIZE, **change}), P, 2 * P, 3 * P, pool, 0)
    elif kind == "linear_i8":
        S.sgprs_linear_i8(S.LinearI8Desc(**{**LINEAR, **change}), P, None, P, None, None, None, 2 * P, None, 0, pool, 0)
    elif kind == "append":
        S.sgprs_paged_append(S.PagedAppendDesc(**{**APPEND, **change}), P, 2 * P, None, 3 * P, 4 * P, 5 * P, 6 * P, pool, 0)
    else:
        S.sgprs_paged_attention(S.PagedAttentionDesc(**{**ATTENTION, **change}), P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, None, 0, pool, 0)


FINE = [("rms_norm", {}), ("rms_norm", dict(m=0)), ("rms_norm", dict(out_dtype=1, eps=0.0, ldx=65, ldh=66)), ("rms_norm", dict(m=INT_MAX)), ("rms_norm", dict(c=1 << 20)),
        ("quantize", {}), ("quantize", dict(ldx=65, ldy=1 << 20)), ("linear_i8", {}), ("linear_i8", dict(k=131071, act=3, residual_first=1)),
        ("linear_i8", dict(ldx=17, ldw=16, ldr=9, ldy=8)), ("append", {}), ("append", dict(head_stride=16 * 64, token_stride=64)),
        ("append", dict(page_stride=16 * 64, token_stride=64, head_stride=9 * 16 * 64)), ("append", dict(n_pages=1, page_stride=64)), ("append", dict(page_size=1 << 20)),
        ("attention", {}), ("attention", dict(window=1, sinks=INT_MAX)), ("attention", dict(window=INT_MAX)), ("attention", dict(scale=-2e38, hq=128, ldq=512)),
        ("attention", dict(n_pages=INT_MAX, dtype=0)), ("attention", dict(heads=8192))]


@pytest.mark.parametrize("kind,change", FINE, ids=str)
def test_descriptors_that_are_fine(kind, change):
    with pytest.raises(S.SgprsError, match="pool is NULL"):
        call(kind, **change)


REFUSED = [
    ("rms_norm", dict(dtype=2, out_dtype=2), -5), ("rms_norm", dict(dtype=5), -5), ("rms_norm", dict(out_dtype=0), -5), ("rms_norm", dict(out_dtype=3), -5),
    ("rms_norm", dict(m=-1), -1), ("rms_norm", dict(c=0), -1), ("rms_norm", dict(eps=-1e-9), -1), ("rms_norm", dict(eps=math.nan), -1), ("rms_norm", dict(eps=math.inf), -1),
    ("rms_norm", dict(ldx=63), -1), ("rms_norm", dict(ldr=-64), -1), ("rms_norm", dict(ldh=1), -1), ("rms_norm", dict(ldy=63), -1), ("rms_norm", dict(ldy=(1 << 20) + 1), -5),
    ("rms_norm", dict(c=(1 << 20) + 1), -5),
    ("quantize", dict(dtype=2), -5), ("quantize", dict(m=-1), -1), ("quantize", dict(c=-5), -1), ("quantize", dict(ldx=63), -1), ("quantize", dict(ldy=1 << 21), -5),
    ("linear_i8", dict(dtype=2), -5), ("linear_i8", dict(act=4), -5), ("linear_i8", dict(m=-1), -1), ("linear_i8", dict(n=0), -1), ("linear_i8", dict(k=0), -1),
    ("linear_i8", dict(k=131072), -5), ("linear_i8", dict(residual_first=-1), -1), ("linear_i8", dict(ldx=15), -1), ("linear_i8", dict(ldw=15), -1),
    ("linear_i8", dict(ldr=7), -1), ("linear_i8", dict(ldy=1 << 21), -5)]
for kind in ("append", "attention"):
    REFUSED += [(kind, dict(dtype=2), -5), (kind, dict(n_seqs=0), -1), (kind, dict(n_seqs=(1 << 20) + 1), -5), (kind, dict(kv_heads=0), -1), (kind, dict(head_dim=12), -5),
                (kind, dict(head_dim=136), -5), (kind, dict(head_dim=0), -1), (kind, dict(n_pages=0), -1), (kind, dict(page_size=0), -1), (kind, dict(table_width=-1), -1),
                (kind, dict(table_width=1 << 20, page_size=1025), -5), (kind, dict(token_stride=60), -1), (kind, dict(token_stride=132), -5), (kind, dict(head_stride=1 << 50), -5),
                (kind, dict(token_stride=64), -1), (kind, dict(page_stride=16 * 128 - 8), -1), (kind, dict(head_stride=128), -1), (kind, dict(page_stride=-2048), -1)]
REFUSED += [("attention", dict(n_seqs=1 << 17, heads=4098, kv_heads=2049), -5), ("attention", dict(n_seqs=1 << 20, heads=32 * 257, kv_heads=1), -5)]
REFUSED += [("append", dict(total=-1), -1), ("append", dict(total=(1 << 30) + 1), -5), ("append", dict(ldk=56), -1), ("append", dict(hv=68), -5),
            ("append", dict(ldv=1 << 21), -5), ("attention", dict(heads=3), -1), ("attention", dict(heads=0), -1), ("attention", dict(heads=65536), -5),
            ("attention", dict(window=-1), -1), ("attention", dict(sinks=-1, window=4), -1), ("attention", dict(sinks=1), -1), ("attention", dict(scale=math.nan), -1),
            ("attention", dict(scale=math.inf), -1), ("attention", dict(scale=2.4e38), -5), ("attention", dict(ldq=252), -5), ("attention", dict(ho=56), -1), ("attention", dict(ldo=1 << 21), -5)]


@pytest.mark.parametrize("kind,change,status", REFUSED, ids=str)
def test_descriptors_that_are_refused(kind, change, status):
    with pytest.raises(S.SgprsError) as e:
        call(kind, **change)
    assert e.value.status == status and "pool" not in str(e.value), str(e.value)


def test_null_and_partition_arguments_are_refused():
    lib = S.lib()
    assert lib.sgprs_rms_norm(None, None, None, None, None, None, None, None, 0) == -1
    assert lib.sgprs_quantize_i8(None, None, None, None, None, 0) == -1
    assert lib.sgprs_linear_i8(None, None, None, None, None, None, None, None, None, 0, None, 0) == -1
    assert lib.sgprs_paged_append(None, None, None, None, None, None, None, None, None, 0) == -1
    assert lib.sgprs_paged_attention(None, None, None, None, None, None, None, None, 0, None, 0) == -1
    assert lib.sgprs_linear_i8_workspace(ctypes.byref(S.LinearI8Desc(**LINEAR)), 256, None) == -1
    assert lib.sgprs_paged_attention_workspace(None, 256, ctypes.byref(ctypes.c_size_t())) == -1
    for cus in (0, -3, 513):
        with pytest.raises(S.SgprsError):
            S.sgprs_linear_i8_workspace(S.LinearI8Desc(**LINEAR), cus)
        with pytest.raises(S.SgprsError):
            S.sgprs_paged_attention_workspace(S.PagedAttentionDesc(**ATTENTION), cus)


def test_workspaces_do_not_grow_with_the_lengths():
    """Two partial sums a workgroup, whatever the sequences: 32 rows of 128 channels at most."""
    for change in ({}, dict(table_width=1 << 20, n_pages=1 << 24, n_seqs=1 << 20), dict(heads=64, kv_heads=1, head_dim=128), dict(heads=8190, kv_heads=4095)):
        need = S.sgprs_paged_attention_workspace(S.PagedAttentionDesc(**{**ATTENTION, **change}), 512)
        assert 0 < need <= 1024 * (16 + 2 * 32 * (128 * 4 + 8)), change


@pytest.mark.parametrize("kind,args", [
    ("rms_norm", lambda p, i: (S.RmsNormDesc(**NORM), p, None, None, None, 2 * P, 3 * P, None, i)),
    ("quantize_i8", lambda p, i: (S.QuantizeDesc(**QUANTIZE), p, 2 * P, 3 * P, None, i)),
    ("linear_i8", lambda p, i: (S.LinearI8Desc(**LINEAR), p, None, P, None, None, None, 2 * P, None, 0, None, i)),
    ("paged_append", lambda p, i: (S.PagedAppendDesc(**APPEND), p, 2 * P, None, 3 * P, 4 * P, 5 * P, 6 * P, None, i)),
    ("paged_attention", lambda p, i: (S.PagedAttentionDesc(**ATTENTION), p, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, None, 0, None, i))])
def test_both_routes_reach_the_entry_point(kind, args, monkeypatch):
    entry, calls, native = getattr(S, "sgprs_" + kind), [], S.binding._calls()

    class Spy:
        def __getattr__(self, attr):
            def f(*a):
                rc = getattr(native, attr)(*a)
                calls.append(rc)
                return rc
            return f
    monkeypatch.setattr(S.binding, "_native", Spy())
    with pytest.raises(S.SgprsError, match="pool is NULL"):
        entry(*args(P, 0))
    assert calls == [-1]                               # the extension made the call
    with pytest.raises(S.SgprsError, match="pool is NULL"):
        entry(*args(c_void_p(P), 0))
    assert calls == [-1, None]                         # a c_void_p is for ctypes
    for bad in (args(P, 1.5), args(1.5, 0)):
        with pytest.raises(ctypes.ArgumentError):
            entry(*bad)
    for bad in (S.LinearDesc(), 16, None, ctypes.byref(S.ConvDesc())):
        with pytest.raises((ctypes.ArgumentError, TypeError)):
            entry(bad, *args(P, 0)[1:])


# ---- the oracles against brute force -------------------------------------------------------------
def test_rows_of_integers_by_hand():
    t = torch.tensor([[127.0, 0.5, 1.5, -2.5, 3.4999, -127.0], [0.0] * 6, [1.0, math.nan, 0, 0, 0, 0], [1.0, -math.inf, 0, 0, 0, 0], [2.0 ** -149, 0, 0, 0, 0, -(2.0 ** -149)]])
    q, scales = ref.quantize(t)
    assert q.tolist() == [[127, 0, 2, -2, 3, -127], [0] * 6, [0] * 6, [0] * 6, [127, 0, 0, 0, 0, -127]]
    assert scales[:2].tolist() == [1.0, 0.0] and bool(scales[2:4].isnan().all()) and float(scales[4]) == 2.0 ** -149 / 127


def test_norm_product_and_attention_by_hand():
    g = torch.Generator().manual_seed(1)
    x, r, ga = torch.randn(2, 5, generator=g).bfloat16(), torch.randn(2, 5, generator=g).bfloat16(), torch.randn(5, generator=g)
    h, y, _ = ref.rms_norm(x, r, ga, 1e-3, False)
    _, q, scales = ref.rms_norm(x, r, ga, 1e-3, True)
    for i in range(2):
        row = [float(torch.tensor(float(x[i, c]) + float(r[i, c])).bfloat16()) for c in range(5)]
        assert row == h[i].tolist()
        size = math.sqrt(sum(v * v for v in row) / 5 + 1e-3)
        z = [v * float(ga[c]) / size for c, v in enumerate(row)]
        most = max(abs(v) for v in z)
        for c in range(5):
            assert abs(float(y[i, c]) - z[c]) < 1e-12 and int(q[i, c]) == round(127 * z[c] / most)
        assert abs(float(scales[i]) - most / 127) < 1e-12
    a, w = torch.randint(-128, 128, (2, 7), generator=g, dtype=torch.int8), torch.randint(-128, 128, (3, 7), generator=g, dtype=torch.int8)
    sx, sw, b = torch.rand(2, generator=g), torch.rand(3, generator=g), torch.randn(3, generator=g)
    res = torch.randn(2, 3, generator=g)
    for first in (0, 1):
        y, _ = ref.linear_i8(a, sx, w, sw, b, res, 1, first, torch.float32)
        for i in range(2):
            for j in range(3):
                z = sum(int(a[i, c]) * int(w[j, c]) for c in range(7)) * float(sx[i]) * float(sw[j]) + float(b[j])
                want = max(0.0, z + float(res[i, j])) if first else max(0.0, z) + float(res[i, j])
                assert abs(float(y[i, j]) - want) < 1e-9
    q, k, v = torch.randn(2, 4, 8, generator=g), torch.randn(6, 3, 2, 8, generator=g), torch.randn(6, 3, 2, 8, generator=g)
    table = torch.tensor([[4, 1, 0, -1], [2, -1, -1, -1]], dtype=torch.int32)
    y, _ = ref.paged_attention(q, k, v, table, [8, 0], 4, 2, 0.5)
    assert bool((y[1] == 0).all())
    rows = [(4, 0), (4, 1), (1, 1), (1, 2), (0, 0), (0, 1)]  # positions 0, 1 and 4 to 7
    for head in range(4):
        s = [0.5 * sum(float(q[0, head, c]) * float(k[p, i, head // 2, c]) for c in range(8)) for p, i in rows]
        e = [math.exp(t - max(s)) for t in s]
        for c in range(8):
            assert abs(float(y[0, head, c]) - sum(w * float(v[p, i, head // 2, c]) for w, (p, i) in zip(e, rows)) / sum(e)) < 1e-12
    kc, vc = ref.paged_append(k[0, :, :, :], v[0, :, :, :], [0, 2, 3], table, [4, 1], torch.zeros_like(k), torch.zeros_like(v))
    assert torch.equal(kc[4, 2], k[0, 0]) and torch.equal(kc[1, 0], k[0, 1]) and torch.equal(vc[2, 0], v[0, 2]) and int((kc != 0).any(-1).sum()) == 6
