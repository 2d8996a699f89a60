"""GPU parity of the decoding step's operators with 64-bit definitions, at the sizes, strides, lengths, pages and values
where a kernel can go wrong."""
import math

import pytest
import torch

import block_ops_util
import decode_ops_util as ref
import paper_2406_09425_amd as S
from linear_i8_shapes import SHAPES
from test_gpu_block_ops import CUS, DT, Rows, gen, pools, ptr  # noqa: F401  (pools is a fixture)

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


class Bytes(Rows):
    """Rows of 8-bit integers."""

    def __init__(self, host, pad=0, lead=0):
        m, c = host.shape
        self.buf = torch.full((lead + m * (c + pad) + 64,), 77, dtype=torch.int8)
        self.view_of(self.buf, m, c, pad, lead).copy_(host)
        self.before = self.buf.clone()
        self.buf = self.buf.cuda()
        self.t = self.view_of(self.buf, m, c, pad, lead)
        self.args = (m, c, pad, lead)
        self.ld = c + pad


def bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def same(got, want, what):
    assert torch.equal(got.cpu(), want), f"{what}: {int((got.cpu() != want).sum())} of {want.numel()} integers differ"


# ---- norm and rows of integers -------------------------------------------------------------------
def run_norm(pools, name, x, res=None, gamma=None, eps=1e-6, i8=True, keep=True, pads=(0, 0, 0, 0), lead=0, cus=CUS, on=None, repeat=True):
    """on: "x" or "res", where the sum goes (y in the dtype, if there is no sum)."""
    dt, tdt = DT[name]
    m, c = x.shape
    X, R = Rows(x, pads[0], lead), Rows(res, pads[1], lead) if res is not None else None
    keep = keep and res is not None
    place = X if on == "x" else R if on == "res" else None
    H = (place or Rows(torch.full((m, c), NAN).to(tdt), pads[2], lead)) if keep else None
    Y = Bytes(torch.full((m, c), 99, dtype=torch.int8), pads[3], lead) if i8 else place if place and not keep else Rows(torch.full((m, c), NAN).to(tdt), pads[3], lead)
    G = gamma.cuda() if gamma is not None else None
    scales = torch.full((m + 1,), 55.0, device="cuda")
    d = S.RmsNormDesc(m=m, c=c, dtype=dt, out_dtype=S.SGPRS_I8 if i8 else dt, eps=eps, ldx=X.ld, ldr=R.ld if R else 0, ldh=H.ld if H else 0, ldy=Y.ld)
    pool = pools(cus)
    torch.cuda.synchronize()

    def call():
        S.sgprs_rms_norm(d, ptr(X.t), ptr(R.t) if R else None, ptr(G), ptr(H.t) if H else None, ptr(Y.t), ptr(scales) if i8 else None, pool, 0)
        pool.sync()
        return [t.cpu().clone() for t in (H.t if H else Y.t, Y.t, scales)]

    h, y, s = call()
    what = f"rms_norm {name} {m}x{c} i8 {i8} pads {pads} lead {lead} on {on} cus {cus}"
    want = ref.rms_norm(x, res, gamma, eps, i8)
    if keep:
        assert torch.equal(bits(h[~want[0].isnan()]), bits(want[0][~want[0].isnan()])) and torch.equal(h.isnan(), want[0].isnan()), what
    if i8:
        same(y, want[1], what)
        block_ops_util.assert_within(s[:m], want[2], 24 * ref.U * want[2].abs() + 2.0 ** -149, what)
        assert float(s[m]) == 55.0
    else:
        block_ops_util.assert_within(y, want[1], want[2], what)
    for t in (X, Y, R, H):
        assert t is None or t.outside_untouched(), what
    if repeat and place is None:
        for a, b in zip(call(), (h, y, s)):
            assert torch.equal(bits(a), bits(b)), f"{what}: a second call gives other bits"


def run_quantize(pools, name, x, pads=(0, 0), lead=0, cus=CUS):
    m, c = x.shape
    X, Y = Rows(x, pads[0], lead), Bytes(torch.full((m, c), 99, dtype=torch.int8), pads[1], lead)
    scales = torch.full((m + 1,), 55.0, device="cuda")
    d = S.QuantizeDesc(m=m, c=c, dtype=DT[name][0], ldx=X.ld, ldy=Y.ld)
    pool = pools(cus)
    torch.cuda.synchronize()
    S.sgprs_quantize_i8(d, ptr(X.t), ptr(Y.t), ptr(scales), pool, 0)
    pool.sync()
    q, want = ref.quantize(x)
    what = f"quantize {name} {m}x{c} pads {pads} lead {lead}"
    same(Y.t, q, what)
    block_ops_util.assert_within(scales[:m], want, 2 * ref.U * want.abs() + 2.0 ** -149, what)
    assert float(scales[m]) == 55.0 and X.outside_untouched() and Y.outside_untouched(), what


ROWS = [(1, 1), (3, 3), (2, 7), (5, 8), (4, 9), (7, 64), (9, 255), (130, 256), (33, 509), (6, 512), (3, 1023), (2000, 1024), (1100, 1030), (5, 2048), (1050, 2049), (1, 4096),
        (1030, 4096), (3, 4099), (2, 8192), (70, 8200), (1, 16384), (3, 16385), (2, 32768), (1, 65536), (2, 65537), (1, 131077)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ROWS, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("i8", [True, False], ids=["i8", "same"])
def test_norm_shapes(pools, name, shape, i8):
    m, c = shape
    i = ROWS.index(shape)
    g = gen(i)
    x, r = ((torch.randn(m, c, generator=g) * 2).to(DT[name][1]) for _ in range(2))
    pad, lead = [(0, 0), (8, 0), (3, 1)][i % 3]
    run_norm(pools, name, x, r if i % 4 else None, torch.rand(c, generator=g) + 0.5 if i % 5 else None, i8=i8, keep=i % 3 != 1, pads=(pad, pad + i % 2, 2 * pad, pad), lead=lead)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ROWS, ids=lambda s: "x".join(map(str, s)))
def test_quantize_shapes(pools, name, shape):
    m, c = shape
    i = ROWS.index(shape)
    pad, lead = [(0, 0), (16, 0), (3, 1)][i % 3]
    run_quantize(pools, name, torch.randn(m, c, generator=gen(i)).to(DT[name][1]), pads=(pad, pad), lead=lead)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("i8", [True, False], ids=["i8", "same"])
@pytest.mark.parametrize("on", ["x", "res"])
@pytest.mark.parametrize("c", [100, 5000, 70001])
def test_norm_results_on_top_of_inputs(pools, name, i8, on, c):
    """The sum on x or on the residual; without a sum, y."""
    g = gen(c)
    x, r = (torch.randn(3, c, generator=g).to(DT[name][1]) for _ in range(2))
    run_norm(pools, name, x, r, torch.rand(c, generator=g), i8=i8, on=on, pads=(8, 8, 8, 8))
    if not i8:
        run_norm(pools, name, x, r, torch.rand(c, generator=g), i8=False, keep=False, on=on, pads=(8, 8, 8, 8))
        if on == "x":
            run_norm(pools, name, x, None, None, i8=False, on="x")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("c", [24, 600, 3000, 66000])
def test_rows_of_every_size_of_value(pools, name, c):
    """From the smallest subnormal to the largest number, rows of zeros, rows of one value, values beside huge ones."""
    g = gen(c)
    t = torch.randn(14, c, generator=g)
    big = torch.finfo(DT[name][1]).max
    for row, size in enumerate((1e-44, 1e-40, 1e-30, 1e-20, 1e-12, 1.0, 1e12, 1e20, 1e30, 7e37)):
        t[row] = t[row].clamp(-4, 4) * size
    t[10] = 0
    t[11] = 3.0
    t[12, 0], t[13, -1] = big, -big
    x = t.to(DT[name][1])
    ga = torch.randn(c, generator=g)
    run_quantize(pools, name, x)
    for gamma in (None, ga):
        for i8 in (True, False):
            run_norm(pools, name, x, None, gamma, eps=1e-6, i8=i8)
    nonzero = x[x.double().abs().amax(1) > 0]
    run_norm(pools, name, nonzero, None, ga, eps=0.0, i8=False)
    run_norm(pools, name, nonzero, None, ga * 1e20, eps=0.0, i8=True)
    run_norm(pools, name, x, None, ga, eps=0.0, i8=True)      # a row of zeros: 0 / 0
    run_norm(pools, name, x, None, ga, eps=0.0, i8=False)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("c", [24, 600, 3000, 66000])
def test_rows_that_are_not_finite(pools, name, c):
    x = torch.randn(7, c, generator=gen(c)).to(DT[name][1])
    x[0, 0], x[1, c // 2], x[2, -1], x[3, 1], x[4, 0], x[4, 1] = NAN, INF, -INF, NAN, INF, -INF
    ga = torch.ones(c)
    run_quantize(pools, name, x)
    run_norm(pools, name, x, None, ga, i8=True)
    run_norm(pools, name, x, None, ga, i8=False)
    big = torch.full((2, c), torch.finfo(DT[name][1]).max).to(DT[name][1])
    run_norm(pools, name, big, big, ga, i8=True)  # the sum overflows
    ga[c // 3] = NAN
    run_norm(pools, name, x[5:], None, ga, i8=True)
    ga[c // 3] = INF
    run_norm(pools, name, x[5:], None, ga, i8=True)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("c", [16, 250, 2000, 9000])
def test_integers_next_to_and_on_the_border(pools, name, c):
    """max|t| = 127 of some unit, so halves of it are ties, to even; and for fp32 values one bit beside them."""
    g = gen(c)
    k = torch.randint(-254, 255, (40, c), generator=g)
    t = k.double() / 2
    t[:, 0] = 127
    if name == "bf16":  # 8 significant bits: halves up to 64
        t = torch.where(t.abs() < 64, t, t.round())
    else:
        step = torch.randint(-1, 2, t.shape, generator=g).double() * 2.0 ** -17  # a bit of 64 to 128
        step[:, 0] = 0
        t = t + torch.where(t.abs() < 120, step, 0.0)
    unit = 2.0 ** torch.randint(-30, 30, (40, 1), generator=g).double()
    x = (t * unit).to(DT[name][1])
    assert torch.equal(x.double(), t * unit)
    run_quantize(pools, name, x)
    run_norm(pools, name, x, None, None, i8=True)
    run_norm(pools, name, x, None, torch.full((c,), 3.0), i8=True)


@pytest.mark.parametrize("cus", [8, 40, 256])
@pytest.mark.parametrize("m", [1, 20, 300, 5000])
def test_norm_on_partitions(pools, cus, m):
    g = gen(m)
    run_norm(pools, "bf16", torch.randn(m, 700, generator=g).bfloat16(), torch.randn(m, 700, generator=g).bfloat16(), torch.rand(700, generator=g), cus=cus)


# ---- linear product of 8-bit integers ------------------------------------------------------------
def run_linear(pools, name, m, n, k, act=0, bias=True, res=False, first=0, pads=(0, 0, 0, 0), lead=0, cus=CUS, seed=0, x=None, w=None, scales=(True, True),
               inplace=False, sx=None):
    dt, tdt = DT[name]
    g = gen(seed)
    x = torch.randint(-128, 128, (m, k), generator=g, dtype=torch.int8) if x is None else x
    w = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int8) if w is None else w
    sx = (torch.rand(m, generator=g) + 0.1) / 100 if sx is None and scales[0] else sx
    sw = (torch.rand(n, generator=g) + 0.1) / (60 * math.sqrt(k)) if scales[1] else None
    bh = torch.randn(n, generator=g) if bias else None
    rh = torch.randn(m, n, generator=g).to(tdt) if res else None
    X, W = Bytes(x, pads[0], lead), Bytes(w, pads[1], lead)
    R = Rows(rh, pads[2], lead) if res else None
    Y = R if inplace else Rows(torch.full((m, n), NAN).to(tdt), pads[3], lead)
    B, SX, SW = (t.cuda() if t is not None else None for t in (bh, sx, sw))
    pool = pools(cus)
    d = S.LinearI8Desc(m=m, n=n, k=k, dtype=dt, act=act, residual_first=first, ldx=X.ld, ldw=W.ld, ldr=R.ld if res else 0, ldy=Y.ld)
    ws_bytes = S.sgprs_linear_i8_workspace(d, cus)
    ws = torch.full((max(ws_bytes, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_linear_i8(d, ptr(X.t), ptr(SX), ptr(W.t), ptr(SW), ptr(B), ptr(R.t) if res else None, ptr(Y.t), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    want, bound = ref.linear_i8(x, sx, w, sw, bh, rh, act, first, tdt)
    what = f"linear_i8 {name} {m}x{k}->{n} act {act} pads {pads} lead {lead} cus {cus}"
    block_ops_util.assert_within(Y.t, want, bound, what)
    for t in (X, W, Y) + ((R,) if res else ()):
        assert t.outside_untouched(), what
    return Y.t.cpu()


LINEAR = [(1, 1, 1), (1, 1000, 512), (2, 3, 7), (5, 16, 15), (8, 40, 17), (16, 33, 64), (17, 64, 40), (24, 512, 1024), (31, 100, 2048), (33, 65, 72), (48, 1000, 520),
          (64, 64, 64), (65, 130, 96), (100, 1000, 512), (128, 128, 128), (129, 257, 136), (200, 2049, 64), (255, 256, 1032), (256, 256, 256), (257, 300, 512),
          (500, 96, 4096), (784, 512, 512), (1025, 768, 200), (2048, 1040, 264), (3137, 64, 64), (3, 20, 131071), (300, 70, 5000), (4100, 520, 130)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LINEAR, ids=lambda s: "x".join(map(str, s)))
def test_linear_shapes(pools, name, shape):
    m, n, k = shape
    i = LINEAR.index(shape)
    run_linear(pools, name, m, n, k, act=i % 4, bias=i % 3 != 1, res=i % 2 == 1, first=(i // 2) % 2, seed=i)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(4090, 4080, 1024), (12500, 500, 512), (12500, 517, 509), (1000, 1001, 2050), (250, 4096, 2048), (256, 2040, 4096), (120, 4096, 4096), (24, 4096, 4096),
                                   (50, 4090, 4096), (40, 1000, 8192),
                                   (1000, 4096, 2048), (700, 2040, 1536), (1000, 1024, 648), (500, 4096, 1024),
                                   (700, 701, 700), (1500, 300, 300), (2100, 517, 131)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("res", [False, True], ids=["", "residual"])
def test_linear_tiles_of_every_size(pools, name, shape, res):
    m, n, k = shape
    run_linear(pools, name, m, n, k, act=int(res), bias=not res, res=res, seed=m)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("kernel,shape", SHAPES, ids=lambda s: s if isinstance(s, str) else "x".join(map(str, s)))
def test_linear_by_every_kernel(pools, name, kernel, shape):
    m, n, k = shape
    for res in (False, True):
        run_linear(pools, name, m, n, k, act=3 if res else 0, bias=not res, res=res, first=int(res), seed=n)


@pytest.mark.parametrize("shape", [(1, 100, 512), (20, 64, 300), (40, 200, 130), (300, 130, 96), (1000, 1500, 200), (3000, 2100, 256)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("pads,lead", [((16, 0, 8, 8), 0), ((16, 32, 0, 0), 16), ((3, 0, 1, 5), 0), ((0, 1, 3, 0), 1), ((8, 4, 2, 6), 4), ((1, 1, 1, 1), 7)], ids=str)
def test_linear_strides_and_alignment(pools, shape, pads, lead):
    m, n, k = shape
    for name in ("f32", "bf16"):
        run_linear(pools, name, m, n, k, act=m % 4, res=True, first=n // 10 % 2, pads=pads, lead=lead, seed=k)


@pytest.mark.parametrize("shape", [(1, 64, 700), (30, 33, 130), (70, 64, 1000), (1000, 300, 64), (5000, 1300, 300)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("cus", [8, 72, 256])
def test_linear_on_partitions_gives_the_same_bits(pools, shape, cus):
    m, n, k = shape
    a, b = (run_linear(pools, "f32", m, n, k, act=0, res=True, cus=c, seed=m) for c in (cus, CUS))
    assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("m,n,k", [(2, 5, 131071), (40, 70, 131071), (300, 300, 4099)])
@pytest.mark.parametrize("value", [-128, 127])
def test_linear_of_the_largest_sums(pools, m, n, k, value):
    x, w = torch.full((m, k), value, dtype=torch.int8), torch.full((n, k), -128, dtype=torch.int8)
    y = run_linear(pools, "f32", m, n, k, bias=False, x=x, w=w, scales=(False, False))
    assert bool((y.double() == float(torch.tensor(float(value * -128 * k)))).all())


def test_linear_of_rows_without_a_scale(pools):
    """NaN scales give NaN rows, zeros zeros (and the bias), and no other row is touched."""
    for m in (5, 40, 700):
        sx = torch.rand(m, generator=gen(m))
        sx[1], sx[2], sx[4] = NAN, 0.0, INF
        run_linear(pools, "bf16", m, 300, 128, sx=sx, seed=m)
        run_linear(pools, "f32", m, 50, 100, sx=sx, bias=False, seed=m)


@pytest.mark.parametrize("m", [3, 50, 600])
def test_linear_on_top_of_the_residual(pools, m):
    for name in ("f32", "bf16"):
        run_linear(pools, name, m, 130, 260, act=1, res=True, first=1, inplace=True, pads=(0, 0, 6, 6), seed=m)


def test_rows_behind_four_gigabytes(pools):
    """The last rows of a norm and a product whose operands pass 2^32 bytes (repeated rows: what is before them is the same)."""
    pool, m, c = pools(), (1 << 26) + 67, 72
    g = gen(6)
    few = torch.randn(67, c, generator=g).bfloat16()
    x = few.cuda().repeat((m + 66) // 67, 1)[:m].contiguous()
    q8, sx = torch.zeros(m, c, dtype=torch.int8, device="cuda"), torch.zeros(m, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_rms_norm(S.RmsNormDesc(m=m, c=c, dtype=1, out_dtype=2, eps=1e-6), ptr(x), None, None, None, ptr(q8), ptr(sx), pool, 0)
    pool.sync()
    want = ref.rms_norm(few, None, None, 1e-6, True)
    rows = torch.arange(m - 200, m)
    same(q8[m - 200:], want[1][rows % 67], "last rows")
    assert torch.equal(bits(q8[:67 * 1000000].view(1000000, 67, c)), bits(q8[:67].expand(1000000, 67, c).contiguous()))
    S.sgprs_quantize_i8(S.QuantizeDesc(m=m, c=c, dtype=1), ptr(x), ptr(q8), ptr(sx), pool, 0)
    pool.sync()
    want, ws = ref.quantize(few)
    same(q8[m - 200:], want[rows % 67], "last rows")
    w = torch.randint(-127, 128, (40, c), generator=g, dtype=torch.int8)
    gw, y = w.cuda(), torch.zeros(m, 40, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_linear_i8(S.LinearI8Desc(m=m, n=40, k=c, dtype=1), ptr(q8), ptr(sx), ptr(gw), None, None, None, ptr(y), None, 0, pool, 0)
    pool.sync()
    got, bound = ref.linear_i8(want, sx[:67].cpu(), w, None, None, None, 0, 0, torch.bfloat16)
    block_ops_util.assert_within(y[m - 200:], got[rows % 67], bound[rows % 67], "last rows")
    assert torch.equal(bits(y[:67 * 1000000].view(1000000, 67, 40)), bits(y[:67].expand(1000000, 67, 40).contiguous()))


@pytest.mark.parametrize("n,k", [(1, 8), (8, 16)])
def test_linear_of_more_tiles_than_a_launch_holds(pools, n, k):
    """2^30 rows and a few: 2^24 tiles of 64 of them, 256 threads each, are 2^32 threads (repeated rows: what is before the
    last ones is the same)."""
    m, few, g = (1 << 30) + 5, 61, gen(k)
    x, w = (torch.randint(-127, 128, (rows, k), generator=g, dtype=torch.int8) for rows in (few, n))
    sx, res = torch.rand(few, generator=g), torch.randn(few, n, generator=g).bfloat16()

    def repeated(t):
        whole, full = torch.empty((m,) + t.shape[1:], dtype=t.dtype, device="cuda"), m // few
        whole[:full * few].view((full,) + t.shape).copy_(t.cuda().expand((full,) + t.shape))
        whole[full * few:] = t[:m - full * few].cuda()
        return whole

    X, SX, R, W, Y = repeated(x), repeated(sx), repeated(res), w.cuda(), torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    pool = pools()
    torch.cuda.synchronize()
    S.sgprs_linear_i8(S.LinearI8Desc(m=m, n=n, k=k, dtype=1), ptr(X), ptr(SX), ptr(W), None, None, ptr(R), ptr(Y), None, 0, pool, 0)
    pool.sync()
    want, bound = ref.linear_i8(x, sx, w, None, None, res, 0, 0, torch.bfloat16)
    rows = torch.arange(m - 400, m)  # on both sides of 2^30 - 64
    block_ops_util.assert_within(Y[m - 400:], want[rows % few], bound[rows % few], "last rows")
    block_ops_util.assert_within(Y[:few], want, bound, "first rows")
    blocks = Y[:m // few * few].view(-1, few, n).view(torch.int16)
    for part in blocks.split(1 << 22):
        assert bool((part == blocks[0]).all())
    del X, SX, R, Y, blocks, part
    torch.cuda.empty_cache()


# ---- paged cache ---------------------------------------------------------------------------------
class Cache:
    """Caches of n_pages pages; layout: the order of the page's positions and heads."""

    def __init__(self, name, kv, page, hk, dim, layout="token", spare=3, seed=0, pad=0, fill=None, extra=0):
        g = gen(seed)
        used = [-(-v // page) for v in kv]
        self.n_pages, self.width, self.page = sum(used) + spare, max(max(used, default=0), 1) + extra, page
        order = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((len(kv), self.width), -1, dtype=torch.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at:at + u]
            at += u
        shape = dict(token=(self.n_pages, page, hk, dim + pad), head=(self.n_pages, hk, page, dim + pad), outer=(hk, self.n_pages, page, dim + pad))[layout]
        self.to = dict(token=lambda t: t, head=lambda t: t.transpose(1, 2), outer=lambda t: t.permute(1, 2, 0, 3))[layout]
        self.k, self.v = ((torch.randn(shape, generator=g) if fill is None else torch.full(shape, fill)).to(DT[name][1]) for _ in range(2))
        view = self.to(self.k)
        self.strides = dict(page_stride=view.stride(0), token_stride=view.stride(1), head_stride=view.stride(2))
        self.dims = dict(kv_heads=hk, head_dim=dim, dtype=DT[name][0], n_pages=self.n_pages, page_size=page, table_width=self.width, n_seqs=len(kv), **self.strides)
        self.dim = dim
        self.lens = torch.tensor(kv, dtype=torch.int32)

    def host(self):
        return tuple(self.to(t)[..., :self.dim].contiguous() for t in (self.k, self.v))

    def to_gpu(self):
        self.gk, self.gv, self.gtable, self.glens = self.k.cuda(), self.v.cuda(), self.table.cuda(), self.lens.cuda()
        return self


def poison(c, kv, window=0, sinks=0, value=NAN):
    """Every place that no sequence sees."""
    seen = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
    for s, n in enumerate(kv):
        at = torch.tensor(ref.visible(n, window, sinks), dtype=torch.long)
        seen[c.table[s].long()[at // c.page], at % c.page] = True
    for t in (c.k, c.v):
        c.to(t)[~seen] = value


def run_attention(pools, name, kv, heads, hk, dim, page=16, window=0, sinks=0, scale=0.0, layout="token", q_pad=0, pad=0, seed=0, cus=CUS, unseen=NAN, lens=None,
                  cache=None, q=None, extra=0):
    dt, tdt = DT[name]
    c = cache or Cache(name, kv, page, hk, dim, layout, seed=seed, pad=pad, extra=extra)
    if unseen is not None:
        poison(c, kv, window, sinks, unseen)
    if lens is not None:
        c.lens = torch.tensor(lens, dtype=torch.int32)
    c.to_gpu()
    n = len(kv)
    qh = (torch.randn(n, heads * dim, generator=gen(seed + 1)) * 1.5).to(tdt) if q is None else q
    Q, O = Rows(qh, q_pad), Rows(torch.full((n, heads * dim), NAN).to(tdt), q_pad)
    d = S.PagedAttentionDesc(heads=heads, window=window, sinks=sinks, scale=scale, ldq=Q.ld, ldo=O.ld, **c.dims)
    need = S.sgprs_paged_attention_workspace(d, cus)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    pool = pools(cus)
    torch.cuda.synchronize()

    def call():
        S.sgprs_paged_attention(d, ptr(Q.t), ptr(c.gk), ptr(c.gv), ptr(c.gtable), ptr(c.glens), ptr(O.t), ptr(ws), need, pool, 0)
        pool.sync()
        return O.t.cpu().clone()

    got = call()
    what = f"paged_attention {name} {str(kv)[:60]} heads {heads}/{hk} dim {dim} page {page} window {window}+{sinks} {layout} cus {cus}"
    k, v = c.host()
    want, bound = ref.paged_attention(qh.view(n, heads, dim), k, v, c.table, kv, window, sinks, scale)
    block_ops_util.assert_within(got.view(n, heads, dim), want, bound, what)
    assert Q.outside_untouched() and O.outside_untouched(), what
    assert bool((ws[need:] == 255).all()), f"{what}: behind the workspace"
    assert torch.equal(bits(call()), bits(got)), f"{what}: a second call gives other bits"
    return got


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("kv", [[1], [0], [31], [32], [33], [127], [128], [129], [1000], [0, 5, 0, 0, 300, 0], [1, 2, 3, 4, 5, 6, 7], [5000], [700, 1, 128, 0, 2500]], ids=str)
def test_attention_lengths(pools, name, kv):
    run_attention(pools, name, kv, 4, 2, 64, seed=sum(kv))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("heads,hk", [(1, 1), (6, 2), (8, 8)])
def test_attention_heads(pools, name, dim, heads, hk):
    run_attention(pools, name, [333, 64, 1], heads, hk, dim, seed=dim)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heads,hk", [(31, 1), (32, 1), (33, 1), (96, 2), (71, 1)])
def test_attention_of_many_heads_of_a_key_head(pools, name, heads, hk):
    run_attention(pools, name, [400, 9, 0, 170], heads, hk, 64, seed=heads)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("page", [1, 2, 3, 5, 7, 16, 31, 32, 33, 48, 64, 100, 128, 256, 1000])
def test_attention_pages(pools, name, page):
    run_attention(pools, name, [513, 100, 1, 0, 47], 4, 2, 64, page=page, seed=page, extra=page % 3)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["token", "head", "outer"])
@pytest.mark.parametrize("pad,q_pad", [(0, 0), (8, 8), (16, 0)])
def test_attention_layouts(pools, name, layout, pad, q_pad):
    run_attention(pools, name, [300, 77, 129], 8, 4, 72, page=12, layout=layout, pad=pad, q_pad=q_pad, seed=pad)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (32, 4), (100, 33), (128, 0), (250, 7), (2000, 4), (1 << 30, 3), (300, 1 << 30)])
def test_attention_windows(pools, name, window, sinks):
    """Around a length equal to the window, and sinks that reach into it."""
    run_attention(pools, name, [0, 1, 2, 31, 104, 127, 128, 129, 132, 250, 251, 257, 700, 2001, 2005, 3000], 4, 2, 64, page=24, window=window, sinks=sinks, seed=window % 97)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("unseen", [NAN, INF, -INF, 3e38])
def test_attention_does_not_read_what_is_not_seen(pools, name, unseen):
    run_attention(pools, name, [300, 65, 0, 2], 4, 1, 40, page=32, window=90, sinks=3, unseen=unseen)
    run_attention(pools, name, [300, 65, 0, 2], 4, 1, 128, page=32, unseen=unseen)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_attention_values_that_are_not_finite_where_they_are_seen(pools, name):
    """Infinities and NaNs of v at seen positions reach their channel, and no other sequence or head."""
    kv = [200, 33, 500]
    c = Cache(name, kv, 16, 2, 64, seed=5)
    c.to(c.v)[c.table[0, 3], 2, 1, 7] = NAN
    c.to(c.v)[c.table[1, 2], 0, 0, 9] = INF       # the only key of its tile
    c.to(c.v)[c.table[2, 20], 5, 0, 63] = -INF
    run_attention(pools, name, kv, 4, 2, 64, cache=c, unseen=None, seed=5)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_attention_of_a_channel_of_infinities(pools, name):
    """Whatever parts a weight has, each is above zero: infinities of one sign stay what they are."""
    kv = [1, 31, 700, 64]
    c = Cache(name, kv, 16, 2, 64, seed=9)
    c.to(c.v)[..., 0, 5], c.to(c.v)[..., 1, 60] = INF, -INF
    run_attention(pools, name, kv, 6, 2, 64, cache=c, unseen=None, seed=9)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heads,dim", [(4, 64), (24, 128)])
def test_attention_queries_and_keys_that_are_not_finite(pools, name, heads, dim):
    """A NaN of a query stays in its head, one of a key in the heads that read it."""
    kv, group = [200, 33, 700], heads // 2
    q = (torch.randn(3, heads * dim, generator=gen(6)) * 1.5).to(DT[name][1])
    clean = run_attention(pools, name, kv, heads, 2, dim, q=q, unseen=None, seed=5).view(3, heads, dim)
    for at, value in ((0, NAN), (2, NAN), (2, INF)):
        bad = q.clone()
        bad.view(3, heads, dim)[at, 1, 3] = value
        got = run_attention(pools, name, kv, heads, 2, dim, q=bad, unseen=None, seed=5).view(3, heads, dim)
        assert bool(got[at, 1].isnan().all())
        got[at, 1] = clean[at, 1]
        assert torch.equal(bits(got), bits(clean)), (at, value)
    c = Cache(name, kv, 16, 2, dim, seed=5)
    c.to(c.k)[c.table[2, 20], 5, 1, 2] = NAN
    got = run_attention(pools, name, kv, heads, 2, dim, q=q, cache=c, unseen=None, seed=5).view(3, heads, dim)
    assert bool(got[2, group:].isnan().all())
    got[2, group:] = clean[2, group:]
    assert torch.equal(bits(got), bits(clean))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [2, 6, 9])
@pytest.mark.parametrize("first,last", [(0, 128), (0, 300), (128, 256), (40, 400), (0, 399)])
def test_attention_scores_of_minus_infinity(pools, name, heads, first, last):
    """Keys whose scores are -inf have no weight, as if they were not there, in tiles of nothing else too."""
    kv, dim = [400, 100], 64
    q = (torch.randn(2, heads * dim, generator=gen(6)) * 1.5).to(DT[name][1])
    q.view(2, heads, dim)[:, :, 9] = 1.0
    c = Cache(name, kv, 16, 1, dim, seed=7)
    pos = torch.arange(first, last)
    c.to(c.k)[c.table[0].long()[pos // 16], pos % 16, 0, 9] = -INF
    got = run_attention(pools, name, kv, heads, 1, dim, q=q, cache=c, unseen=None, seed=7).view(2, heads, dim)
    pos = torch.tensor([p for p in range(400) if not first <= p < last])
    k, v = (t[c.table[0].long()[pos // 16], pos % 16] for t in c.host())
    want, bound = block_ops_util.attention(q[:1].view(1, heads, dim), k, v, [1], [len(pos)], False, 0.0)
    block_ops_util.assert_within(got[:1], want, bound, f"{name} without {first} to {last}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.3, 1.0, 30.0, 1e-30])
def test_attention_scales(pools, name, scale):
    run_attention(pools, name, [300, 40], 2, 2, 32, scale=scale)


@pytest.mark.parametrize("heads,hk,dim", [(4, 2, 64), (8, 2, 128), (33, 1, 32), (2, 1, 72)])
def test_attention_results_are_rounded_once(pools, heads, hk, dim):
    """The weights' own error counts for less than 2^-14 in the sum of |p v|: in bf16 they are two parts, of which the second
    (below 2^-7 of the weight) is off by half a step, 2^-8 of it.  The rest is the bound of fp32 and the result's rounding."""
    kv = [3000, 1, 0, 513, 31, 1024]
    c = Cache("bf16", kv, 16, hk, dim, seed=dim)
    q = (torch.randn(len(kv), heads * dim, generator=gen(dim)) * 0.5).bfloat16()
    got = run_attention(pools, "bf16", kv, heads, hk, dim, cache=c, q=q).view(len(kv), heads, dim)
    k, v = (torch.where(t.isnan(), 0.0, t.float()) for t in c.host())  # (what is not seen holds NaNs)
    want, bound = ref.paged_attention(q.float().view(len(kv), heads, dim), k, v, c.table, kv, 0, 0, 0.0)
    spread, _ = ref.paged_attention(q.float().view(len(kv), heads, dim), k, v.abs(), c.table, kv, 0, 0, 0.0)
    block_ops_util.assert_within(got, want, bound + 2.0 ** -14 * spread + 1.01 * 2.0 ** -8 * want.abs(), f"{heads}/{hk} heads of {dim}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("cus", [8, 32, 104, 256])
def test_attention_on_partitions(pools, name, cus):
    run_attention(pools, name, [3000, 1, 0, 700, 128, 129, 64, 2111], 6, 2, 96, page=20, cus=cus, seed=cus)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [255, 256, 257, 600, 3000])
def test_attention_of_many_sequences(pools, name, n):
    g = gen(n)
    kv = torch.randint(0, 40, (n,), generator=g).tolist()
    kv[n // 3], kv[-1], kv[0] = 1500, 300, 0
    run_attention(pools, name, kv, 2, 1, 32, page=8, seed=n)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [300, 2000])
def test_attention_of_tables_for_long_sequences(pools, name, n):
    """Room for 2^30 positions a sequence: the costs of all of them fit 31 bits in units of 8 (n 300) or 32 (2000) tiles only.
    Sequences of a fraction of a unit, whole ones and one that several workgroups share read the same page."""
    dim, heads, tdt = 8, 2, DT[name][1]
    kv = torch.randint(0, 40, (n,), generator=gen(n)).tolist()
    for s, length in ((0, 0), (7, 255), (8, 256), (9, 257), (10, 1024), (11, 1025), (n // 2, 60001), (n - 2, 5000), (n - 1, 300)):
        kv[s] = length
    k, v = (torch.randn(1, max(kv), 1, dim, generator=gen(i)).to(tdt) for i in (1, 2))
    q = (torch.randn(n, heads * dim, generator=gen(3)) * 1.5).to(tdt)
    d = S.PagedAttentionDesc(n_seqs=n, heads=heads, kv_heads=1, head_dim=dim, dtype=DT[name][0], n_pages=1, page_size=1 << 30, table_width=1)
    need = S.sgprs_paged_attention_workspace(d, CUS)
    gk, gv, gq, lens, table = k.cuda(), v.cuda(), q.cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    o, ws = torch.full_like(gq, NAN), torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_paged_attention(d, ptr(gq), ptr(gk), ptr(gv), ptr(table), ptr(lens), ptr(o), ptr(ws), need, pools(), 0)
    pools().sync()
    want, bound = ref.paged_attention(q.view(n, heads, dim), k, v, table.cpu(), kv, 0, 0, 0.0)
    block_ops_util.assert_within(o.view(n, heads, dim), want, bound, f"{name} {n}")
    assert bool((ws[need:] == 255).all())


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heads,hk,dim", [(2, 1, 32), (3, 1, 128), (5, 1, 64), (8, 1, 24), (14, 2, 128), (16, 2, 96), (9, 1, 32), (16, 1, 128)])
def test_attention_of_few_heads_of_a_key_head(pools, name, heads, hk, dim):
    run_attention(pools, name, [333, 64, 1, 0, 130], heads, hk, dim, seed=heads + dim)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n,hk,dim,most", [(127, 1, 64, 512), (128, 1, 64, 512), (128, 1, 64, 513), (64, 2, 128, 512), (128, 2, 128, 512), (129, 2, 128, 512), (257, 2, 32, 300), (256, 2, 32, 300)])
def test_attention_of_items_that_have_a_workgroup_each(pools, name, n, hk, dim, most):
    """On both sides of where a sequence's keys are no longer split, with equal and different lengths."""
    kv = torch.randint(0, most + 1, (n,), generator=gen(n + most)).tolist()
    kv[0], kv[n // 2] = most, 0
    run_attention(pools, name, kv, 2 * hk, hk, dim, seed=n)
    run_attention(pools, name, [most] * n, 2 * hk, hk, dim, seed=n)


@pytest.mark.parametrize("strides", [dict(page_stride=(1 << 27) + 8, token_stride=256, head_stride=128), dict(page_stride=16 * 128, token_stride=128, head_stride=(1 << 32) + 16),
                                     dict(page_stride=16 << 20, token_stride=1 << 20, head_stride=128)], ids=["page", "head", "token"])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_append_and_attention_of_places_far_apart(pools, name, strides):
    """Offsets that pass 32 bits."""
    dt, tdt = DT[name]
    c = Cache(name, [300, 0, 17, 130], 16, 2, 128, seed=4)
    last = (c.n_pages - 1) * strides["page_stride"] + 15 * strides["token_stride"] + strides["head_stride"] + 128
    bufs = [torch.empty(last, dtype=tdt, device="cuda") for _ in range(2)]
    view = [b.as_strided((c.n_pages, 16, 2, 128), (strides["page_stride"], strides["token_stride"], strides["head_stride"], 1)) for b in bufs]
    c.to_gpu()
    for at, t in zip(view, (c.gk, c.gv)):
        at.copy_(t)
    dims = {**c.dims, **strides}
    new = [torch.randn(4, 256, generator=gen(i)).to(tdt) for i in (1, 2)]
    q = torch.randn(4, 512, generator=gen(3)).to(tdt)
    gnew, gq, o = [t.cuda() for t in new], q.cuda(), torch.empty(4, 512, dtype=tdt, device="cuda")
    da, dt_ = S.PagedAppendDesc(total=4, **dims), S.PagedAttentionDesc(heads=4, **dims)
    need = S.sgprs_paged_attention_workspace(dt_, CUS)
    ws, pool = torch.empty(need, dtype=torch.uint8, device="cuda"), pools()
    torch.cuda.synchronize()
    S.sgprs_paged_append(da, ptr(gnew[0]), ptr(gnew[1]), None, ptr(c.gtable), ptr(c.glens), ptr(bufs[0]), ptr(bufs[1]), pool, 0)
    S.sgprs_paged_attention(dt_, ptr(gq), ptr(bufs[0]), ptr(bufs[1]), ptr(c.gtable), ptr(c.glens), ptr(o), ptr(ws), need, pool, 0)
    pool.sync()
    k, v = ref.paged_append(*(t.view(4, 2, 128) for t in new), None, c.table, c.lens.tolist(), *c.host())
    for at, want in zip(view, (k, v)):
        assert torch.equal(bits(at.cpu()), bits(want))
    want, bound = ref.paged_attention(q.view(4, 4, 128), k, v, c.table, c.lens.tolist(), 0, 0, 0.0)
    block_ops_util.assert_within(o.view(4, 4, 128), want, bound, f"{name} {strides}")


def test_attention_of_a_long_cache(pools):
    run_attention(pools, "bf16", [70001, 3, 20000], 8, 2, 128, page=64, seed=1, unseen=None)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_attention_lengths_and_tables_outside_their_range(pools, name):
    """Lengths count as the nearest possible ones; entries of no page read some page: finite values, nothing else asked."""
    kv = [64, 0, 48]
    run_attention(pools, name, kv, 2, 1, 32, page=16, lens=[1 << 30, -5, 48], extra=0, unseen=0.5)
    c = Cache(name, kv, 16, 1, 32, seed=3)
    good = c.table.clone()
    c.table[0, 1], c.table[0, 2], c.table[2, 0] = -7, 2 ** 31 - 1, c.n_pages
    c.to_gpu()
    q, o = (torch.randn(3, 64, device="cuda").to(DT[name][1]) for _ in range(2))
    d = S.PagedAttentionDesc(heads=2, **c.dims)
    need = S.sgprs_paged_attention_workspace(d, CUS)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_paged_attention(d, ptr(q), ptr(c.gk), ptr(c.gv), ptr(c.gtable), ptr(c.glens), ptr(o), ptr(ws), need, pools(), 0)
    pools().sync()
    assert bool(torch.isfinite(o).all()) and bool((o[1] == 0).all()) and good is not None


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_attention_of_other_sequences_beside_entries_of_no_page(pools, name):
    """Sequences whose entries are fine give the bits that they give beside good ones, with and without a split."""
    kv = [64, 0, 48, 700, 33, 5000]
    c = Cache(name, kv, 16, 2, 64, seed=3).to_gpu()
    q, o = (torch.randn(len(kv), 256, generator=gen(i)).to(DT[name][1]).cuda() for i in (1, 2))
    d = S.PagedAttentionDesc(heads=4, **c.dims)
    need = S.sgprs_paged_attention_workspace(d, CUS)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")

    def call():
        torch.cuda.synchronize()
        S.sgprs_paged_attention(d, ptr(q), ptr(c.gk), ptr(c.gv), ptr(c.gtable), ptr(c.glens), ptr(o), ptr(ws), need, pools(), 0)
        pools().sync()
        return o.cpu()

    good = call()
    c.gtable[0, 1], c.gtable[0, 2], c.gtable[2, 0], c.gtable[3, 40] = -7, 2 ** 31 - 1, c.n_pages, -2 ** 31
    got = call()
    for s in (1, 4, 5):
        assert torch.equal(bits(got[s]), bits(good[s])), s
    assert bool(torch.isfinite(got).all())


# ---- new keys and values -------------------------------------------------------------------------
def run_append(pools, name, kv, new, hk, dim, page=16, layout="token", pad=0, cache_pad=0, seed=0, cus=CUS, table=None, lens=None):
    c = Cache(name, kv, page, hk, dim, layout, seed=seed, pad=cache_pad, extra=1)
    if table:
        for (s, i), entry in table.items():
            c.table[s, i] = entry(c)
    if lens is not None:
        c.lens = torch.tensor(lens, dtype=torch.int32)
    c.to_gpu()
    off = None if new is None else torch.tensor([0] + new).cumsum(0).to(torch.int32)
    total = len(kv) if new is None else sum(new)
    K, V = (Rows(torch.randn(total, hk * dim, generator=gen(seed + i)).to(DT[name][1]), pad) for i in (1, 2))
    d = S.PagedAppendDesc(total=total, ldk=K.ld, ldv=V.ld, **c.dims)
    goff = off.cuda() if off is not None else None
    torch.cuda.synchronize()
    S.sgprs_paged_append(d, ptr(K.t), ptr(V.t), ptr(goff), ptr(c.gtable), ptr(c.glens), ptr(c.gk), ptr(c.gv), pools(cus), 0)
    pools(cus).sync()
    k, v = c.host()
    heads = [t.t.cpu().reshape(total, hk, dim) for t in (K, V)]
    want = ref.paged_append(*heads, off.tolist() if off is not None else None, c.table, c.lens.tolist(), k, v)
    for was, now, w in zip((c.k, c.v), (c.gk, c.gv), want):
        c.to(was)[..., :dim] = w
        assert torch.equal(bits(now.cpu()), bits(was)), f"append {name} {kv} {new} page {page} {layout}"


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("hk,dim", [(1, 8), (1, 64), (3, 24), (2, 72), (8, 128), (5, 128), (40, 128)])
@pytest.mark.parametrize("layout", ["token", "head", "outer"])
def test_append(pools, name, hk, dim, layout):
    run_append(pools, name, [17, 1, 0, 64, 33], None, hk, dim, layout=layout, seed=dim)
    run_append(pools, name, [17, 1, 0, 64, 33, 5], [17, 1, 0, 3, 0, 5], hk, dim, page=7, layout=layout, pad=16, cache_pad=8, seed=hk)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [63, 64, 65, 300, 5000])
def test_append_to_many_sequences(pools, name, n):
    kv = torch.randint(0, 30, (n,), generator=gen(n)).tolist()
    new = [int(v * f) for v, f in zip(kv, torch.rand(n, generator=gen(n + 1)).tolist())]
    new[n // 2] = kv[n // 2] = 777
    run_append(pools, name, kv, new, 1, 16, page=8, seed=n)
    run_append(pools, name, kv, None, 2, 32, page=8, seed=n)


def test_append_to_no_place(pools):
    """More tokens than positions, lengths of zero and below, entries of no page: those tokens go nowhere, the others to theirs."""
    run_append(pools, "bf16", [20, 3, 40, 8], [5, 6, 40, 8], 2, 32, page=8, lens=[0, 3, 40, -9])
    run_append(pools, "f32", [20, 3, 40, 8], [20, 3, 40, 8], 2, 32, page=8, table={(0, 1): lambda c: -1, (2, 0): lambda c: c.n_pages, (2, 3): lambda c: 2 ** 31 - 1})
    run_append(pools, "f32", [20, 3], None, 2, 32, page=8, lens=[1 << 30, 0], table={(0, 3): lambda c: 0})


def test_append_with_offsets_that_are_wrong(pools):
    """Offsets that fall, are negative or pass the number of tokens: what is written comes from k and v, and nothing else changes."""
    c = Cache("f32", [40, 40, 40, 40], 8, 2, 32, seed=2).to_gpu()
    before = c.gk.clone(), c.gv.clone()
    k, v = (torch.full((20, 64), t, device="cuda") for t in (5.0, 6.0))
    for offsets in ([0, 12, 3, 9, 20], [-7, 2, 5, 9, 20], [0, 5, 9, 30, 2 ** 31 - 1], [7, 7, 7, 7, 7], [-2 ** 31, 2 ** 31 - 1, 0, -5, 3], [2 ** 31 - 1] * 5):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        S.sgprs_paged_append(S.PagedAppendDesc(total=20, **c.dims), ptr(k), ptr(v), ptr(off), ptr(c.gtable), ptr(c.glens), ptr(c.gk), ptr(c.gv), pools(), 0)
        pools().sync()
        for now, was, new in ((c.gk, before[0], 5.0), (c.gv, before[1], 6.0)):
            assert bool(((now == was) | (now == new)).all()), offsets


# ---- calls ---------------------------------------------------------------------------------------
def test_refusals_that_need_a_pool(pools):
    pool, p = pools(), torch.zeros(4096, device="cuda").data_ptr()
    q = p + 4096

    def refused(status, f, *args):
        with pytest.raises(S.SgprsError) as e:
            f(*args)
        assert e.value.status == status, str(e.value)

    n = S.RmsNormDesc(m=2, c=8, dtype=S.SGPRS_F32, out_dtype=S.SGPRS_F32)
    n8 = S.RmsNormDesc(m=2, c=8, dtype=S.SGPRS_F32, out_dtype=S.SGPRS_I8)
    for args in ((n, None, None, None, None, q, None), (n, p, None, None, None, None, None), (n, p, None, None, q + 64, q, None), (n, p, None, None, None, q, q),
                 (n, p, q, None, q + 64, q + 64, None), (n8, p, None, None, None, q, None), (n8, p, None, None, None, p, q), (n8, p, q, None, None, q, p + 64),
                 (n, p + 2, None, None, None, q, None), (n, p, None, q + 1, None, q, None), (n8, p, None, None, None, q + 1, q + 66),
                 (S.RmsNormDesc(m=2, c=8, dtype=0, out_dtype=0, ldx=9), p, None, None, None, p, None), (S.RmsNormDesc(m=2, c=8, dtype=0, out_dtype=0, ldr=9), p, q, None, q, p + 512, None)):
        refused(-1, S.sgprs_rms_norm, *args, pool, 0)
    z = S.QuantizeDesc(m=2, c=8, dtype=S.SGPRS_BF16)
    for args in ((z, None, q, p), (z, p, None, q), (z, p, q, None), (z, p, p, q), (z, p + 1, q, q + 64), (z, p, q, q + 62)):
        refused(-1, S.sgprs_quantize_i8, *args, pool, 0)
    li = S.LinearI8Desc(m=2, n=4, k=8, dtype=S.SGPRS_BF16)
    for args in ((None, None, q, None, None, None, q), (p, None, None, None, None, None, q), (p, None, q, None, None, None, None), (p, None, q, None, None, None, p),
                 (p, None, q, None, None, None, q), (p, q + 2, q, None, None, None, q + 64), (p, None, q, None, None, q + 65, q + 128)):
        refused(-1, S.sgprs_linear_i8, li, *args, None, 0, pool, 0)
    refused(-1, S.sgprs_linear_i8, S.LinearI8Desc(m=2, n=4, k=8, dtype=1, ldr=5), p, None, q, None, None, q + 64, q + 64, None, 0, pool, 0)
    cache = dict(n_seqs=2, kv_heads=1, head_dim=8, dtype=S.SGPRS_F32, n_pages=2, page_size=4, table_width=1)
    ap = S.PagedAppendDesc(total=2, **cache)
    fine = [p, p + 512, None, q, q + 64, q + 512, q + 1024]
    for i, bad in ((0, None), (1, p + 8), (2, q + 2), (3, None), (4, q + 66), (5, None), (5, p), (6, q + 512), (6, q + 1028)):
        args = list(fine)
        args[i] = bad
        refused(-1, S.sgprs_paged_append, ap, *args, pool, 0)
    refused(-1, S.sgprs_paged_append, S.PagedAppendDesc(total=1, **cache), *fine, pool, 0)
    at = S.PagedAttentionDesc(heads=2, **cache)
    need = S.sgprs_paged_attention_workspace(at, CUS)
    ws = torch.zeros(need + 16, dtype=torch.uint8, device="cuda").data_ptr()
    fine = [p, p + 512, p + 1024, q, q + 64, q + 512, ws, need]
    for i, bad in ((0, None), (0, p + 8), (1, None), (2, None), (3, None), (3, q + 2), (4, None), (5, None), (5, p), (5, q + 8), (6, None), (6, ws + 8), (7, need - 1)):
        args = list(fine)
        args[i] = bad
        refused(-1, S.sgprs_paged_attention, at, *args, pool, 0)
    for f, d, args in ((S.sgprs_rms_norm, n, (p, None, None, None, q, None)), (S.sgprs_quantize_i8, z, (p, q, q + 64))):
        refused(-1, f, d, *args, pool, 1)


def test_empty_calls_write_nothing(pools):
    y = torch.full((64,), 5.0, device="cuda")
    p, out, pool = torch.ones(256, device="cuda").data_ptr(), y.data_ptr(), pools()
    torch.cuda.synchronize()
    S.sgprs_rms_norm(S.RmsNormDesc(m=0, c=8, dtype=0, out_dtype=2), p, None, None, None, out, out, pool, 0)
    S.sgprs_quantize_i8(S.QuantizeDesc(m=0, c=8, dtype=0), p, out, out, pool, 0)
    S.sgprs_linear_i8(S.LinearI8Desc(m=0, n=8, k=8, dtype=0), p, None, p, None, None, None, out, None, 0, pool, 0)
    cache = dict(n_seqs=2, kv_heads=1, head_dim=8, dtype=S.SGPRS_F32, n_pages=1, page_size=1, table_width=1)
    S.sgprs_paged_append(S.PagedAppendDesc(total=0, **cache), p, p, p, p, p, out, out + 64, pool, 0)
    torch.cuda.synchronize()
    assert bool((y == 5.0).all())


def test_a_step_in_a_graph_follows_lengths_that_grow(pools):
    """Norm, product, append and attention captured once and replayed while the sequences grow, against the same calls."""
    pool, g = pools(), gen(3)
    n, c, heads, hk, dim, page, steps = 5, 256, 4, 2, 64, 16, 4
    start = [1, 15, 130, 0, 700]
    cache = Cache("bf16", [v + steps for v in start], page, hk, dim, seed=2)
    cache.lens = torch.tensor(start, dtype=torch.int32)
    cache.to_gpu()
    kv = hk * dim
    x, ga = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda"), (torch.rand(c, generator=g) + 0.5).cuda()
    w = torch.randint(-127, 128, (heads * dim + 2 * kv, c), generator=g, dtype=torch.int8).cuda()
    sw = torch.full((w.shape[0],), 1 / (74 * 16), device="cuda")
    q8, sx = torch.zeros(n, c, dtype=torch.int8, device="cuda"), torch.zeros(n, device="cuda")
    rows, out = torch.zeros(n, w.shape[0], dtype=torch.bfloat16, device="cuda"), torch.zeros(n, heads * dim, dtype=torch.bfloat16, device="cuda")
    dn = S.RmsNormDesc(m=n, c=c, dtype=1, out_dtype=2, eps=1e-6)
    dl = S.LinearI8Desc(m=n, n=w.shape[0], k=c, dtype=1)
    da = S.PagedAppendDesc(total=n, ldk=w.shape[0], ldv=w.shape[0], **cache.dims)
    dt = S.PagedAttentionDesc(heads=heads, ldq=w.shape[0], **cache.dims)
    nl, nt = S.sgprs_linear_i8_workspace(dl, CUS), S.sgprs_paged_attention_workspace(dt, CUS)
    ws = torch.empty(max(nl, nt, 16), dtype=torch.uint8, device="cuda")
    one = rows.element_size()

    def step():
        S.sgprs_rms_norm(dn, ptr(x), None, ptr(ga), None, ptr(q8), ptr(sx), pool, 0)
        S.sgprs_linear_i8(dl, ptr(q8), ptr(sx), ptr(w), ptr(sw), None, None, ptr(rows), ptr(ws), nl, pool, 0)
        S.sgprs_paged_append(da, ptr(rows) + heads * dim * one, ptr(rows) + (heads * dim + kv) * one, None, ptr(cache.gtable), ptr(cache.glens), ptr(cache.gk), ptr(cache.gv), pool, 0)
        S.sgprs_paged_attention(dt, ptr(rows), ptr(cache.gk), ptr(cache.gv), ptr(cache.gtable), ptr(cache.glens), ptr(out), ptr(ws), nt, pool, 0)

    torch.cuda.synchronize()
    step()
    pool.sync()
    stream, graph = torch.cuda.ExternalStream(pool.stream(0)), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        graph.capture_begin()
        step()
        graph.capture_end()
    for i in range(steps):
        cache.glens.add_(1)
        x.copy_(torch.randn(n, c, generator=gen(40 + i)).bfloat16())
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        replayed, k = out.clone(), cache.gk.clone()
        out.zero_()
        torch.cuda.synchronize()
        step()
        pool.sync()
        assert torch.equal(replayed, out) and torch.equal(bits(k), bits(cache.gk)) and bool((out != 0).any(1).all()), i
        lens = (torch.tensor(start) + i + 1).tolist()
        cache.k, cache.v = cache.gk.cpu(), cache.gv.cpu()
        hk_, hv_ = cache.host()
        got_rows = rows.cpu()
        want, bound = ref.paged_attention(got_rows[:, :heads * dim].reshape(n, heads, dim), hk_, hv_, cache.table, lens, 0, 0, 0.0)
        block_ops_util.assert_within(out.view(n, heads, dim), want, bound, f"step {i}")
        h, q, s = ref.rms_norm(x.cpu(), None, ga.cpu(), 1e-6, True)
        same(q8, q, f"step {i}")
        want, bound = ref.linear_i8(q, sx.cpu(), w.cpu(), sw.cpu(), None, None, 0, 0, torch.bfloat16)
        block_ops_util.assert_within(rows, want, bound, f"step {i}")
        for s_, p in enumerate(lens):
            assert torch.equal(bits(hk_[cache.table[s_, (p - 1) // page], (p - 1) % page]), bits(got_rows[s_, heads * dim:heads * dim + kv].view(hk, dim)))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_a_layer_of_a_decoding_step(pools, name):
    """All of the operators in a row, as a layer uses them: weights to integers once, then norm, q / k / v, append, attention,
    output product on top of the residual, norm with its addition, and the two products behind it; each against the
    definition of what the one before it gave."""
    dt, tdt = DT[name]
    pool, g = pools(), gen(9)
    n, c, heads, hk, dim, wide = 6, 320, 4, 2, 40, 700
    kv = hk * dim
    cache = Cache(name, [5, 1, 260, 33, 700, 64], 16, hk, dim, seed=2).to_gpu()
    lens = cache.lens.tolist()

    def empty(*shape, dtype=tdt):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    def weights(rows, k):
        w = (torch.randn(rows, k, generator=g) / math.sqrt(k)).to(tdt)
        gw, q, sc = w.cuda(), empty(rows, k, dtype=torch.int8), empty(rows, dtype=torch.float32)
        torch.cuda.synchronize()
        S.sgprs_quantize_i8(S.QuantizeDesc(m=rows, c=k, dtype=dt), ptr(gw), ptr(q), ptr(sc), pool, 0)
        pool.sync()
        want, ws = ref.quantize(w)
        same(q, want, "weights")
        return q, sc

    def product(x, sx, w, act=0, res=None, on=None):
        q, sw = w
        rows = q.shape[0]
        y = on if on is not None else empty(n, rows)
        rh = res.cpu() if res is not None else None
        d = S.LinearI8Desc(m=n, n=rows, k=q.shape[1], dtype=dt, act=act)
        torch.cuda.synchronize()
        S.sgprs_linear_i8(d, ptr(x), ptr(sx), ptr(q), ptr(sw), None, ptr(res) if res is not None else None, ptr(y), None, 0, pool, 0)
        pool.sync()
        want, bound = ref.linear_i8(x.cpu(), sx.cpu(), q.cpu(), sw.cpu(), None, rh, act, 0, tdt)
        block_ops_util.assert_within(y, want, bound, f"product to {rows}")
        return y

    def norm(x, res, gamma, sum_on):
        q, sc, xh, rh = empty(n, c, dtype=torch.int8), empty(n, dtype=torch.float32), x.cpu(), res.cpu() if res is not None else None
        torch.cuda.synchronize()
        S.sgprs_rms_norm(S.RmsNormDesc(m=n, c=c, dtype=dt, out_dtype=S.SGPRS_I8, eps=1e-6), ptr(x), ptr(res) if res is not None else None, ptr(gamma),
                         ptr(sum_on) if sum_on is not None else None, ptr(q), ptr(sc), pool, 0)
        pool.sync()
        h, want, _ = ref.rms_norm(xh, rh, gamma.cpu(), 1e-6, True)
        same(q, want, "norm")
        assert sum_on is None or torch.equal(bits(sum_on.cpu()), bits(h))
        return q, sc

    w_qkv, w_o, w_up, w_down = weights(heads * dim + 2 * kv, c), weights(c, heads * dim), weights(wide, c), weights(c, wide)
    gamma = [(torch.rand(c, generator=g) + 0.5).cuda() for _ in range(3)]
    x = torch.randn(n, c, generator=g).to(tdt).cuda()
    rows = product(*norm(x, None, gamma[0], None), w_qkv)
    es, ld = rows.element_size(), rows.shape[1]
    S.sgprs_paged_append(S.PagedAppendDesc(total=n, ldk=ld, ldv=ld, **cache.dims), ptr(rows) + heads * dim * es, ptr(rows) + (heads * dim + kv) * es, None, ptr(cache.gtable),
                         ptr(cache.glens), ptr(cache.gk), ptr(cache.gv), pool, 0)
    d = S.PagedAttentionDesc(heads=heads, ldq=ld, **cache.dims)
    need, o = S.sgprs_paged_attention_workspace(d, CUS), empty(n, heads * dim)
    ws = empty(need, dtype=torch.uint8)
    torch.cuda.synchronize()
    S.sgprs_paged_attention(d, ptr(rows), ptr(cache.gk), ptr(cache.gv), ptr(cache.gtable), ptr(cache.glens), ptr(o), ptr(ws), need, pool, 0)
    pool.sync()
    rh = rows.cpu()
    k, v = ref.paged_append(*(t.reshape(n, hk, dim) for t in rh[:, heads * dim:].split(kv, 1)), None, cache.table, lens, *cache.host())
    cache.k, cache.v = cache.gk.cpu(), cache.gv.cpu()
    for a, b in zip(cache.host(), (k, v)):
        assert torch.equal(bits(a), bits(b))
    want, bound = ref.paged_attention(rh[:, :heads * dim].reshape(n, heads, dim), k, v, cache.table, lens, 0, 0, 0.0)
    block_ops_util.assert_within(o.view(n, heads, dim), want, bound, "attention")
    q8, sc = empty(n, heads * dim, dtype=torch.int8), empty(n, dtype=torch.float32)
    torch.cuda.synchronize()
    S.sgprs_quantize_i8(S.QuantizeDesc(m=n, c=heads * dim, dtype=dt), ptr(o), ptr(q8), ptr(sc), pool, 0)
    pool.sync()
    same(q8, ref.quantize(o.cpu())[0], "attention's rows")
    y = product(q8, sc, w_o)
    up = product(*norm(y, x, gamma[1], x), w_up, act=3)
    q8, sc = empty(n, wide, dtype=torch.int8), empty(n, dtype=torch.float32)
    torch.cuda.synchronize()
    S.sgprs_quantize_i8(S.QuantizeDesc(m=n, c=wide, dtype=dt), ptr(up), ptr(q8), ptr(sc), pool, 0)
    pool.sync()
    product(q8, sc, w_down, res=x, on=x)
    norm(x, None, gamma[2], None)


def test_two_graphs_that_share_a_workspace(pools):
    """Replayed in turn on one stream, with lengths that change between the replays."""
    pool = pools()
    kv = [900, 3000, 17, 0]
    calls = []
    for i, (name, heads, hk, dim) in enumerate((("bf16", 8, 2, 64), ("f32", 6, 2, 96))):
        c = Cache(name, kv, 16, hk, dim, seed=i).to_gpu()
        d = S.PagedAttentionDesc(heads=heads, **c.dims)
        q = torch.randn(len(kv), heads * dim, generator=gen(i)).to(DT[name][1])
        calls.append((c, d, q, q.cuda(), torch.empty_like(q, device="cuda"), S.sgprs_paged_attention_workspace(d, CUS)))
    ws = torch.empty(max(t[5] for t in calls), dtype=torch.uint8, device="cuda")
    stream, graphs = torch.cuda.ExternalStream(pool.stream(0)), []

    def call(c, d, _, gq, o, need):
        S.sgprs_paged_attention(d, ptr(gq), ptr(c.gk), ptr(c.gv), ptr(c.gtable), ptr(c.glens), ptr(o), ptr(ws), need, pool, 0)

    torch.cuda.synchronize()
    for t in calls:
        call(*t)
        pool.sync()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(stream):
            graphs[-1].capture_begin()
            call(*t)
            graphs[-1].capture_end()
    for lens in (kv, [3, 2500, 17, 0], [0, 0, 0, 0], kv, [900, 1, 0, 0]):
        for c, _, _, _, o, _ in calls:
            c.glens.copy_(torch.tensor(lens, dtype=torch.int32))
            o.fill_(NAN)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for c, d, q, _, o, _ in calls:
            k, v = c.host()
            want, bound = ref.paged_attention(q.view(len(kv), d.heads, d.head_dim), k, v, c.table, lens, 0, 0, 0.0)
            block_ops_util.assert_within(o.view(len(kv), d.heads, d.head_dim), want, bound, f"{lens}")


def test_two_partitions_at_once(pools):
    """Attention over the same cache on two partitions, each with a workspace of its own."""
    pool = S.Pool(2, 128)
    try:
        c = Cache("bf16", [900, 3000, 17], 16, 2, 64, seed=8).to_gpu()
        q = [torch.randn(3, 256, generator=gen(i)).bfloat16().cuda() for i in range(2)]
        o = [torch.zeros_like(t) for t in q]
        d = S.PagedAttentionDesc(heads=4, **c.dims)
        need = S.sgprs_paged_attention_workspace(d, 128)
        ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                S.sgprs_paged_attention(d, ptr(q[i]), ptr(c.gk), ptr(c.gv), ptr(c.gtable), ptr(c.glens), ptr(o[i]), ptr(ws[i]), need, pool, i)
        pool.sync()
        k, v = c.host()
        for i in range(2):
            want, bound = ref.paged_attention(q[i].cpu().view(3, 4, 64), k, v, c.table, [900, 3000, 17], 0, 0, 0.0)
            block_ops_util.assert_within(o[i].view(3, 4, 64), want, bound, f"partition {i}")
    finally:
        pool.destroy()
