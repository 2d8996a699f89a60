"""GPU parity of the attention-block operators (linear, group norm, attention) with 64-bit definitions, at
the sizes, strides, lengths and masks where a kernel can go wrong."""
import math

import pytest
import torch

import paper_2406_09425_amd as S
import block_ops_util as ref

pytestmark = pytest.mark.gpu

DT = {"f32": (S.SGPRS_F32, torch.float32), "bf16": (S.SGPRS_BF16, torch.bfloat16)}
CUS = 256


@pytest.fixture(scope="module")
def pools():
    made = {}

    def get(cus=CUS):
        if cus not in made:
            made[cus] = S.Pool(1, cus)
        return made[cus]

    yield get
    for p in made.values():
        p.destroy()


def ptr(t):
    return t.data_ptr() if t is not None else None


def gen(seed):
    return torch.Generator().manual_seed(seed)


class Rows:
    """`m` rows of `c` values inside a wider buffer whose other values are a sentinel that nothing may change."""

    def __init__(self, host, pad=0, lead=0):
        m, c = host.shape
        self.buf = torch.full((lead + m * (c + pad) + 64,), 777.0, dtype=host.dtype)
        self.view_of(self.buf, m, c, pad, lead).copy_(host)
        self.before = self.buf.clone()
        self.buf = self.buf.cuda()
        self.t = self.view_of(self.buf, m, c, pad, lead)
        self.args = (m, c, pad, lead)
        self.ld = c + pad

    @staticmethod
    def view_of(buf, m, c, pad, lead):
        return buf[lead:lead + m * (c + pad)].view(m, c + pad)[:, :c]

    def outside_untouched(self):
        now, was = self.buf.cpu(), self.before.clone()
        self.view_of(now, *self.args).zero_()
        self.view_of(was, *self.args).zero_()
        return torch.equal(now, was)


# ---- linear --------------------------------------------------------------------------------------
def run_linear(pools, name, m, n, k, act=0, bias=True, res=False, first=0, pads=(0, 0, 0, 0), lead=0, cus=CUS, seed=0, x=None, w=None, inplace=False):
    dt, tdt = DT[name]
    g = gen(seed)
    x = torch.randn(m, k, generator=g) if x is None else x
    w = torch.randn(n, k, generator=g) / math.sqrt(k) if w is None else w
    xh, wh = x.to(tdt), w.to(tdt)
    bh = torch.randn(n, generator=g) if bias else None
    rh = torch.randn(m, n, generator=g).to(tdt) if res else None
    X, W = Rows(xh, pads[0], lead), Rows(wh, pads[1], lead)
    R = Rows(rh, pads[2], lead) if res else None
    Y = R if inplace else Rows(torch.full((m, n), float("nan")).to(tdt), pads[3], lead)
    B = bh.cuda() if bias else None
    pool = pools(cus)
    d = S.LinearDesc(m=m, n=n, k=k, dtype=dt, act=act, residual_first=first, ldx=X.ld, ldw=W.ld, ldr=R.ld if res else 0, ldy=Y.ld)
    ws_bytes = S.sgprs_linear_workspace(d, cus)
    ws = torch.full((max(ws_bytes, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def call():
        S.sgprs_linear(d, ptr(X.t), ptr(W.t), ptr(B), ptr(R.t) if res else None, ptr(Y.t), ptr(ws), ws_bytes, pool, 0)
        pool.sync()
        return Y.t.cpu().clone()

    got = call()
    want, bound = ref.linear(xh, wh, bh, rh, act, first)
    what = f"linear {name} {m}x{k}->{n} act {act} pads {pads} lead {lead} cus {cus}"
    ref.assert_within(got, want, bound, what)
    for t in (X, W, Y) + ((R,) if res else ()):
        assert t.outside_untouched(), what
    if not inplace:
        assert torch.equal(call().nan_to_num(), got.nan_to_num()), f"{what}: a second call gives other bits"
    return got


LINEAR = [(1, 1, 1), (1, 1000, 512), (2, 3, 7), (5, 16, 32), (16, 33, 64), (17, 64, 40), (24, 512, 1024), (31, 100, 2048), (33, 65, 72), (48, 1000, 520),
          (64, 64, 64), (65, 130, 96), (100, 1000, 512), (128, 128, 128), (129, 257, 136), (200, 2049, 64), (255, 256, 1032), (256, 256, 256),
          (257, 300, 512), (500, 96, 4096), (784, 512, 512), (1025, 768, 200), (2048, 1040, 264), (3137, 64, 64)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LINEAR, ids=lambda s: "x".join(map(str, s)))
def test_linear_shapes(pools, name, shape):
    m, n, k = shape
    i = LINEAR.index(shape)
    run_linear(pools, name, m, n, k, act=i % 4, bias=i % 3 != 1, res=i % 2 == 1, first=(i // 2) % 2, seed=i)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("first", [0, 1])
@pytest.mark.parametrize("m", [3, 150])
def test_linear_epilogues(pools, name, act, first, m):
    run_linear(pools, name, m, 136, 48, act=act, res=True, first=first, seed=50 + act)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 20, 70, 300])
@pytest.mark.parametrize("pads,lead", [((8, 8, 8, 8), 0), ((3, 0, 0, 0), 0), ((0, 1, 0, 0), 0), ((0, 0, 3, 0), 0), ((0, 0, 0, 5), 0), ((5, 3, 1, 7), 1), ((4, 4, 4, 4), 4)],
                         ids=str)
def test_linear_strides_and_alignment(pools, name, m, pads, lead):
    run_linear(pools, name, m, 200, 136, res=True, pads=pads, lead=lead, seed=3)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n,k", [(130, 517), (509, 67), (61, 130), (131, 4), (129, 2)])
@pytest.mark.parametrize("m", [1, 19, 130, 333])
def test_linear_odd_widths(pools, name, m, n, k):
    run_linear(pools, name, m, n, k, act=2, res=True, seed=m + n)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("cus", [8, 40, 128])
@pytest.mark.parametrize("shape", [(9, 256, 2048), (196, 512, 512), (700, 640, 256)], ids=str)
def test_linear_on_partitions(pools, name, cus, shape):
    run_linear(pools, name, *shape, act=3, cus=cus, seed=cus)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape,cus", [((2816, 2800, 520), 128), ((2815, 2817, 512), 128), ((1500, 1400, 96), 64), ((1501, 1300, 101), 64)], ids=str)
def test_linear_large_tiles(pools, name, shape, cus):
    """Products whose tiles fill a partition: the largest tiles, ragged at both edges, with and without whole chunks."""
    run_linear(pools, name, *shape, act=2, res=True, cus=cus, seed=1)


@pytest.mark.parametrize("m,n,k,cus", [(300, 140, 96, 256), (600, 700, 40, 8)])
def test_linear_fp32_at_the_ends_of_the_range(pools, m, n, k, cus):
    """Values that round up to infinity in fewer bits, and values whose lower parts fall below the normal range."""
    g = gen(10)
    x, w = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g)
    x[3] = 0.0
    x[3, 1] = 3.4028e38
    w[:, 1] = w[:, 1].clamp(-0.9, 0.9)
    x[40:70] *= 2.0 ** -118
    x[100, :] = 2.0 ** -120
    x[101, :] = 0.0
    run_linear(pools, "f32", m, n, k, bias=False, x=x, w=w, cus=cus)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("m", [7, 40, 300])
def test_linear_in_place_residual(pools, name, m):
    run_linear(pools, name, m, 264, 512, res=True, inplace=True, pads=(0, 0, 8, 0), seed=m)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("m", [5, 300])
def test_linear_non_finite_and_extreme_values(pools, name, m):
    """NaN and infinity reach their own rows and columns only; large and tiny values keep their range."""
    g = gen(9)
    x, w = torch.randn(m, 96, generator=g), torch.randn(140, 96, generator=g) / 8
    x[0, 5], x[1, 7], x[2, 95] = float("nan"), float("inf"), float("-inf")
    w[3, 11] = float("inf")
    x[m - 1] *= 1e30
    x[m - 2] *= 1e-30
    x[:, 11] = x[:, 11].abs() + 0.1
    w[:, 7] = w[:, 7].abs() + 0.1
    w[:, 95] = w[:, 95].abs() + 0.1
    w[3, 95] = -w[3, 95]  # the row with -inf meets the column with +inf: both at +inf
    run_linear(pools, name, m, 140, 96, bias=False, x=x, w=w)


def test_linear_rows_beyond_32_bit_offsets(pools):
    """Rows 2^20 elements apart: the last ones lie more than 4 GiB behind the first."""
    m, n, k, ld = 2200, 72, 64, 1 << 20
    g = gen(4)
    xh, wh = torch.randn(m, k, generator=g).bfloat16(), torch.randn(n, k, generator=g).bfloat16()
    buf = torch.empty(m * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(m, ld)[:, :k]
    x.copy_(xh)
    y = buf.view(m, ld)[:, 4096:4096 + n]
    wd = wh.cuda()
    pool = pools()
    d = S.LinearDesc(m=m, n=n, k=k, dtype=S.SGPRS_BF16, ldx=ld, ldy=ld)
    ws_bytes = S.sgprs_linear_workspace(d, CUS)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    S.sgprs_linear(d, ptr(x), ptr(wd), None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    want, bound = ref.linear(xh, wh, None, None, 0, 0)
    ref.assert_within(y.cpu(), want, bound, "rows 2^20 apart")


# ---- group norm ----------------------------------------------------------------------------------
def run_norm(pools, name, n, hw, c, groups, act=0, affine=True, res=False, pads=(0, 0, 0), lead=0, cus=CUS, seed=0, x=None, eps=1e-5, inplace=None):
    dt, tdt = DT[name]
    g = gen(seed)
    x = torch.randn(n * hw, c, generator=g) * 1.5 + torch.randn(c, generator=g) if x is None else x
    xh = x.to(tdt)
    gh, bh = (torch.rand(c, generator=g) + 0.5, torch.randn(c, generator=g)) if affine else (None, None)
    rh = torch.randn(n * hw, c, generator=g).to(tdt) if res else None
    X = Rows(xh, pads[0], lead)
    R = Rows(rh, pads[1], lead) if res else None
    Y = X if inplace == "x" else R if inplace == "residual" else Rows(torch.full((n * hw, c), float("nan")).to(tdt), pads[2], lead)
    G, B = (gh.cuda(), bh.cuda()) if affine else (None, None)
    pool = pools(cus)
    d = S.GroupNormDesc(n=n, hw=hw, c=c, groups=groups, dtype=dt, act=act, eps=eps, ldx=X.ld, ldr=R.ld if res else 0, ldy=Y.ld)
    ws_bytes = S.sgprs_group_norm_workspace(d, cus)
    ws = torch.full((max(ws_bytes, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def call():
        S.sgprs_group_norm(d, ptr(X.t), ptr(G), ptr(B), ptr(R.t) if res else None, ptr(Y.t), ptr(ws), ws_bytes, pool, 0)
        pool.sync()
        return Y.t.cpu().clone()

    got = call()
    want, bound = ref.group_norm(xh, gh, bh, rh, n, hw, groups, eps, act)
    what = f"group norm {name} {n}x{hw}x{c} groups {groups} act {act} pads {pads} lead {lead} cus {cus}"
    ref.assert_within(got, want, bound, what)
    for t in (X, Y) + ((R,) if res else ()):
        assert t.outside_untouched(), what
    if not inplace:
        assert torch.equal(call().nan_to_num(), got.nan_to_num()), f"{what}: a second call gives other bits"


def test_group_norm_of_many_positions(pools):
    """More chunks of positions than a grid's second dimension holds."""
    hw, c = 600000, 2048
    x = torch.empty(hw, c, dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.zeros_like(x)
    d = S.GroupNormDesc(n=1, hw=hw, c=c, groups=8, dtype=S.SGPRS_BF16, eps=1e-5)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_group_norm(d, ptr(x), None, None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    for at in (0, hw // 2, hw - 64):
        part = x[at:at + 64].double().reshape(64, 8, 256)
        mean = torch.stack([x[:, i * 256:(i + 1) * 256].float().mean().double() for i in range(8)])[None, :, None]
        var = torch.stack([x[:, i * 256:(i + 1) * 256].float().var().double() for i in range(8)])[None, :, None]
        want = ((part - mean) / (var + 1e-5).sqrt()).reshape(64, c)
        assert float((y[at:at + 64].double() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) + 1e-4


NORM = [(1, 1, 1, 1), (1, 1, 64, 1), (3, 1, 512, 1), (1000, 1, 512, 1), (77, 1, 1000, 1), (5, 1, 4096, 1), (9, 1, 33, 3), (1, 49, 512, 32), (2, 49, 512, 512),
        (13, 196, 256, 32), (4, 196, 256, 1), (2, 784, 128, 32), (1, 3136, 64, 32), (3, 3136, 64, 8), (1, 12544, 64, 32), (2, 5000, 320, 32), (3, 527, 96, 8),
        (2, 527, 99, 9), (1, 1, 2048, 32), (40, 7, 24, 24), (1, 20000, 8, 1), (2, 333, 1030, 1), (300, 2, 16, 4), (1, 9000, 512, 4)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", NORM, ids=lambda s: "x".join(map(str, s)))
def test_group_norm_shapes(pools, name, shape):
    i = NORM.index(shape)
    run_norm(pools, name, *shape, act=i % 4, affine=i % 3 != 2, res=i % 2 == 1, seed=i)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 50, 96, 8), (2, 3000, 64, 32), (100, 1, 256, 1), (2, 700, 60, 4)], ids=str)
@pytest.mark.parametrize("pads,lead", [((8, 8, 8), 0), ((3, 0, 0), 0), ((0, 3, 0), 0), ((0, 0, 3), 0), ((5, 3, 1), 1), ((4, 4, 4), 4)], ids=str)
def test_group_norm_strides_and_alignment(pools, name, shape, pads, lead):
    run_norm(pools, name, *shape, act=3, res=True, pads=pads, lead=lead, seed=2)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 50, 96, 8), (2, 6000, 64, 32), (100, 1, 256, 1)], ids=str)
@pytest.mark.parametrize("inplace", ["x", "residual"])
def test_group_norm_in_place(pools, name, shape, inplace):
    run_norm(pools, name, *shape, act=1, res=True, inplace=inplace, seed=6)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("cus", [8, 40, 128])
@pytest.mark.parametrize("shape", [(1, 49, 512, 32), (5, 3136, 64, 32), (500, 1, 512, 1)], ids=str)
def test_group_norm_on_partitions(pools, name, cus, shape):
    run_norm(pools, name, *shape, act=3, cus=cus, seed=cus)


@pytest.mark.parametrize("shape", [(2, 49, 64, 8), (1, 12544, 64, 32), (50, 1, 512, 1)], ids=str)
def test_group_norm_with_a_mean_far_from_zero(pools, shape):
    """A thousand deviations from zero: a variance from the mean of squares would be lost."""
    n, hw, c, groups = shape
    run_norm(pools, "f32", n, hw, c, groups, x=torch.randn(n * hw, c, generator=gen(1)) + 1000.0, seed=1)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 49, 64, 8), (2, 12544, 64, 32), (50, 1, 512, 1)], ids=str)
def test_group_norm_non_finite_stays_in_its_group(pools, name, shape):
    n, hw, c, groups = shape
    x = torch.randn(n * hw, c, generator=gen(8))
    x[hw // 2, 3] = float("nan")
    x[n * hw - 1, c - 1] = float("inf")
    x[(n - 1) * hw, : c // groups] = 0.0
    run_norm(pools, name, n, hw, c, groups, x=x, seed=8)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_group_norm_of_constant_groups(pools, name):
    run_norm(pools, name, 2, 300, 64, 8, x=torch.full((600, 64), 3.25), seed=1)
    run_norm(pools, name, 7, 1, 48, 48, x=torch.randn(7, 48, generator=gen(2)), seed=2)  # groups of one value


# ---- attention -----------------------------------------------------------------------------------
def heads_buffer(host, layout, pad):
    """[tokens][heads][dim] in device memory, tokens or heads first, between sentinels; returns buffer, view and strides."""
    t, h, d = host.shape
    if layout == "tokens":
        buf = torch.full((max(t, 1), h * d + pad), 777.0, dtype=host.dtype, device="cuda")
        view, strides = buf[:t, :h * d].view(t, h, d) if pad == 0 else buf[:t, :h * d].unflatten(1, (h, d)), (h * d + pad, d)
    else:
        buf = torch.full((h, max(t, 1) + 1, d + pad), 777.0, dtype=host.dtype, device="cuda")
        view, strides = buf[:, :t, :d].transpose(0, 1), (d + pad, (max(t, 1) + 1) * (d + pad))
    view.copy_(host)
    return buf, view, strides


def offsets(lens):
    return torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).cuda()


def run_attention(pools, name, q_lens, kv_lens, heads, kv_heads, dim, causal, scale=0.0, layout="tokens", pad=0, cus=CUS, seed=0, change=None, repeat=True):
    dt, tdt = DT[name]
    g = gen(seed)
    tq, tk = sum(q_lens), sum(kv_lens)
    qh = (torch.randn(tq, heads, dim, generator=g) * 1.5).to(tdt)
    kh, vh = (torch.randn(tk, kv_heads, dim, generator=g).to(tdt) for _ in range(2))
    if change:
        change(qh, kh, vh)
    (qb, q, qs), (kb, k, ks), (vb, v, vs) = (heads_buffer(t, layout, pad) for t in (qh, kh, vh))
    ob, o, os_ = heads_buffer(torch.full((tq, heads, dim), float("nan")).to(tdt), layout, pad)
    qo, ko = offsets(q_lens), offsets(kv_lens)
    pool = pools(cus)
    d = S.AttentionDesc(n_seqs=len(q_lens), total_q=tq, total_kv=tk, max_q=max(q_lens), max_kv=max(kv_lens), heads=heads, kv_heads=kv_heads, head_dim=dim,
                        dtype=dt, causal=int(causal), scale=scale, ldq=qs[0], hq=qs[1], ldk=ks[0], hk=ks[1], ldv=vs[0], hv=vs[1], ldo=os_[0], ho=os_[1])
    ws_bytes = S.sgprs_attention_workspace(d, cus)
    ws = torch.full((max(ws_bytes, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def call():
        S.sgprs_attention(d, ptr(qb), ptr(kb), ptr(vb), ptr(qo), ptr(ko), ptr(ob), ptr(ws), ws_bytes, pool, 0)
        pool.sync()
        return o.cpu().clone()

    got = call()
    what = f"attention {name} q {q_lens} kv {kv_lens} heads {heads}/{kv_heads}x{dim} causal {causal} {layout} pad {pad} cus {cus}"
    want, bound = ref.attention(qh, kh, vh, q_lens, kv_lens, causal, scale)
    ref.assert_within(got, want, bound, what)
    o.fill_(777.0)
    assert bool((ob == 777.0).all()), f"{what}: something beside the output was written"
    if repeat:
        assert torch.equal(call().nan_to_num(), got.nan_to_num()), f"{what}: a second call gives other bits"


LENGTHS = [[1], [2, 1], [0, 5, 0], [16], [17, 31], [32, 33], [63, 64, 65], [1, 127, 0, 128, 129], [200, 3], [257], [300, 1, 1, 70], [513]]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", LENGTHS, ids=str)
def test_attention_packed_lengths(pools, name, causal, lens):
    i = LENGTHS.index(lens)
    run_attention(pools, name, lens, lens, [4, 2, 3][i % 3], [2, 1, 3][i % 3], [64, 128, 32][i % 3 if i % 2 else 0], causal, seed=i)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 48, 64, 72, 80, 96, 104, 128])
def test_attention_head_dims(pools, name, causal, dim):
    run_attention(pools, name, [70, 9, 130], [70, 9, 130], 4, 2, dim, causal, seed=dim)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (8, 1), (6, 2), (32, 8), (7, 1), (40, 2)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1, 1], [300, 1, 65]), ([33, 100], [33, 100])], ids=["tokens", "prompts"])
def test_attention_grouped_heads(pools, name, heads, kv_heads, q_lens, kv_lens):
    run_attention(pools, name, q_lens, kv_lens, heads, kv_heads, 64, True, seed=heads)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [1]), ([1], [5000]), ([1, 1, 1, 1], [1025, 0, 64, 2049]), ([2, 1, 3], [700, 63, 129]), ([5, 0, 7], [4097, 12, 7]),
                                            ([1] * 20, list(range(50, 1050, 50))), ([16], [3000]), ([17], [1500]),
                                            ([50, 7], [1700, 90]), ([61], [1000])], ids=str)
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (3, 3, 64)])
def test_attention_against_caches(pools, name, causal, q_lens, kv_lens, heads, kv_heads, dim):
    run_attention(pools, name, q_lens, kv_lens, heads, kv_heads, dim, causal, seed=len(q_lens))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,kv_lens", [([5], [0]), ([5, 3], [2, 0]), ([100, 40], [7, 200]), ([300], [100]), ([4, 4], [3, 4]), ([200, 64], [136, 0])], ids=str)
def test_attention_rows_without_keys(pools, name, causal, q_lens, kv_lens):
    """More queries than keys: under the causal mask the first ones see none and get zeros."""
    run_attention(pools, name, q_lens, kv_lens, 4, 2, 64, causal, seed=5)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,kv_lens", [([40, 1100], [40, 1100]), ([200, 33], [2100, 1500]), ([1000], [420]), ([140, 60, 1], [1300, 0, 1900])], ids=str)
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 1, 128), (1, 1, 64)])
def test_attention_prompts_split_by_keys(pools, name, causal, q_lens, kv_lens, heads, kv_heads, dim):
    """Few tiles and many keys: a tile's keys go to several workgroups, some of which hold none that it sees."""
    d = S.AttentionDesc(n_seqs=len(q_lens), total_q=sum(q_lens), total_kv=sum(kv_lens), max_q=max(q_lens), max_kv=max(kv_lens), heads=heads, kv_heads=kv_heads,
                        head_dim=dim, dtype=DT[name][0], causal=int(causal))
    if max(kv_lens) >= 1000:
        assert S.sgprs_attention_workspace(d, CUS) > 0
    run_attention(pools, name, q_lens, kv_lens, heads, kv_heads, dim, causal, seed=dim)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attention_split_prompts_do_not_spread_what_is_not_finite(pools, bad):
    def change(q, k, v):
        v[700, :, 5] = bad

    run_attention(pools, "bf16", [1200], [1200], 2, 1, 64, True, seed=3, change=change)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("layout,pad", [("tokens", 8), ("tokens", 64), ("heads", 0), ("heads", 8)])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 2], [300, 65]), ([90, 200], [90, 200])], ids=["tokens", "prompts"])
def test_attention_layouts(pools, name, layout, pad, q_lens, kv_lens):
    run_attention(pools, name, q_lens, kv_lens, 4, 2, 80, True, layout=layout, pad=pad, seed=7)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("cus", [8, 40, 128])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [2000, 77]), ([196] * 3, [196] * 3)], ids=["tokens", "prompts"])
def test_attention_on_partitions(pools, name, cus, q_lens, kv_lens):
    run_attention(pools, name, q_lens, kv_lens, 8, 4, 64, False, cus=cus, seed=cus)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,kv_lens", [([3], [900]), ([150], [150])], ids=["tokens", "prompts"])
@pytest.mark.parametrize("scale", [2.0, -2.0, 1e-3])
def test_attention_scales(pools, name, q_lens, kv_lens, scale):
    """Scores that leave one key all the weight, of either sign, and scores that are all alike."""
    run_attention(pools, name, q_lens, kv_lens, 4, 2, 64, True, scale=scale, seed=11)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 3e38, -3e38])
@pytest.mark.parametrize("q_lens,kv_lens,at", [([100, 100], [100, 100], 60), ([130, 20], [130, 20], 129), ([4, 4], [500, 500], 498), ([40, 1], [300, 30], 290)], ids=str)
def test_attention_keys_that_a_query_does_not_see(pools, name, bad, q_lens, kv_lens, at):
    """What is not finite in v (and, NaN and infinity aside, in k) at a key reaches the queries that see it and no
    other: not those before it, not those of the next sequence in the same buffers."""

    def change(q, k, v):
        v[at, :, 3] = bad
        if math.isnan(bad):
            k[at, 0, 1] = bad

    if not math.isfinite(bad):
        run_attention(pools, name, q_lens, kv_lens, 4, 2, 64, True, seed=13, change=change)
    else:
        run_attention(pools, name, q_lens[:1], kv_lens[:1], 4, 2, 64, True, seed=13, change=lambda q, k, v: v[at].fill_(bad / 4))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_attention_scores_beyond_the_exponentials_range(pools, name):
    """Scores thousands apart, growing and falling along the keys: the running maximum has to follow them."""

    def ramp(q, k, v):
        q.fill_(1.0)
        k.copy_((torch.arange(k.shape[0]).float() * (1 if up else -1)).to(k.dtype)[:, None, None].expand_as(k))

    for up in (True, False):
        run_attention(pools, name, [1, 1], [700, 90], 2, 1, 64, False, seed=1, change=ramp)
        run_attention(pools, name, [260], [260], 2, 1, 64, True, seed=1, change=ramp)


def test_attention_cache_beyond_32_bit_offsets(pools):
    """Heads first with 2^31 elements and more between the key heads, and tokens 2^17 elements apart."""
    dim, kv_heads, tokens, ld = 64, 2, 17000, 1 << 17
    g = gen(3)
    kh, vh = (torch.randn(tokens, kv_heads, dim, generator=g).bfloat16() for _ in range(2))
    qh = torch.randn(2, 4, dim, generator=g).bfloat16()
    buf = torch.empty(tokens * ld, dtype=torch.bfloat16, device="cuda")  # 4.5 GB
    at = buf.view(tokens, ld)
    k, v = (at[:, i * 4096:i * 4096 + kv_heads * dim].view(tokens, kv_heads, dim) for i in (0, 1))
    k.copy_(kh)
    v.copy_(vh)
    q, o = qh.cuda(), torch.zeros(2, 4, dim, dtype=torch.bfloat16, device="cuda")
    q_lens, kv_lens = [1, 1], [16000, 1000]
    d = S.AttentionDesc(n_seqs=2, total_q=2, total_kv=tokens, max_q=1, max_kv=16000, heads=4, kv_heads=kv_heads, head_dim=dim, dtype=S.SGPRS_BF16, ldk=ld, ldv=ld)
    pool = pools()
    ws_bytes = S.sgprs_attention_workspace(d, CUS)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    qo, ko = offsets(q_lens), offsets(kv_lens)
    torch.cuda.synchronize()
    S.sgprs_attention(d, ptr(q), ptr(k), ptr(v), ptr(qo), ptr(ko), ptr(o), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    want, bound = ref.attention(qh, kh, vh, q_lens, kv_lens, False, 0.0)
    ref.assert_within(o.cpu(), want, bound, "tokens 2^17 apart")
    # a prompt over the last tokens of the same buffers
    m = 90
    qh = torch.randn(m, 4, dim, generator=g).bfloat16()
    q, o = qh.cuda(), torch.zeros(m, 4, dim, dtype=torch.bfloat16, device="cuda")
    d = S.AttentionDesc(n_seqs=1, total_q=m, total_kv=m, max_q=m, max_kv=m, heads=4, kv_heads=kv_heads, head_dim=dim, dtype=S.SGPRS_BF16, causal=1, ldk=ld, ldv=ld)
    ws_bytes = S.sgprs_attention_workspace(d, CUS)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    qo = offsets([m])
    torch.cuda.synchronize()
    S.sgprs_attention(d, ptr(q), ptr(k) + (tokens - m) * ld * 2, ptr(v) + (tokens - m) * ld * 2, ptr(qo), ptr(qo), ptr(o), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    want, bound = ref.attention(qh, kh[-m:], vh[-m:], [m], [m], True, 0.0)
    ref.assert_within(o.cpu(), want, bound, "the last tokens of a large buffer")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,kv_lens,max_q,max_kv", [([3, 1], [300, 500], 3, 40), ([200, 40], [900, 70], 200, 70), ([3, 60], [300, 500], 3, 500)], ids=str)
def test_attention_sequences_longer_than_said(pools, name, q_lens, kv_lens, max_q, max_kv):
    """Results are unspecified then; what lies beside the output stays as it is."""
    dt, tdt = DT[name]
    heads, dim, tq, tk = 2, 64, sum(q_lens), sum(kv_lens)
    g = gen(2)
    q, k, v = (torch.randn(t, heads * dim, generator=g).to(tdt).cuda() for t in (tq, tk, tk))
    out = torch.full((tq + 8, heads * dim), 777.0, dtype=tdt, device="cuda")
    d = S.AttentionDesc(n_seqs=2, total_q=tq, total_kv=tk, max_q=max_q, max_kv=max_kv, heads=heads, kv_heads=heads, head_dim=dim, dtype=dt, causal=1)
    ws_bytes = S.sgprs_attention_workspace(d, CUS)
    ws = torch.full((ws_bytes + 4096,), 9, dtype=torch.uint8, device="cuda")
    qo, ko = offsets(q_lens), offsets(kv_lens)
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_attention(d, ptr(q), ptr(k), ptr(v), ptr(qo), ptr(ko), ptr(out), ptr(ws) if ws_bytes else None, ws_bytes, pool, 0)
    pool.sync()
    assert bool((out[tq:] == 777.0).all()) and bool((ws[ws_bytes:] == 9).all())


# ---- all together --------------------------------------------------------------------------------
def test_partitions_side_by_side():
    """The same calls on two partitions of a pool at once, each with a workspace of its own, as one after the other."""
    pool = S.Pool(2, 64)
    try:
        g = gen(41)
        m, c, heads = 600, 128, 2
        x, w = torch.randn(m, c, generator=g).bfloat16().cuda(), (torch.randn(3 * c, c, generator=g) / 11).bfloat16().cuda()
        off = offsets([600])
        dl = S.LinearDesc(m=m, n=3 * c, k=c, dtype=S.SGPRS_BF16)
        da = S.AttentionDesc(n_seqs=1, total_q=m, total_kv=m, max_q=m, max_kv=m, heads=heads, kv_heads=heads, head_dim=c // heads, dtype=S.SGPRS_BF16,
                             causal=1, ldq=3 * c, ldk=3 * c, ldv=3 * c)
        dn = S.GroupNormDesc(n=1, hw=m, c=c, groups=4, dtype=S.SGPRS_BF16, eps=1e-5)
        need = [f(d, 64) for f, d in ((S.sgprs_linear_workspace, dl), (S.sgprs_attention_workspace, da), (S.sgprs_group_norm_workspace, dn))]
        state = [dict(rows=torch.zeros(m, 3 * c, dtype=torch.bfloat16, device="cuda"), mixed=torch.zeros_like(x), out=torch.zeros_like(x),
                      ws=torch.empty(max(need + [16]), dtype=torch.uint8, device="cuda")) for _ in range(2)]
        torch.cuda.synchronize()

        def enqueue(p):
            s = state[p]
            S.sgprs_linear(dl, ptr(x), ptr(w), None, None, ptr(s["rows"]), ptr(s["ws"]), need[0], pool, p)
            S.sgprs_attention(da, ptr(s["rows"]), ptr(s["rows"]) + 2 * c, ptr(s["rows"]) + 4 * c, ptr(off), ptr(off), ptr(s["mixed"]), ptr(s["ws"]), need[1], pool, p)
            S.sgprs_group_norm(dn, ptr(s["mixed"]), None, None, ptr(x), ptr(s["out"]), ptr(s["ws"]), need[2], pool, p)

        enqueue(0)
        pool.sync()
        alone = state[0]["out"].clone()
        for _ in range(20):
            enqueue(0)
            enqueue(1)
        pool.sync()
        assert torch.equal(state[0]["out"], alone) and torch.equal(state[1]["out"], alone)
    finally:
        pool.destroy()


def test_refusals_enqueue_nothing(pools):
    pool = pools()
    t = torch.zeros(4096, dtype=torch.float32, device="cuda")
    y = torch.full((4096,), 5.0, dtype=torch.float32, device="cuda")
    off = offsets([4])
    p, out = t.data_ptr(), y.data_ptr()
    lin = dict(m=4, n=8, k=8, dtype=S.SGPRS_F32)
    norm = dict(n=1, hw=4, c=8, groups=2, dtype=S.SGPRS_F32)
    att = dict(n_seqs=1, total_q=4, total_kv=4, max_q=4, max_kv=4, heads=2, kv_heads=1, head_dim=8, dtype=S.SGPRS_F32)
    calls = [
        lambda: S.sgprs_linear(S.LinearDesc(**lin), None, p, None, None, out, None, 0, pool, 0),
        lambda: S.sgprs_linear(S.LinearDesc(**lin), p, p, None, None, out, None, 0, pool, 1),
        lambda: S.sgprs_linear(S.LinearDesc(**lin), p + 2, p, None, None, out, None, 0, pool, 0),
        lambda: S.sgprs_linear(S.LinearDesc(**lin), out, p, None, None, out, None, 0, pool, 0),
        lambda: S.sgprs_linear(S.LinearDesc(**lin, ldr=16), p, p, None, out, out, None, 0, pool, 0),
        lambda: S.sgprs_linear(S.LinearDesc(**lin, ldx=7), p, p, None, None, out, None, 0, pool, 0),
        lambda: S.sgprs_group_norm(S.GroupNormDesc(**norm), p, None, None, None, None, None, 0, pool, 0),
        lambda: S.sgprs_group_norm(S.GroupNormDesc(**norm, ldx=9), out, None, None, None, out, None, 0, pool, 0),
        lambda: S.sgprs_attention(S.AttentionDesc(**att), p, p, p, None, off.data_ptr(), out, None, 0, pool, 0),
        lambda: S.sgprs_attention(S.AttentionDesc(**att), p + 4, p, p, off.data_ptr(), off.data_ptr(), out, None, 0, pool, 0),
        lambda: S.sgprs_attention(S.AttentionDesc(**att), out, p, p, off.data_ptr(), off.data_ptr(), out, None, 0, pool, 0),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(S.SgprsError) as e:
            call()
        assert e.value.status == -1, i
    # nothing to do is no error
    S.sgprs_linear(S.LinearDesc(**{**lin, "m": 0}), p, p, None, None, out, None, 0, pool, 0)
    S.sgprs_group_norm(S.GroupNormDesc(**{**norm, "n": 0}), p, None, None, None, out, None, 0, pool, 0)
    S.sgprs_attention(S.AttentionDesc(**{**att, "total_q": 0, "max_q": 0}), p, p, p, off.data_ptr(), off.data_ptr(), out, None, 0, pool, 0)
    torch.cuda.synchronize()
    assert bool((y == 5.0).all())


def test_block_in_a_graph(pools):
    """Norm, product and attention captured on the partition's stream and replayed on inputs that change."""
    pool = pools()
    n, hw, c, heads = 3, 50, 64, 4
    g = gen(21)
    x = torch.zeros(n * hw, c, dtype=torch.bfloat16, device="cuda")
    wq = (torch.randn(3 * c, c, generator=g) / 8).bfloat16().cuda()
    norm, qkv, out = torch.zeros_like(x), torch.zeros(n * hw, 3 * c, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
    off = offsets([hw] * n)
    dn = S.GroupNormDesc(n=n, hw=hw, c=c, groups=8, dtype=S.SGPRS_BF16, eps=1e-5)
    dl = S.LinearDesc(m=n * hw, n=3 * c, k=c, dtype=S.SGPRS_BF16)
    da = S.AttentionDesc(n_seqs=n, total_q=n * hw, total_kv=n * hw, max_q=hw, max_kv=hw, heads=heads, kv_heads=heads, head_dim=c // heads, dtype=S.SGPRS_BF16,
                         ldq=3 * c, ldk=3 * c, ldv=3 * c)
    need = [S.sgprs_group_norm_workspace(dn, CUS), S.sgprs_linear_workspace(dl, CUS), S.sgprs_attention_workspace(da, CUS)]
    ws = torch.empty(max(need + [16]), dtype=torch.uint8, device="cuda")

    def block():
        S.sgprs_group_norm(dn, ptr(x), None, None, None, ptr(norm), ptr(ws), need[0], pool, 0)
        S.sgprs_linear(dl, ptr(norm), ptr(wq), None, None, ptr(qkv), ptr(ws), need[1], pool, 0)
        S.sgprs_attention(da, ptr(qkv), ptr(qkv) + 2 * c, ptr(qkv) + 4 * c, ptr(off), ptr(off), ptr(out), ptr(ws), need[2], pool, 0)

    torch.cuda.synchronize()
    block()
    pool.sync()
    stream = torch.cuda.ExternalStream(pool.stream(0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        graph.capture_begin()
        block()
        graph.capture_end()
    for i in range(4):
        xi = torch.randn(n * hw, c, generator=gen(30 + i)).bfloat16()
        x.copy_(xi)
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        block()
        pool.sync()
        assert bool(torch.isfinite(out).all()) and float(out.float().abs().max()) > 0
        assert torch.equal(replayed, out), i
