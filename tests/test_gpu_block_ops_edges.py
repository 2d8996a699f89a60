"""GPU parity of the attention-block operators with 64-bit definitions at the edges of what their descriptors allow:
operands at the ends of fp32's range, more rows, images and sequences than a launch or a search step takes at once."""
import time

import pytest
import scipy.special
import torch

import paper_2406_09425_amd as S
import block_ops_util as ref
from test_gpu_block_ops import CUS, DT, gen, offsets, pools, ptr, run_attention, run_norm  # noqa: F401 (pools is a fixture)

pytestmark = pytest.mark.gpu


# ---- linear --------------------------------------------------------------------------------------
def linear_plain(pools, xh, wh, cus=CUS, act=0):
    """x w^T of dense tensors, no bias, no residual."""
    (m, k), n = xh.shape, wh.shape[0]
    x, w = xh.cuda(), wh.cuda()
    y = torch.full((m, n), float("nan"), dtype=xh.dtype, device="cuda")
    d = S.LinearDesc(m=m, n=n, k=k, dtype=S.SGPRS_F32 if xh.dtype == torch.float32 else S.SGPRS_BF16, act=act)
    ws_bytes = S.sgprs_linear_workspace(d, cus)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools(cus)
    S.sgprs_linear(d, ptr(x), ptr(w), None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    return y.cpu()


@pytest.mark.parametrize("small,large", [(116, 112), (122, 118), (126, 122), (135, 123), (140, 100), (138, 0), (66, -72)])
@pytest.mark.parametrize("m,n,k,cus", [(20, 140, 96, 256), (2100, 700, 96, 256), (2050, 570, 101, 256), (600, 700, 40, 8)])
@pytest.mark.parametrize("swap", [False, True])
def test_linear_fp32_operands_near_the_ends_of_the_range(pools, small, large, m, n, k, cus, swap):
    """Small and subnormal values against ordinary and large ones: every operand counts with its 24 bits.  Beside the
    usual bound, each product (in up to six parts) and each addition may round by half of fp32's smallest number."""
    g = gen(small)
    x, w = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g)
    (w if swap else x).mul_(2.0 ** -small)
    (x if swap else w).mul_(2.0 ** large)
    x[5] = 0.0
    x[6] = 0.0
    x[6, 3] = 2.0 ** -149
    want, bound = ref.linear(x, w, None, None, 0, 0)
    ref.assert_within(linear_plain(pools, x, w, cus), want, bound + 8 * k * 2.0 ** -149, f"2^-{small} against 2^{large}, {m}x{k}->{n}")


def test_linear_of_the_largest_number_of_rows_is_refused(pools):
    """More tiles than a launch takes, counted without wrapping; nothing of the tensors is touched."""
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    y = torch.full((64,), 777.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for m in (2 ** 31 - 1, 2 ** 31 - 20):
        with pytest.raises(S.SgprsError) as e:
            S.sgprs_linear(S.LinearDesc(m=m, n=1, k=1, dtype=S.SGPRS_BF16), ptr(x), ptr(x), None, None, ptr(y), None, 0, pools(), 0)
        assert e.value.status == -5
    assert bool((y == 777.0).all())


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 49, 64, 8), (1, 12544, 64, 32), (2, 9000, 512, 4), (50, 1, 512, 1)], ids=str)
def test_group_norms_of_tiny_values_without_eps(pools, name, shape):
    """Deviations of 2^-66: their squares are subnormal, with 16 bits and more of those that count, so that a variance is
    off by 2^-17 and the result by 2^-18; the bound's other parts come on top."""
    n, hw, c, groups = shape
    dt, tdt = DT[name]
    x = (torch.randn(n * hw, c, generator=gen(8)) * 2.0 ** -66).to(tdt)
    xd, y = x.cuda(), torch.zeros(n * hw, c, dtype=tdt, device="cuda")
    d = S.GroupNormDesc(n=n, hw=hw, c=c, groups=groups, dtype=dt, eps=0.0)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_group_norm(d, ptr(xd), None, None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    want, bound = ref.group_norm(x, None, None, None, n, hw, groups, 0.0, 0)
    ref.assert_within(y, want, bound + 2.0 ** -16 * want.abs(), f"tiny values {shape}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("shape,cus", [((1, 12544, 256, 32), 256), ((2, 6000, 96, 3), 40), ((1, 3000, 1030, 5), 8), ((3, 4100, 64, 64), 128), ((1, 700, 4096, 4096), 256)], ids=str)
@pytest.mark.parametrize("inplace", [None, "x", "residual"])
def test_group_norms_of_many_chunks(pools, name, shape, cus, inplace):
    """Chunks that a launch of its own merges; odd numbers of groups and channels, slices of a row."""
    run_norm(pools, name, *shape, act=3, res=True, cus=cus, seed=4, inplace=inplace)


def test_group_norm_of_many_chunks_with_a_mean_far_from_zero(pools):
    n, hw, c, groups = 1, 20000, 96, 4
    run_norm(pools, "f32", n, hw, c, groups, x=torch.randn(n * hw, c, generator=gen(1)) + 1000.0, seed=1)


def test_group_norm_takes_time_by_its_positions(pools):
    """600000 positions are 75000 chunks: as long as a few copies of the tensor, not as chunks that each merge all others."""
    hw, c = 600000, 2048
    x = torch.empty(hw, c, dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.zeros_like(x)
    d = S.GroupNormDesc(n=1, hw=hw, c=c, groups=8, dtype=S.SGPRS_BF16, eps=1e-5)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()

    def seconds(call):
        call()
        pool.sync()
        torch.cuda.synchronize()
        begin = time.perf_counter()
        call()
        pool.sync()
        torch.cuda.synchronize()
        return time.perf_counter() - begin

    copy = seconds(lambda: y.copy_(x))
    norm = seconds(lambda: S.sgprs_group_norm(d, ptr(x), None, None, None, ptr(y), ptr(ws), ws_bytes, pool, 0))
    assert norm <= 25 * copy, (norm, copy)


def test_group_norm_of_the_largest_number_of_positions(pools):
    hw = 2 ** 31 - 1
    x = torch.empty(hw, 1, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    x += 1.0
    y = torch.zeros_like(x)
    d = S.GroupNormDesc(n=1, hw=hw, c=1, groups=1, dtype=S.SGPRS_BF16, eps=1e-5)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_group_norm(d, ptr(x), None, None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    sums = torch.zeros(2, dtype=torch.float64)
    for at in range(0, hw, 1 << 27):
        part = x[at:at + (1 << 27)].double()
        sums += torch.stack([part.sum(), (part * part).sum()]).cpu()
    mean = sums[0] / hw
    deviation = (sums[1] / hw - mean * mean + 1e-5).sqrt()
    for at in (0, hw // 2, hw - 4096):
        want = (x[at:at + 4096].double().cpu() - mean) / deviation
        assert float((y[at:at + 4096].double().cpu() - want).abs().max()) <= 1.01 * 2.0 ** -8 * float(want.abs().max()) + 1e-4


# ---- attention -----------------------------------------------------------------------------------
def test_attention_of_more_pairs_than_a_join_takes_enqueues_nothing(pools):
    """2^24 (token, head) pairs whose keys are split: the second launch is too large, so the first must not run."""
    n, heads, dim, keys = 1 << 19, 32, 8, 256
    q = torch.zeros(n, heads * dim, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(keys, dim, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(q, 777.0)
    q_offsets = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    kv_offsets = torch.full((n + 1,), keys, dtype=torch.int32, device="cuda")
    kv_offsets[0] = 0
    d = S.AttentionDesc(n_seqs=n, total_q=n, total_kv=keys, max_q=1, max_kv=keys, heads=heads, kv_heads=1, head_dim=dim, dtype=S.SGPRS_BF16)
    ws_bytes = S.sgprs_attention_workspace(d, CUS)
    assert ws_bytes > 0  # keys are split
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    with pytest.raises(S.SgprsError) as e:
        S.sgprs_attention(d, ptr(q), ptr(k), ptr(k), ptr(q_offsets), ptr(kv_offsets), ptr(o), ptr(ws), ws_bytes, pool, 0)
    assert e.value.status == -5
    pool.sync()
    assert bool((o == 777.0).all())


# ---- group norm ----------------------------------------------------------------------------------
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("extra", [8, 9])
def test_layer_norms_of_wide_rows_and_many_tokens(pools, name, extra):
    """Rows just beyond those that a wavefront holds, more of them than a launch has images."""
    dt, tdt = DT[name]
    n, c = 70000, (2048 if name == "f32" else 4096) + extra
    x = torch.empty(n, c, dtype=tdt, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(extra))
    y = torch.zeros_like(x)
    gamma = torch.rand(c, generator=gen(1)) + 0.5
    G = gamma.cuda()
    d = S.GroupNormDesc(n=n, hw=1, c=c, groups=1, dtype=dt, eps=1e-5)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_group_norm(d, ptr(x), ptr(G), None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    for at in (0, 65530, n - 8):
        want, bound = ref.group_norm(x[at:at + 8].cpu(), gamma, None, None, 8, 1, 1, 1e-5, 0)
        ref.assert_within(y[at:at + 8], want, bound, f"rows {at} and on of {n} of {c}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("hw,c,groups", [(1, 16, 4), (3, 9, 3)])
def test_group_norms_of_more_images_than_a_launch_takes(pools, name, hw, c, groups):
    run_norm(pools, name, 131075, hw, c, groups, act=3, res=True, seed=c)


def test_group_norms_of_more_large_images_than_a_launch_takes(pools):
    """Statistics of chunks in the workspace, for each of the launches."""
    n, hw, c, groups = 65537, 257, 256, 1
    d = S.GroupNormDesc(n=n, hw=hw, c=c, groups=groups, dtype=S.SGPRS_BF16, eps=1e-5)
    ws_bytes = S.sgprs_group_norm_workspace(d, CUS)
    assert ws_bytes > 0
    x = torch.empty(n, hw, c, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    y = torch.zeros_like(x)
    ws = torch.full((max(ws_bytes, 16),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    pool = pools()
    S.sgprs_group_norm(d, ptr(x), None, None, None, ptr(y), ptr(ws), ws_bytes, pool, 0)
    pool.sync()
    for at in (0, 65534, 65535, 65536):
        want, bound = ref.group_norm(x[at].cpu(), None, None, None, 1, hw, groups, 1e-5, 0)
        ref.assert_within(y[at], want, bound, f"image {at} of {n}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,kv_lens,heads,dim", [([1], [300], 1, 8), ([1, 1, 1], [300, 2, 129], 1, 72), ([99], [1050], 1, 40), ([35], [1100], 3, 8)], ids=str)
def test_attention_partial_sums_of_odd_numbers_of_rows(pools, name, q_lens, kv_lens, heads, dim):
    """Split keys where tokens, heads and chunks are odd: the vectors of partial sums keep to 16 bytes."""
    run_attention(pools, name, q_lens, kv_lens, heads, 1, dim, True, seed=dim)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [65, 70, 4097, 4200])
@pytest.mark.parametrize("longest,cache", [(2, 1500), (300, 1100)], ids=["tokens", "prompt"])
def test_attention_of_more_sequences_than_a_search_step_looks_at(pools, name, n, longest, cache):
    """64 sequences are looked at at once: two and three steps, with empty sequences, one long one and keys that are split."""
    q_lens = torch.randint(0, 3, (n,), generator=gen(n)).tolist()
    kv_lens = torch.randint(0, 4, (n,), generator=gen(n + 1)).tolist()
    at = n * 2 // 3
    q_lens[at], kv_lens[at] = longest, cache
    run_attention(pools, name, q_lens, kv_lens, 2, 1, 32, True, seed=n, repeat=False)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,kv_lens,heads", [([3001], [3001], 1), ([2500, 1, 129], [2500, 2600, 4000], 2)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_thousands_of_queries(pools, name, q_lens, kv_lens, heads, causal):
    run_attention(pools, name, q_lens, kv_lens, heads, 1, 64, causal, seed=heads)


# ---- activations ---------------------------------------------------------------------------------
U = 2.0 ** -24


def activation_by_scipy(z, act):
    """z times the distribution function of a Gaussian or the logistic one, by functions that do not cancel."""
    f = scipy.special.ndtr if act == S.SGPRS_ACT_GELU else scipy.special.expit
    return z.double() * torch.from_numpy(f(z.double().numpy()))


@pytest.mark.parametrize("act", [S.SGPRS_ACT_GELU, S.SGPRS_ACT_SILU], ids=["gelu", "silu"])
@pytest.mark.parametrize("m", [24, 5000])
def test_fp32_activations_keep_their_digits_down_the_negative_side(pools, act, m):
    """x w^T with one input and w = 1 is x itself, so what is off is the activation.  SiLU: an exponential (2 ulp), a sum, a
    product and a quotient, 4 u a step at most.  GELU: its argument is off by 1.5 u, of which erfc makes 2 t^2 + 1 = z^2 + 1
    times as much, and erfc itself by 16 ulp at most.  Results below 2^-126 are multiples of 2^-149, the exponential's too."""
    z = torch.linspace(-110.0 if act == S.SGPRS_ACT_SILU else -14.0, 12.0, m)[:, None]
    want = activation_by_scipy(z, act)
    relative = 16 * U if act == S.SGPRS_ACT_SILU else 2 * (z.double() ** 2 + 1) * U + 34 * U
    ref.assert_within(linear_plain(pools, z, torch.ones(1, 1), act=act), want, relative * want.abs() + (z.double().abs() + 2) * 2.0 ** -149, f"activation {act}")


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("act", [S.SGPRS_ACT_NONE, S.SGPRS_ACT_RELU, S.SGPRS_ACT_GELU, S.SGPRS_ACT_SILU], ids=["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m", [8, 300])
def test_activations_of_what_is_not_finite(pools, name, act, m):
    """As the formulas say, for both types: GELU and SiLU of -infinity are -infinity times 0."""
    z = torch.tensor([float("-inf"), float("inf"), float("nan"), -3e38, 3e38, 0.0, -1.0]).repeat(m)[:m, None].to(DT[name][1])
    w = torch.ones(3, 1, dtype=z.dtype)
    want, bound = ref.linear(z[:, :1].contiguous(), w, None, None, act, 0)
    ref.assert_within(linear_plain(pools, z[:, :1].contiguous(), w, act=act), want, bound, f"activation {act} {name}")
