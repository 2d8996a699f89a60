"""The operators of an attention block on a channels-last feature map, as timed cases.

A network with attention behind (or instead of) convolutions runs, stage by stage on a partition:

  linear      y = act(x w^T + bias) + residual: token- or pixel-wise products, one row to many
  group_norm  y = act(norm(x) gamma + beta + residual), channels last; with one pixel per image and
              one group it is the layer norm of a token
  attention   softmax(q k^T) v over packed sequences of different lengths, grouped heads, causal or
              not; one query per sequence against a long cache is the serving form

Each case is one pass through one operator on the whole GPU; `draw` gives more of the same ranges.
`own` chooses between the plain forms (elementary torch operations in fp32, rounded once at the end)
and the library's kernels.
"""
import math
import weakref

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}
_CUS = 256


def listed():
    return [
        # the classifier of one frame: the smallest product, all latency
        dict(name="linear_bf16_1x512_1000", kind="linear", dtype="bf16", m=1, k=512, n=1000, act="none", bias=True, res=False, pad=0),
        # one decoded token for each of 24 streams through an up-projection: bound by the weights
        dict(name="linear_bf16_24x4096_4096", kind="linear", dtype="bf16", m=24, k=4096, n=4096, act="silu", bias=False, res=False, pad=0),
        # MLP of 64 images of 14 x 14 tokens
        dict(name="linear_bf16_12544x512_2048", kind="linear", dtype="bf16", m=12544, k=512, n=2048, act="gelu", bias=True, res=False, pad=0),
        # output projection with the skip connection in single precision; ragged rows, columns and strides
        dict(name="linear_f32_3137x517_509", kind="linear", dtype="f32", m=3137, k=517, n=509, act="none", bias=True, res=True, pad=3),
        # a batch of long prompts: the largest product
        dict(name="linear_bf16_16384x4096_4096", kind="linear", dtype="bf16", m=16384, k=4096, n=4096, act="none", bias=True, res=True, pad=0),
        # the last feature map of one frame: the smallest norm, all latency
        dict(name="group_norm_bf16_1x49x512", kind="group_norm", dtype="bf16", n=1, hw=49, c=512, groups=32, act="relu", res=False, pad=0),
        # layer norm of 64 images of 14 x 14 tokens
        dict(name="group_norm_bf16_12544x1x512", kind="group_norm", dtype="bf16", n=12544, hw=1, c=512, groups=1, act="none", res=False, pad=0),
        # end of a residual block of a 64-image batch on the first layers' maps: the largest norm
        dict(name="group_norm_bf16_64x12544x64", kind="group_norm", dtype="bf16", n=64, hw=12544, c=64, groups=32, act="silu", res=True, pad=0),
        # 64 images of 14 x 14 tokens attending to themselves
        dict(name="attention_bf16_64x196_8x64", kind="attention", dtype="bf16", q="196," * 63 + "196", kv="", heads=8, kv_heads=8, dim=64, causal=False, pad=0),
        # one token for each of 16 streams against caches of very different lengths
        dict(name="attention_bf16_decode16_32x128", kind="attention", dtype="bf16", q="1," * 15 + "1",
             kv="8192,1,77,4096,513,2048,6001,128,1024,3333,64,7000,15,2500,900,5120", heads=32, kv_heads=8, dim=128, causal=True, pad=0),
        # ragged prompts in single precision, an empty one among them
        dict(name="attention_f32_prompts_6x72", kind="attention", dtype="f32", q="333,1,0,700,95,512", kv="", heads=6, kv_heads=2, dim=72, causal=True, pad=0),
        # packed prompts of different lengths: the largest attention
        dict(name="attention_bf16_prompts_32x128", kind="attention", dtype="bf16", q="4096,2500,3777,1300", kv="", heads=32, kv_heads=8, dim=128, causal=True, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _near(rng, v):
    """v, or a size beside it that is no multiple of anything."""
    return v if rng.random() < 0.5 else max(1, v + rng.randint(-7, 7))


def draw(rng):
    kind = rng.choice(["linear", "group_norm", "attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if kind == "linear":
        while True:
            case = dict(kind=kind, dtype=dtype, m=_log_int(rng, 1, 16384), k=_near(rng, 16 * _log_int(rng, 4, 512)),
                        n=_near(rng, 16 * _log_int(rng, 4, 512)), act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.7,
                        res=rng.random() < 0.4, pad=pad)
            if case["k"] != 3072 and case["n"] != 3072 and work(case)["flops"] <= (2e11 if dtype == "bf16" else 2e10):
                return case
    if kind == "group_norm":
        act, res = rng.choice(["none", "relu", "silu"]), rng.random() < 0.3
        if rng.random() < 0.25:  # layer norm of tokens
            return dict(kind=kind, dtype=dtype, n=_log_int(rng, 1, 16384), hw=1, c=_near(rng, 32 * rng.randint(2, 32)), groups=1, act=act, res=res, pad=pad)
        groups = rng.choice([1, 4, 8, 16, 32])
        c = groups * _log_int(rng, max(1, 32 // groups), 512 // groups)
        hw = rng.randint(5, 112) * rng.randint(5, 112)
        return dict(kind=kind, dtype=dtype, n=_log_int(rng, 1, max(1, min(128, int(4e7 / (hw * c))))), hw=hw, c=c, groups=groups, act=act, res=res, pad=pad)
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4])
    seqs = _log_int(rng, 1, 32)
    if rng.random() < 0.4:  # a token or a few against a cache
        kv = [_log_int(rng, 1, 8192) for _ in range(seqs)]
        q = [min(v, rng.choice([1, 1, 1, 2, 5])) for v in kv]
    else:
        most = min(4096 if dtype == "bf16" else 1024, int(math.sqrt((1e9 if dtype == "bf16" else 2e8) / (seqs * heads))))
        q = [_log_int(rng, max(1, most // 8), max(1, most)) for _ in range(seqs)]
        kv = []
    return dict(kind=kind, dtype=dtype, q=",".join(map(str, q)), kv=",".join(map(str, kv)), heads=heads, kv_heads=kv_heads, dim=dim,
                causal=rng.random() < 0.6, pad=0 if pad == 3 else pad)


def _lens(case):
    q = [int(v) for v in case["q"].split(",")]
    return q, [int(v) for v in case["kv"].split(",")] if case["kv"] else q


# ---- inputs --------------------------------------------------------------------------------------
def _inputs(case, seed):
    """The tensors of a pass. `pad`: elements between the rows of the activations, as where they are part of a wider tensor."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    tdt, pad = _TORCH[case["dtype"]], case["pad"]

    def rows(m, c, std=1.0, mean=0.0):
        return (torch.randn((m, c + pad), generator=g, device="cuda") * std + mean).to(tdt)[:, :c]

    if case["kind"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(x=rows(m, k), w=(torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)).to(tdt),
                    bias=torch.randn(n, generator=g, device="cuda") * 0.1 if case["bias"] else None, res=rows(m, n) if case["res"] else None)
    if case["kind"] == "group_norm":
        n, hw, c = case["n"], case["hw"], case["c"]
        means = torch.randn(c + pad, generator=g, device="cuda")  # channels of a network differ in their means
        return dict(x=rows(n * hw, c, 1.5, means),
                    gamma=torch.rand(c, generator=g, device="cuda") + 0.5, beta=torch.randn(c, generator=g, device="cuda") * 0.1,
                    res=rows(n * hw, c) if case["res"] else None)
    q, kv = _lens(case)
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    offsets = [torch.tensor([0] + v, device="cuda").cumsum(0).to(torch.int32) for v in (q, kv)]
    return dict(q=rows(sum(q), h * d, 1.5), k=rows(sum(kv), hk * d), v=rows(sum(kv), hk * d), q_offsets=offsets[0], kv_offsets=offsets[1],
                max_q=max(q), max_kv=max(kv))


_pools = weakref.WeakValueDictionary()


def _pool():
    import paper_2406_09425_amd as S
    p = _pools.get(_CUS)
    if p is None:
        p = _pools[_CUS] = S.Pool(1, _CUS)
    return p


def _handles(case, st):
    """What a program of the library keeps beside its tensors: the pool, the operator's descriptor, its output and its workspace."""
    import paper_2406_09425_amd as S
    dt = dict(bf16=S.SGPRS_BF16, f32=S.SGPRS_F32)[case["dtype"]]
    kind = case["kind"]
    if kind != "attention":
        act = dict(none=S.SGPRS_ACT_NONE, relu=S.SGPRS_ACT_RELU, gelu=S.SGPRS_ACT_GELU, silu=S.SGPRS_ACT_SILU)[case["act"]]
        ldr = st["res"].stride(0) if case["res"] else 0
    if kind == "linear":
        desc = S.LinearDesc(m=case["m"], n=case["n"], k=case["k"], dtype=dt, act=act, ldx=st["x"].stride(0), ldr=ldr)
        out, ws_bytes = torch.empty((case["m"], case["n"]), device="cuda", dtype=_TORCH[case["dtype"]]), S.sgprs_linear_workspace(desc, _CUS)
    elif kind == "group_norm":
        desc = S.GroupNormDesc(n=case["n"], hw=case["hw"], c=case["c"], groups=case["groups"], dtype=dt, act=act, eps=1e-5,
                               ldx=st["x"].stride(0), ldr=ldr)
        out, ws_bytes = torch.empty((case["n"] * case["hw"], case["c"]), device="cuda", dtype=_TORCH[case["dtype"]]), S.sgprs_group_norm_workspace(desc, _CUS)
    else:
        d = case["dim"]
        desc = S.AttentionDesc(n_seqs=st["q_offsets"].numel() - 1, total_q=st["q"].shape[0], total_kv=st["k"].shape[0], max_q=st["max_q"],
                               max_kv=st["max_kv"], heads=case["heads"], kv_heads=case["kv_heads"], head_dim=d, dtype=dt, causal=int(case["causal"]),
                               ldq=st["q"].stride(0), ldk=st["k"].stride(0), ldv=st["v"].stride(0))
        out, ws_bytes = torch.empty((st["q"].shape[0], case["heads"] * d), device="cuda", dtype=_TORCH[case["dtype"]]), S.sgprs_attention_workspace(desc, _CUS)
    return dict(desc=desc, out=out, ws=torch.empty(max(ws_bytes, 16), device="cuda", dtype=torch.uint8), ws_bytes=ws_bytes, pool=_pool())


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    if own:
        st.update(_handles(case, st))
        torch.cuda.synchronize()  # the partitions' streams are not ordered after torch's
    return st


# ---- one pass ------------------------------------------------------------------------------------
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_linear(st, case):
    z = st["x"].float() @ st["w"].float().t()
    if case["bias"]:
        z = z + st["bias"]
    z = _act(z, case["act"])
    if case["res"]:
        z = z + st["res"].float()
    return z.to(st["x"].dtype)


def _plain_group_norm(st, case):
    n, hw, c, groups = (case[f] for f in ("n", "hw", "c", "groups"))
    x = st["x"].float().reshape(n, hw, groups, c // groups)
    x = x - x.mean((1, 3), keepdim=True)
    x = x * torch.rsqrt((x * x).mean((1, 3), keepdim=True) + 1e-5)
    z = x.reshape(n * hw, c) * st["gamma"] + st["beta"]
    if case["res"]:
        z = z + st["res"].float()
    return _act(z, case["act"]).to(st["x"].dtype)


def _plain_attention(st, case):
    """All sequences at once, each padded to the longest."""
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    qo, ko, lq, lk = st["q_offsets"].long(), st["kv_offsets"].long(), st["max_q"], st["max_kv"]
    nq, nk = qo[1:] - qo[:-1], ko[1:] - ko[:-1]
    i, j = torch.arange(lq, device="cuda"), torch.arange(lk, device="cuda")
    at_q = (qo[:-1, None] + i).clamp_max(st["q"].shape[0] - 1)
    at_k = (ko[:-1, None] + j).clamp_max(st["k"].shape[0] - 1)
    s = len(nq)
    q = st["q"].float()[at_q].reshape(s, lq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(s * hk, (h // hk) * lq, d)
    k = st["k"].float()[at_k].reshape(s, lk, hk, d).permute(0, 2, 3, 1).reshape(s * hk, d, lk)
    v = st["v"].float()[at_k].reshape(s, lk, hk, d).transpose(1, 2).reshape(s * hk, lk, d)
    seen = (j < nk[:, None])[:, None, :].expand(s, lq, lk)
    if case["causal"]:
        seen = seen & (j <= (i + (nk - nq)[:, None])[:, :, None])
    p = torch.bmm(q, k).mul_(1 / math.sqrt(d)).reshape(s, h, lq, lk).masked_fill_(~seen[:, None], -math.inf)
    top = p.amax(3, keepdim=True).clamp_min(-1e30)  # a row without a key has no largest score
    p = p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.bmm(p.reshape(s * hk, (h // hk) * lq, lk), v).reshape(s, h, lq, d) / torch.where(total > 0, total, 1.0)
    return o.transpose(1, 2)[i < nq[:, None]].reshape(-1, h * d).to(st["q"].dtype)


_PLAIN = dict(linear=_plain_linear, group_norm=_plain_group_norm, attention=_plain_attention)


def _run_linear(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_linear(st["desc"], st["x"].data_ptr(), st["w"].data_ptr(), st["bias"].data_ptr() if case["bias"] else None,
                   st["res"].data_ptr() if case["res"] else None, st["out"].data_ptr(), st["ws"].data_ptr(), st["ws_bytes"], st["pool"], 0)


def _run_group_norm(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_group_norm(st["desc"], st["x"].data_ptr(), st["gamma"].data_ptr(), st["beta"].data_ptr(),
                       st["res"].data_ptr() if case["res"] else None, st["out"].data_ptr(), st["ws"].data_ptr(), st["ws_bytes"], st["pool"], 0)


def _run_attention(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_attention(st["desc"], st["q"].data_ptr(), st["k"].data_ptr(), st["v"].data_ptr(), st["q_offsets"].data_ptr(),
                      st["kv_offsets"].data_ptr(), st["out"].data_ptr(), st["ws"].data_ptr(), st["ws_bytes"], st["pool"], 0)


_RUN = dict(linear=_run_linear, group_norm=_run_group_norm, attention=_run_attention)


def run(state):
    case = state["case"]
    if not own:
        return _PLAIN[case["kind"]](state, case)
    _RUN[case["kind"]](state, case)
    return state["out"]


# ---- what a pass cannot do without ---------------------------------------------------------------
def work(case):
    kind, es = case["kind"], _ES[case["dtype"]]
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=(m * k + n * k + m * n * (2 if case["res"] else 1)) * es + (4 * n if case["bias"] else 0), flops=2.0 * m * n * k)
    if kind == "group_norm":
        size = case["n"] * case["hw"] * case["c"]
        return dict(bytes=size * es * (3 if case["res"] else 2) + 8 * case["c"], flops=6.0 * size)
    q, kv = _lens(case)
    pairs = 0
    for a, b in zip(q, kv):
        if not case["causal"]:
            pairs += a * b
        else:  # the last m rows see b - m + 1 to b keys, any rows before them none
            m = min(a, b)
            pairs += m * (b - m + 1 + b) // 2
    h, hk, d = case["heads"], case["kv_heads"], case["dim"]
    return dict(bytes=2 * (sum(q) * h + sum(kv) * hk) * d * es, flops=4.0 * pairs * h * d)


# ---- the definitions in 64 bits ------------------------------------------------------------------
def exact(case, seed):
    t = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    activation = dict(none=lambda z: z, relu=lambda z: torch.where(z > 0, z, 0.0), silu=lambda z: z * torch.sigmoid(z),
                      gelu=lambda z: z * torch.special.ndtr(z)).get(case.get("act"))
    if case["kind"] == "linear":
        y = torch.matmul(t["x"], t["w"].t().contiguous())
        y = activation(y if t["bias"] is None else y + t["bias"])
        return y if t["res"] is None else y + t["res"]
    if case["kind"] == "group_norm":
        per = case["c"] // case["groups"]
        x = t["x"].reshape(case["n"], case["hw"], case["groups"], per)
        var, mean = torch.var_mean(x, dim=(1, 3), correction=0, keepdim=True)
        y = ((x - mean) / (var + 1e-5).sqrt()).reshape(-1, case["c"]) * t["gamma"] + t["beta"]
        return activation(y if t["res"] is None else y + t["res"])
    d, group, out = case["dim"], case["heads"] // case["kv_heads"], torch.zeros_like(t["q"])
    at_q = at_k = 0
    for nq, nk in zip(*_lens(case)):  # one sequence and one head at a time
        for head in range(case["heads"] if nq and nk else 0):
            cols, kv_cols = slice(head * d, head * d + d), slice(head // group * d, head // group * d + d)
            score = t["q"][at_q:at_q + nq, cols] @ t["k"][at_k:at_k + nk, kv_cols].t().contiguous() / math.sqrt(d)
            if case["causal"]:
                ahead = torch.ones((nq, nk), dtype=torch.bool, device="cuda").triu(nk - nq + 1)
                score = score.masked_fill(ahead, -math.inf)
            p = torch.softmax(score, 1).nan_to_num(0.0) if nq > nk else torch.softmax(score, 1)
            out[at_q:at_q + nq, cols] = p @ t["v"][at_k:at_k + nk, kv_cols]
        at_q, at_k = at_q + nq, at_k + nk
    return out
