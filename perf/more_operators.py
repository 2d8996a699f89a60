"""The operators of a decoding step with 8-bit weights and a paged cache, as timed cases.

A decoder that runs beside the convolutional networks goes, for each new token (or batch of prompts), through

  rms_norm         h = x + residual, y = h gamma / sqrt(mean h^2 + eps), as 8-bit integers with a scale for each row or in the type
  quantize_i8      rows to 8-bit integers with a scale each: weights once, activations that no norm precedes
  linear_i8        y = act(sx sw sum x w + bias) + residual, 8-bit integers summed exactly
  paged_append     new keys and values to their places in a cache of pages
  paged_attention  one new token of each sequence against its pages; with a window, the window and the first few tokens

Each case is one pass through one operator on the whole GPU; `draw` gives more of the same ranges.
`own` chooses between the plain forms (elementary torch operations) and the library's kernels.  8-bit results are whole
numbers that the definition fixes (nearest, ties to even), returned beside the scales of their rows.
"""
import math
import weakref

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4}
_CUS = 256
_EPS = 1e-6


def listed():
    return [
        # one decoded token into an attention block: the smallest norm, all latency
        dict(name="rms_norm_i8_bf16_1x4096", kind="rms_norm", dtype="bf16", out="i8", m=1, c=4096, res=True, pad=0),
        # a batch of long prompts: the largest norm
        dict(name="rms_norm_i8_bf16_16384x4096", kind="rms_norm", dtype="bf16", out="i8", m=16384, c=4096, res=True, pad=0),
        # attention results of 24 streams on their way to the output projection
        dict(name="quantize_i8_bf16_24x4096", kind="quantize_i8", dtype="bf16", m=24, c=4096, pad=0),
        # a weight matrix in single precision; ragged rows and strides
        dict(name="quantize_i8_f32_4093x4099", kind="quantize_i8", dtype="f32", m=4093, c=4099, pad=3),
        # one decoded token for each of 24 streams through an up-projection: bound by the weights
        dict(name="linear_i8_bf16_24x4096_4096", kind="linear_i8", dtype="bf16", m=24, k=4096, n=4096, act="silu", bias=False, res=False, pad=0),
        # output projection with the skip connection in single precision; ragged rows, columns and strides
        dict(name="linear_i8_f32_3137x517_509", kind="linear_i8", dtype="f32", m=3137, k=517, n=509, act="none", bias=True, res=True, pad=3),
        # a batch of long prompts: the largest product
        dict(name="linear_i8_bf16_16384x4096_4096", kind="linear_i8", dtype="bf16", m=16384, k=4096, n=4096, act="none", bias=True, res=True, pad=0),
        # one new token of each of 24 streams: the smallest write
        dict(name="paged_append_bf16_24_8x128", kind="paged_append", dtype="bf16", new="1," * 23 + "1", kv="64,1,77,96,113,48,101,128,24,133,64,70,15,250,90,51,33,16,17,200,5,2,31,160",
             kv_heads=8, dim=128, page=16, pad=0),
        # the keys and values of four prompts
        dict(name="paged_append_bf16_prompts_8x128", kind="paged_append", dtype="bf16", new="4096,2500,3777,1300", kv="4096,2600,3777,1300", kv_heads=8, dim=128, page=16, pad=0),
        # three short chats, one of which has just ended: all latency
        dict(name="paged_attention_bf16_3_8x64", kind="paged_attention", dtype="bf16", kv="333,0,700", heads=8, kv_heads=8, dim=64, page=16, window=0, sinks=0, pad=0),
        # one token for each of 16 streams against caches of very different lengths
        dict(name="paged_attention_bf16_16_32x128", kind="paged_attention", dtype="bf16", kv="32768,1,77,4096,513,2048,6001,128,1024,3333,64,7000,15,2500,900,5120",
             heads=32, kv_heads=8, dim=128, page=16, window=0, sinks=0, pad=0),
        # long streams in single precision that see a window and their first tokens; pages that end inside a tile
        dict(name="paged_attention_f32_5_6x72_window", kind="paged_attention", dtype="f32", kv="40000,2000,65000,31,20001", heads=6, kv_heads=2, dim=72, page=48,
             window=12000, sinks=4, pad=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _near(rng, v):
    """v, or a size beside it that is no multiple of anything."""
    return v if rng.random() < 0.5 else max(1, v + rng.randint(-7, 7))


def draw(rng):
    kind = rng.choice(["rms_norm", "quantize_i8", "linear_i8", "linear_i8", "paged_append", "paged_attention", "paged_attention"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 16, 3])
    if kind in ("rms_norm", "quantize_i8"):
        c = _near(rng, 16 * _log_int(rng, 4, 1024))
        case = dict(kind=kind, dtype=dtype, m=_log_int(rng, 1, max(1, min(16384, (1 << 25) // c))), c=c, pad=pad)
        return dict(case, out=rng.choice(["i8", "i8", "same"]), res=rng.random() < 0.6) if kind == "rms_norm" else case
    if kind == "linear_i8":
        while True:
            case = dict(kind=kind, dtype=dtype, m=_log_int(rng, 1, 16384), k=_near(rng, 16 * _log_int(rng, 4, 512)), n=_near(rng, 16 * _log_int(rng, 4, 512)),
                        act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.random() < 0.7, res=rng.random() < 0.4, pad=pad)
            if work(case)["flops"] <= 4e11:
                return case
    dim = rng.choice([32, 64, 64, 72, 96, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    page = rng.choice([1, 7, 16, 16, 32, 48, 64, 128, 256])
    pad = 0 if pad == 3 else pad
    seqs = _log_int(rng, 1, 48)
    most = max(16, min(65536, int((1.2e8 if kind == "paged_attention" else 2.4e7) / (seqs * kv_heads * dim * _ES[dtype]))))
    kv = [_log_int(rng, 1, most) - (rng.random() < 0.05) for _ in range(seqs)]
    kv[rng.randrange(seqs)] = max(1, most // rng.randint(1, 8))
    case = dict(kind=kind, dtype=dtype, kv=",".join(map(str, kv)), kv_heads=kv_heads, dim=dim, page=page, pad=pad)
    if kind == "paged_append":
        one = rng.random() < 0.5
        return dict(case, new=",".join(str(1 if one and v else rng.randint(min(1, v), v)) for v in kv))
    window = rng.choice([0, 0, _log_int(rng, 1, 16384)])
    return dict(case, heads=kv_heads * rng.choice([1, 2, 4, 8]), window=window, sinks=rng.choice([0, 1, 4, 20]) if window else 0)


def _ints(text):
    return [int(v) for v in text.split(",")]


# ---- inputs --------------------------------------------------------------------------------------
def _rows_i8(g, m, c, pad):
    """Rows as quantize_i8 leaves them: normal values, the largest of a row at 127; `pad` bytes between rows."""
    x = torch.randn((m, c + pad), generator=g, device="cuda")
    most = x[:, :c].abs().amax(1)
    return (x * (127 / most)[:, None]).round_().clamp_(-127, 127).to(torch.int8)[:, :c], most / 127


def _inputs(case, seed):
    """The tensors of a pass. `pad`: elements between the rows of the activations, as where they are part of a wider tensor."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, tdt, pad = case["kind"], _TORCH[case["dtype"]], case["pad"]

    def rows(m, c, std=1.0):
        return (torch.randn((m, c + pad), generator=g, device="cuda") * std).to(tdt)[:, :c]

    if kind in ("rms_norm", "quantize_i8"):
        m, c = case["m"], case["c"]
        st = dict(x=rows(m, c, 2.0))
        if kind == "rms_norm":  # the stream of a deep network, and what a block adds to it
            st.update(residual=rows(m, c) if case["res"] else None, gamma=torch.rand(c, generator=g, device="cuda") + 0.5)
        return st
    if kind == "linear_i8":
        m, n, k = case["m"], case["n"], case["k"]
        x, sx = _rows_i8(g, m, k, pad)
        w, sw = _rows_i8(g, n, k, 0)
        return dict(x=x, x_scales=sx, w=w, w_scales=sw / math.sqrt(k), bias=torch.randn(n, generator=g, device="cuda") * 0.1 if case["bias"] else None,
                    residual=rows(m, n) if case["res"] else None)
    # a cache some of whose pages belong to others; a sequence's pages lie anywhere, and its table ends in entries without a page
    kv, page, hk, d = _ints(case["kv"]), case["page"], case["kv_heads"], case["dim"]
    used = [-(-v // page) for v in kv]
    n_pages, width = sum(used) + max(2, sum(used) // 8), max(max(used), 1) + 1
    places = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    col, of = torch.arange(width, device="cuda"), torch.tensor(used, device="cuda")
    at = (of.cumsum(0) - of)[:, None] + col
    st = dict(table=torch.where(col < of[:, None], places[at.clamp_max(n_pages - 1)], -1).to(torch.int32).contiguous(),
              kv_lens=torch.tensor(kv, device="cuda", dtype=torch.int32))
    cache = [(torch.randn((n_pages, page, hk, d), generator=g, device="cuda")).to(tdt) for _ in range(2)]
    st.update(k_cache=cache[0], v_cache=cache[1])
    if kind == "paged_append":
        new = _ints(case["new"])
        st.update(k=rows(sum(new), hk * d), v=rows(sum(new), hk * d))
        if max(new) > 1 or min(new) < 1:
            st.update(offsets=torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32))
        return st
    return dict(st, q=rows(len(kv), case["heads"] * d, 1.5))


_pools = weakref.WeakValueDictionary()


def _pool():
    import paper_2406_09425_amd as S
    p = _pools.get(_CUS)
    if p is None:
        p = _pools[_CUS] = S.Pool(1, _CUS)
    return p


def _handles(case, st):
    """What a program of the library keeps beside its tensors: the pool, the operator's descriptor, its outputs and its workspace."""
    import paper_2406_09425_amd as S
    dt, kind = dict(bf16=S.SGPRS_BF16, f32=S.SGPRS_F32)[case["dtype"]], case["kind"]
    tdt = _TORCH[case["dtype"]]
    new = dict(pool=_pool(), ws=None, ws_bytes=0)

    def empty(m, c, dtype=tdt):
        return torch.empty((m, c), device="cuda", dtype=dtype)

    def workspace(need):
        new.update(ws=torch.empty(max(need, 16), device="cuda", dtype=torch.uint8), ws_bytes=need)

    if kind == "rms_norm":
        i8 = case["out"] == "i8"
        new.update(desc=S.RmsNormDesc(m=case["m"], c=case["c"], dtype=dt, out_dtype=S.SGPRS_I8 if i8 else dt, eps=_EPS, ldx=st["x"].stride(0),
                                      ldr=st["residual"].stride(0) if case["res"] else 0),
                   sum=empty(case["m"], case["c"]) if case["res"] else None, y=empty(case["m"], case["c"], torch.int8 if i8 else tdt),
                   scales=torch.empty(case["m"], device="cuda") if i8 else None)
    elif kind == "quantize_i8":
        new.update(desc=S.QuantizeDesc(m=case["m"], c=case["c"], dtype=dt, ldx=st["x"].stride(0)), y=empty(case["m"], case["c"], torch.int8),
                   scales=torch.empty(case["m"], device="cuda"))
    elif kind == "linear_i8":
        act = dict(none=S.SGPRS_ACT_NONE, relu=S.SGPRS_ACT_RELU, gelu=S.SGPRS_ACT_GELU, silu=S.SGPRS_ACT_SILU)[case["act"]]
        new.update(desc=S.LinearI8Desc(m=case["m"], n=case["n"], k=case["k"], dtype=dt, act=act, ldx=st["x"].stride(0),
                                       ldr=st["residual"].stride(0) if case["res"] else 0), y=empty(case["m"], case["n"]))
        workspace(S.sgprs_linear_i8_workspace(new["desc"], _CUS))
    else:
        cache = dict(kv_heads=case["kv_heads"], head_dim=case["dim"], dtype=dt, n_pages=st["k_cache"].shape[0], page_size=case["page"],
                     table_width=st["table"].shape[1], n_seqs=st["table"].shape[0])
        if kind == "paged_append":
            new.update(desc=S.PagedAppendDesc(total=st["k"].shape[0], ldk=st["k"].stride(0), ldv=st["v"].stride(0), **cache))
        else:
            new.update(desc=S.PagedAttentionDesc(heads=case["heads"], window=case["window"], sinks=case["sinks"], ldq=st["q"].stride(0), **cache),
                       y=empty(st["q"].shape[0], case["heads"] * case["dim"]))
            workspace(S.sgprs_paged_attention_workspace(new["desc"], _CUS))
    return new


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


def _plain_rows_i8(t):
    """Nearest integers of 127 t / max|t|, in 64 bits: what lies next to a border between two of them falls to its own side."""
    t = t.double()
    most = t.abs().amax(1, keepdim=True)
    return torch.round(127 * t / torch.where(most > 0, most, 1.0)).to(torch.int8), most[:, 0]


def _plain_rms_norm(st, case):
    h = st["x"] if not case["res"] else (st["x"].float() + st["residual"].float()).to(st["x"].dtype)
    f = h.float()
    r = torch.rsqrt((f * f).mean(1) + _EPS)
    kept = [h] if case["res"] else []
    if case["out"] != "i8":
        return kept + [(f * r[:, None] * st["gamma"]).to(h.dtype)]
    q, most = _plain_rows_i8(h.double() * st["gamma"].double())
    return kept + [q, most.float() * r / 127]


def _plain_quantize_i8(st, case):
    q, most = _plain_rows_i8(st["x"])
    return [q, (most / 127).float()]


def _plain_linear_i8(st, case):
    z = st["x"].float() @ st["w"].float().t() * st["x_scales"][:, None] * st["w_scales"]
    if case["bias"]:
        z = z + st["bias"]
    z = _act(z, case["act"])
    if case["res"]:
        z = z + st["residual"].float()
    return z.to(_TORCH[case["dtype"]])


def _plain_paged_append(st, case):
    total, page = st["k"].shape[0], case["page"]
    token = torch.arange(total, device="cuda")
    if "offsets" in st:
        offsets = st["offsets"].long()
        seq = (token[:, None] >= offsets[None, 1:]).sum(1)
        place = st["kv_lens"].long()[seq] - (offsets[seq + 1] - token)
    else:
        seq, place = token, st["kv_lens"].long() - 1
    row = st["table"].long()[seq, place // page] * page + place % page
    shape = (total, case["kv_heads"], case["dim"])
    st["k_cache"].view(-1, *shape[1:])[row] = st["k"].reshape(shape)
    st["v_cache"].view(-1, *shape[1:])[row] = st["v"].reshape(shape)
    return [st["k_cache"], st["v_cache"]]


def _plain_paged_attention(st, case):
    """All sequences at once, each padded to the longest."""
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    s, lk = len(st["kv_lens"]), (st["table"].shape[1] - 1) * page
    j, n = torch.arange(lk, device="cuda"), st["kv_lens"].long()[:, None]
    row = (st["table"].long().clamp_min(0)[:, j // page] * page + j % page).reshape(-1)
    k = st["k_cache"].view(-1, hk, d)[row].float().reshape(s, lk, hk, d).permute(0, 2, 3, 1).reshape(s * hk, d, lk)
    v = st["v_cache"].view(-1, hk, d)[row].float().reshape(s, lk, hk, d).transpose(1, 2).reshape(s * hk, lk, d)
    seen = j < n
    if case["window"]:
        seen = seen & ((j < case["sinks"]) | (j >= n - case["window"]))
    p = torch.bmm(st["q"].float().reshape(s * hk, h // hk, d), k).mul_(1 / math.sqrt(d)).reshape(s, h, lk).masked_fill_(~seen[:, None], -math.inf)
    top = p.amax(2, keepdim=True).clamp_min(-1e30)  # a sequence without a key has no largest score
    p = p.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    o = torch.bmm(p.reshape(s * hk, h // hk, lk), v).reshape(s, h, d) / torch.where(total > 0, total, 1.0)
    return o.reshape(s, h * d).to(st["q"].dtype)


_PLAIN = dict(rms_norm=_plain_rms_norm, quantize_i8=_plain_quantize_i8, linear_i8=_plain_linear_i8, paged_append=_plain_paged_append,
              paged_attention=_plain_paged_attention)


def _at(t):
    return None if t is None else t.data_ptr()


def _run_rms_norm(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_rms_norm(st["desc"], _at(st["x"]), _at(st["residual"]), _at(st["gamma"]), _at(st["sum"]), _at(st["y"]), _at(st["scales"]), st["pool"], 0)
    return ([st["sum"]] if case["res"] else []) + [st["y"]] + ([st["scales"]] if case["out"] == "i8" else [])


def _run_quantize_i8(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_quantize_i8(st["desc"], _at(st["x"]), _at(st["y"]), _at(st["scales"]), st["pool"], 0)
    return [st["y"], st["scales"]]


def _run_linear_i8(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_linear_i8(st["desc"], _at(st["x"]), _at(st["x_scales"]), _at(st["w"]), _at(st["w_scales"]), _at(st["bias"]), _at(st["residual"]), _at(st["y"]),
                      _at(st["ws"]), st["ws_bytes"], st["pool"], 0)
    return st["y"]


def _run_paged_append(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_paged_append(st["desc"], _at(st["k"]), _at(st["v"]), _at(st.get("offsets")), _at(st["table"]), _at(st["kv_lens"]), _at(st["k_cache"]),
                         _at(st["v_cache"]), st["pool"], 0)
    return [st["k_cache"], st["v_cache"]]


def _run_paged_attention(st, case):
    import paper_2406_09425_amd as S
    S.sgprs_paged_attention(st["desc"], _at(st["q"]), _at(st["k_cache"]), _at(st["v_cache"]), _at(st["table"]), _at(st["kv_lens"]), _at(st["y"]),
                            _at(st["ws"]), st["ws_bytes"], st["pool"], 0)
    return st["y"]


_RUN = dict(rms_norm=_run_rms_norm, quantize_i8=_run_quantize_i8, linear_i8=_run_linear_i8, paged_append=_run_paged_append,
            paged_attention=_run_paged_attention)


def run(state):
    case = state["case"]
    return (_RUN if own else _PLAIN)[case["kind"]](state, case)


# ---- what a pass cannot do without ---------------------------------------------------------------
def _seen(case, n):
    """Positions that a new token sees in a sequence of n."""
    if not case["window"] or n <= case["window"]:
        return n
    return case["window"] + min(case["sinks"], n - case["window"])


def work(case):
    kind, es = case["kind"], _ES[case["dtype"]]
    if kind == "rms_norm":
        size = case["m"] * case["c"]
        written = size + 4 * case["m"] if case["out"] == "i8" else size * es
        return dict(bytes=size * es * (3 if case["res"] else 1) + written + 4 * case["c"], flops=6.0 * size)
    if kind == "quantize_i8":
        size = case["m"] * case["c"]
        return dict(bytes=size * (es + 1) + 4 * case["m"], flops=3.0 * size)
    if kind == "linear_i8":
        m, n, k = case["m"], case["n"], case["k"]
        return dict(bytes=m * k + n * k + m * n * es * (2 if case["res"] else 1) + 4 * (m + n) + (4 * n if case["bias"] else 0), flops=2.0 * m * n * k)
    kv, page, hk, d = _ints(case["kv"]), case["page"], case["kv_heads"], case["dim"]
    if kind == "paged_append":
        new = _ints(case["new"])
        return dict(bytes=4 * sum(new) * hk * d * es + 4 * sum(-(-v // page) for v in new) + 8 * len(kv), flops=0.0)
    seen = [_seen(case, n) for n in kv]
    return dict(bytes=(2 * sum(seen) * hk + 2 * len(kv) * case["heads"]) * d * es + 4 * sum(-(-v // page) for v in seen) + 4 * len(kv),
                flops=4.0 * sum(seen) * case["heads"] * d)


# ---- the definitions in 64 bits ------------------------------------------------------------------
def _exact_rows_i8(t):
    most = t.abs().max(1).values
    return torch.round(t * 127 / most.clamp_min(1e-300)[:, None]).to(torch.int8), most


def _exact_rows(case, t):
    if case["kind"] == "quantize_i8":
        q, most = _exact_rows_i8(t["x"])
        return [q, most / 127]
    h = t["x"]
    kept = []
    if case["res"]:  # the stream as it is stored, from which the norm is taken
        h = (h + t["residual"]).to(_TORCH[case["dtype"]]).double()
        kept = [h]
    size = torch.sqrt(h.square().sum(1) / case["c"] + _EPS)
    if case["out"] != "i8":
        return kept + [t["gamma"] * h / size[:, None]]
    q, most = _exact_rows_i8(t["gamma"] * h)
    return kept + [q, most / (127 * size)]


def exact(case, seed):
    t = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    if case["kind"] in ("rms_norm", "quantize_i8"):
        return _exact_rows(case, t)
    if case["kind"] == "linear_i8":
        y = torch.matmul(t["x"].double(), t["w"].double().t().contiguous()) * (t["x_scales"][:, None] * t["w_scales"])
        y = y if t["bias"] is None else y + t["bias"]
        y = dict(none=lambda z: z, relu=lambda z: torch.where(z > 0, z, 0.0), silu=lambda z: z * torch.sigmoid(z), gelu=lambda z: z * torch.special.ndtr(z))[case["act"]](y)
        return y if t["residual"] is None else y + t["residual"]
    kv, page, hk, d = _ints(case["kv"]), case["page"], case["kv_heads"], case["dim"]
    tables = t["table"].tolist()
    if case["kind"] == "paged_append":
        at = 0
        for s, (n, new) in enumerate(zip(kv, _ints(case["new"]))):
            for first in range(n - new, n):  # page by page
                if first > n - new and first % page:
                    continue
                there, count = tables[s][first // page], min(page - first % page, n - first)
                for name in ("k", "v"):
                    t[name + "_cache"][there, first % page:first % page + count] = t[name][at:at + count].reshape(count, hk, d)
                at += count
        return [t["k_cache"], t["v_cache"]]
    group, out = case["heads"] // hk, torch.zeros_like(t["q"])
    for s, n in enumerate(kv):  # one sequence and one key head at a time
        if n == 0:
            continue
        first = max(0, n - case["window"]) if case["window"] else 0
        places = torch.tensor(list(range(min(case["sinks"], first))) + list(range(first, n)), device="cuda")
        rows = t["table"][s].long()[places // page], places % page
        for head in range(hk):
            q = t["q"][s, head * group * d:(head + 1) * group * d].reshape(group, d)
            p = torch.softmax(q @ t["k_cache"][rows[0], rows[1], head].t().contiguous() / math.sqrt(d), 1)
            out[s, head * group * d:(head + 1) * group * d] = (p @ t["v_cache"][rows[0], rows[1], head]).reshape(-1)
    return out
