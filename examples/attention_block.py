"""ResNet18 with a self-attention block between its third and fourth layer, on one partition.

The block works on the channels-last feature map that stage 3 leaves (14 x 14 positions of 256 channels an
image): group norm, one product for queries, keys and values, attention among an image's positions, the
output projection onto the skip connection, and a two-layer perceptron behind a layer norm.  Images are
packed sequences, so a batch needs no padding; q, k and v are three column ranges of one product's rows.

    python -m examples.attention_block [batch]
"""
import math
import sys

import torch

import paper_2406_09425_amd as S

TORCH_DT = {S.SGPRS_F32: torch.float32, S.SGPRS_BF16: torch.bfloat16}


def make_params(c, dtype, seed=0, hidden=None):
    """Random weights of a block of `c` channels, on the host: matrices in the compute type, the rest in fp32."""
    g = torch.Generator().manual_seed(seed)
    hidden = 4 * c if hidden is None else hidden

    def matrix(n, k):
        return (torch.randn(n, k, generator=g) / math.sqrt(k)).to(TORCH_DT[dtype])

    def affine():
        return torch.rand(c, generator=g) + 0.5, torch.randn(c, generator=g) * 0.1

    gamma1, beta1 = affine()
    gamma2, beta2 = affine()
    return dict(gamma1=gamma1, beta1=beta1, w_qkv=matrix(3 * c, c), w_out=matrix(c, c), b_out=torch.randn(c, generator=g) * 0.1, gamma2=gamma2, beta2=beta2,
                w_up=matrix(hidden, c), b_up=torch.randn(hidden, generator=g) * 0.1, w_down=matrix(c, hidden), b_down=torch.randn(c, generator=g) * 0.1)


class AttentionBlock:
    """Holds the weights, descriptors, offsets and scratch for `n` images of `hw` positions on one partition."""

    EPS = 1e-5

    def __init__(self, params, n, hw, dtype, pool, partition, heads=8, groups=32):
        self.pool, self.partition = pool, partition
        self.p = {k: v.cuda() for k, v in params.items()}
        c, hidden = params["w_out"].shape[0], params["w_up"].shape[0]
        m, cus, tdt = n * hw, pool.partition_cus(partition), TORCH_DT[dtype]
        self.norm1 = S.GroupNormDesc(n=n, hw=hw, c=c, groups=groups, dtype=dtype, eps=self.EPS)
        self.norm2 = S.GroupNormDesc(n=m, hw=1, c=c, groups=1, dtype=dtype, eps=self.EPS)  # a layer norm of tokens
        self.qkv = S.LinearDesc(m=m, n=3 * c, k=c, dtype=dtype)
        self.out = S.LinearDesc(m=m, n=c, k=c, dtype=dtype)
        self.up = S.LinearDesc(m=m, n=hidden, k=c, dtype=dtype, act=S.SGPRS_ACT_GELU)
        self.down = S.LinearDesc(m=m, n=c, k=hidden, dtype=dtype)
        self.attention = S.AttentionDesc(n_seqs=n, total_q=m, total_kv=m, max_q=hw, max_kv=hw, heads=heads, kv_heads=heads, head_dim=c // heads,
                                         dtype=dtype, ldq=3 * c, ldk=3 * c, ldv=3 * c)
        self.offsets = (torch.arange(n + 1, dtype=torch.int32) * hw).cuda()
        self.normed, self.rows = torch.empty(m, c, dtype=tdt, device="cuda"), torch.empty(m, 3 * c, dtype=tdt, device="cuda")
        self.mixed, self.hidden = torch.empty(m, c, dtype=tdt, device="cuda"), torch.empty(m, hidden, dtype=tdt, device="cuda")
        self.ws_bytes = max([S.sgprs_group_norm_workspace(d, cus) for d in (self.norm1, self.norm2)] +
                            [S.sgprs_linear_workspace(d, cus) for d in (self.qkv, self.out, self.up, self.down)] +
                            [S.sgprs_attention_workspace(self.attention, cus)])
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()  # partitions are not ordered after torch's stream

    def run(self, x: int):
        """Enqueues the block on the feature map at device address x; the result takes its place."""
        p, at, size = {k: v.data_ptr() for k, v in self.p.items()}, (self.pool, self.partition), self.rows.element_size()
        ws, rows, c = (self.ws.data_ptr(), self.ws_bytes), self.rows.data_ptr(), self.out.n
        normed, mixed, hidden = self.normed.data_ptr(), self.mixed.data_ptr(), self.hidden.data_ptr()
        S.sgprs_group_norm(self.norm1, x, p["gamma1"], p["beta1"], None, normed, *ws, *at)
        S.sgprs_linear(self.qkv, normed, p["w_qkv"], None, None, rows, *ws, *at)
        S.sgprs_attention(self.attention, rows, rows + c * size, rows + 2 * c * size, self.offsets.data_ptr(), self.offsets.data_ptr(), mixed, *ws, *at)
        S.sgprs_linear(self.out, mixed, p["w_out"], p["b_out"], x, x, *ws, *at)
        S.sgprs_group_norm(self.norm2, x, p["gamma2"], p["beta2"], None, normed, *ws, *at)
        S.sgprs_linear(self.up, normed, p["w_up"], p["b_up"], None, hidden, *ws, *at)
        S.sgprs_linear(self.down, hidden, p["w_down"], p["b_down"], x, x, *ws, *at)


def main(batch: int) -> None:
    from workloads import BN_EPS, make_input, make_resnet18_params
    dtype = S.SGPRS_BF16
    total = S.Pool(1, 8).info()["total_cus"]
    pool = S.Pool(1, total)
    task = S.Task(make_resnet18_params(1, 0, bf16=True), dtype, batch, BN_EPS)
    block = AttentionBlock(make_params(256, dtype), batch, 14 * 14, dtype, pool, 0)
    x = torch.from_numpy(make_input(1, 0, (batch, 224, 224, 3), bf16=True)).bfloat16().cuda()
    maps = [torch.empty(task.stage_io(j, batch)["out_bytes"], dtype=torch.uint8, device="cuda") for j in range(6)]
    torch.cuda.synchronize()

    def infer():
        at = x.data_ptr()
        for j in range(6):
            task.stage_run(j, batch, at, maps[j].data_ptr(), pool, 0)
            at = maps[j].data_ptr()
            if j == 3:
                block.run(at)

    infer()
    pool.sync()
    stream = torch.cuda.ExternalStream(pool.stream(0))
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record(stream)
    for _ in range(20):
        infer()
    end.record(stream)
    pool.sync()
    logits = maps[5].view(torch.float32).view(batch, 1000)
    assert bool(torch.isfinite(logits).all())
    print(f"{batch} images: {begin.elapsed_time(end) / 20:.3f} ms an inference with the block, classes {logits.argmax(1)[:8].tolist()}")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 64)
