"""The attention block of the example, all its operators in a row, against the same block in 64 bits."""
import pytest
import torch

import block_ops_util as ref
import paper_2406_09425_amd as S
from examples.attention_block import TORCH_DT, AttentionBlock, main, make_params
from gpu_util import TOL

pytestmark = pytest.mark.gpu


def in_64_bits(p, x, n, hw, heads, groups):
    c = x.shape[1]
    p, x = {k: v.double() for k, v in p.items()}, x.double()
    t = ref.group_norm(x, p["gamma1"], p["beta1"], None, n, hw, groups, AttentionBlock.EPS, 0)[0]
    q, k, v = ((t @ p["w_qkv"].t()).view(n * hw, 3, heads, c // heads).unbind(1))
    mixed = ref.attention(q, k, v, [hw] * n, [hw] * n, False, 0.0)[0].reshape(n * hw, c)
    x = x + mixed @ p["w_out"].t() + p["b_out"]
    t = ref.group_norm(x, p["gamma2"], p["beta2"], None, n * hw, 1, 1, AttentionBlock.EPS, 0)[0]
    return x + ref.activation(t @ p["w_up"].t() + p["b_up"], 2) @ p["w_down"].t() + p["b_down"]


@pytest.mark.parametrize("dtype", [S.SGPRS_F32, S.SGPRS_BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,hw,c,heads,groups,cus", [(1, 49, 64, 2, 8, 256), (3, 196, 256, 8, 32, 256), (2, 61, 96, 1, 12, 40)])
def test_block_against_64_bits(dtype, n, hw, c, heads, groups, cus):
    params = make_params(c, dtype, seed=c)
    x = torch.randn(n * hw, c, generator=torch.Generator().manual_seed(n)).to(TORCH_DT[dtype])
    want = in_64_bits(params, x, n, hw, heads, groups)
    pool = S.Pool(1, cus)
    try:
        block = AttentionBlock(params, n, hw, dtype, pool, 0, heads=heads, groups=groups)
        xd = x.cuda()
        torch.cuda.synchronize()
        block.run(xd.data_ptr())
        pool.sync()
        err = float((xd.double().cpu() - want).abs().max() / want.abs().max())
        assert err <= TOL[dtype], err
    finally:
        pool.destroy()


def test_example_runs():
    main(4)
