"""The encoder block with its normalisations, GELU and residual additions in the library's kernels, against the same block step by step."""
import pytest
import torch
import torch.nn.functional as F

from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import vit_block

pytestmark = pytest.mark.gpu


def step_by_step(blk):
    """forward_fused's operators one at a time, with fp32 tensors between them and torch's own fp32 additions (exact: one rounding each)."""
    B, T, D, H, M = blk.batch, blk.T, blk.D, blk.heads, blk.M
    gamma, beta = blk.ln32

    def linear(name, x, mode):
        L, xs, *_ = blk.layers[name]
        x4, x8, _ = L.quantize_lower(x, xs, slabs=(torch.empty(M * L.K, dtype=torch.uint8, device=x.device), None))
        return L.mixed_gemm(x4, None, M, xs, 1.0, mode)
    h = linear("qkv", fx.group_norm(blk.x, 1, gamma, beta, out_dtype=torch.float32), fx.OUT_DEQUANT_F16).view(B, T, 3, H, D // H).permute(2, 0, 3, 1, 4)
    a = F.scaled_dot_product_attention(h[0], h[1], h[2]).transpose(1, 2).reshape(M, D).contiguous()
    x = (linear("proj", a, fx.OUT_DEQUANT_F32) + blk.x.float()).half()
    L, xs, *_ = blk.layers["fc1"]
    x4, _, _ = L.quantize_lower(fx.group_norm(x, 1, gamma, beta, out_dtype=torch.float32), xs, slabs=(torch.empty(M * D, dtype=torch.uint8, device=x.device), None))
    g = L.mixed_gemm_act(x4, None, M, xs, fx.ACT_GELU, fx.OUT_DEQUANT_F32)
    return (linear("fc2", g, fx.OUT_DEQUANT_F32) + x.float()).half()


@pytest.mark.parametrize("model, batch", [("deits", 1), ("deits", 3), ("vitb", 2)])
def test_fused_block(model, batch):
    blk = vit_block.Block(model, batch, torch.device("cuda:0"))
    for ratio in (0.0, 0.5, 1.0):
        blk.set_ratio(ratio)
        assert torch.equal(blk.forward_fused(), step_by_step(blk))
    blk.set_ratio(0.0)
    stock, fused = blk.forward().float(), blk.forward_fused().float()
    # the stock block rounds the normalised and the activated values to fp16 before it quantizes them, which moves some of them by a step of
    # 1/127 of the range: the blocks agree to a few per cent of what they add to the stream, and are not the same computation
    added = (stock - blk.x.float()).norm()
    assert float((stock - fused).norm() / added) < 0.05
    rows = vit_block.measure(blk, 2, fused=True)
    assert all(r["finite"] and r["fused_block_us"] > 0 for r in rows)
    fx.flexiq_check_status()
    blk.close()
