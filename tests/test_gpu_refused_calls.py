"""Calls that the operators between the quantized layers refuse: overlapping memory."""
import numpy as np
import pytest
import torch

from paper_2510_02822_b200 import binding as fx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def refused(call, message):
    with pytest.raises(fx.FlexiqError) as e:
        call()
    assert e.value.code == fx.ERR_INVALID_ARG and message in str(e.value)


def layer(dev, K=64, N=32, conv=None):
    W = torch.ones((K, N) if conv is None else (N, 3, 3, K), dtype=torch.int8, device=dev)
    return fx.Layer(W, torch.ones(N, device=dev), None, np.arange(K // 16, dtype=np.int32), np.zeros(K // 16, np.uint8), 16, conv=conv)


def test_overlaps(dev):
    L, Cv = layer(dev), layer(dev, conv=(1, 1))
    buf = torch.randn(40, 9, 64, device=dev)
    for lo, hi in ((slice(0, 20), slice(1, 21)), (slice(5, 25), slice(0, 20)), (slice(0, 20), slice(19, 39))):
        refused(lambda: fx.group_norm(buf[lo], 8, Y=buf[hi]), "overlap")
    apart = fx.group_norm(buf[:20], 8)
    assert torch.equal(fx.group_norm(buf[:20], 8, Y=buf[20:]), apart)
    raw = torch.zeros(1 << 16, dtype=torch.uint8, device=dev)
    x = raw[4096:4096 + 20 * 64 * 4].view(torch.float32).view(20, 64)
    for start in (4096, 4096 - 20 * 64 + 16, 4096 + 20 * 64 * 4 - 16):
        refused(lambda: L.group_norm_to_slab(x, 8, None, None, 0.1, slab=raw[start:start + 20 * 64]), "overlap")
    for start in (4096 - 20 * 64, 4096 + 20 * 64 * 4):
        L.group_norm_to_slab(x, 8, None, None, 0.1, slab=raw[start:start + 20 * 64])
    x4 = torch.zeros(36 * 64, dtype=torch.uint8, device=dev)
    for M, call in ((36, lambda **k: L.mixed_gemm_act(x4, None, 36, 1.0, fx.ACT_RELU, **k)), (36, lambda **k: Cv.mixed_conv_act(x4, None, 1, 6, 6, 1.0, fx.ACT_RELU, **k))):
        for t, mode, out in ((torch.float32, fx.OUT_DEQUANT_F32, torch.float32), (torch.float16, fx.OUT_DEQUANT_F32, torch.float32), (torch.bfloat16, fx.OUT_REQUANT_I8, torch.int8)):
            size = M * 32 * torch.empty(0, dtype=t).element_size()
            r = raw[8192:8192 + size].view(t).view(M, 32)
            n = M * 32 * torch.empty(0, dtype=out).element_size()
            for start in (8192 + 16, 8192 - n + 16, 8192 + size - 16):
                refused(lambda: call(residual=r, out_mode=mode, Y=raw[start:start + n].view(out).view(M, 32)), "overlap")
            for start in (8192 - n, 8192 + size):
                call(residual=r, out_mode=mode, Y=raw[start:start + n].view(out).view(M, 32))
    torch.cuda.synchronize()
    L.close()
    Cv.close()
