"""Calls that the operators between the quantized layers refuse: overlapping memory, numbers that the library's arguments cannot hold."""
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


@pytest.mark.parametrize("native", [True, False])
def test_numbers_beyond_32_bits(dev, native, monkeypatch):
    """Cut off to 32 bits each of these would be an ordinary call."""
    big = 2 ** 32
    L, Cv, B = layer(dev), layer(dev, conv=(1, 1)), layer(dev, K=32)
    if not native:
        monkeypatch.setattr(fx, "_native_calls", lambda: None)
        for each in (L, Cv, B):
            each._calls = None
    x = torch.randn(36, 64, device=dev)
    x4 = torch.zeros(36 * 64, dtype=torch.uint8, device=dev)
    r = torch.zeros(36, 32, device=dev)
    linear = dict(act=fx.ACT_RELU, out_mode=fx.OUT_DEQUANT_F32, residual=r, residual_order=0)
    L.mixed_gemm_act(x4, None, 36, 1.0, **linear)
    for name in ("act", "out_mode", "residual_order"):
        refused(lambda: L.mixed_gemm_act(x4, None, 36, 1.0, **{**linear, name: linear[name] + big}), name)
    conv = dict(Nb=1, H=6, W=6, act=fx.ACT_RELU, out_mode=fx.OUT_DEQUANT_F32, residual=r, residual_order=0, Y=torch.empty(36, 32, device=dev))
    Cv.mixed_conv_act(x4, None, x_scale=1.0, **conv)
    for name in ("Nb", "H", "W", "act", "out_mode", "residual_order"):
        refused(lambda: Cv.mixed_conv_act(x4, None, x_scale=1.0, **{**conv, name: conv[name] + big}), name)
    slab = dict(act=fx.ACT_RELU, out_order=0, slab=torch.empty(36 * 32, dtype=torch.uint8, device=dev))
    for call, more in ((lambda **k: L.mixed_gemm_act_to_slab(x4, None, 36, 1.0, B, 1.0, **k), {}), (lambda **k: Cv.mixed_conv_act_to_slab(x4, None, x_scale=1.0, nxt=B, next_x_scale=1.0, **k), dict(Nb=1, H=6, W=6))):
        whole = {**slab, **more}
        call(**whole)
        for name in whole:
            if name != "slab":
                refused(lambda: call(**{**whole, name: whole[name] + big}), name)
    for name in ("groups", "act"):
        norm = dict(groups=8, act=fx.ACT_RELU)
        refused(lambda: fx.group_norm(x, **{**norm, name: norm[name] + big}), name)
        refused(lambda: L.group_norm_to_slab(x, gamma=None, beta=None, x_scale=1.0, **{**norm, name: norm[name] + big}), name)
        refused(lambda: L.group_norm_to_slab(x, gamma=None, beta=None, x_scale=1.0, **{**norm, name: norm[name] - big}), name)
    refused(lambda: fx.group_norm(torch.empty(1, big + 64, dtype=torch.float16, device=dev), 8), "channels")
    torch.cuda.synchronize()
    for each in (L, Cv, B):
        each.close()


def test_first_call_in_a_capture(dev):
    """Nothing that a first call has to set up is missing or refused under a capture: each way of cutting an image, once, in a process of its own."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2510_02822_b200 import binding as fx
calls = [((32, 784, 256), 32), ((2, 3136, 64), 8), ((40, 49, 64), 32), ((2, 40000, 64), 8), ((1, 66000, 128), 32), ((50, 1, 768), 1)]
xs = [torch.randn(s, device="cuda").half() for s, _ in calls]
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    ys = [fx.group_norm(x, groups, act=fx.ACT_SILU) for x, (_, groups) in zip(xs, calls)]
g.replay()
torch.cuda.synchronize()
assert all(torch.equal(y, fx.group_norm(x, groups, act=fx.ACT_SILU)) for x, y, (_, groups) in zip(xs, ys, calls))
fx.flexiq_check_status()
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
