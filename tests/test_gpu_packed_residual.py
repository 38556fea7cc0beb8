"""A residual on the packed low-bit path with the widest tiles and many of them a block, where the operand ring has the fewest stages."""
import numpy as np
import pytest
import torch

import helpers
from paper_2510_02822_b200 import binding as fx
from test_gpu_epilogue_ops import MODE, TYPES, check, residual

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def make(dev, K, N, G, seed, conv=None):
    rng = np.random.default_rng(seed)
    W = torch.from_numpy(rng.integers(-60, 61, (K, N) if conv is None else (N, conv[0], conv[0], K)).astype(np.int8)).to(dev)
    L = fx.Layer(W, torch.full((N,), 1e-4, device=dev), torch.randn(N, device=dev), rng.permutation(K // G).astype(np.int32), rng.integers(0, 5, K // G).astype(np.uint8), G,
                 conv=None if conv is None else conv[1:])
    return L


def compare(call, plain, shape, dev, seed):
    v = plain()
    for i, t in enumerate(TYPES):
        for first in (False, True):
            r = residual(shape, TYPES[(i + first) % 3], dev, seed + i)
            kw = dict(residual=r, residual_order=int(first))
            for _ in range(3):
                y, guard = helpers.with_guard(torch, shape, t, dev)
                call(fx.ACT_SILU if first else fx.ACT_NONE, MODE[t], Y=y, **kw)
                torch.cuda.synchronize()
                guard()
                check(y, v, fx.ACT_SILU if first else fx.ACT_NONE, r, first)
            y32 = call(fx.ACT_NONE, fx.OUT_DEQUANT_F32, **kw)
            y8 = call(fx.ACT_NONE, fx.OUT_REQUANT_I8, y_scale=0.05, **kw)
            assert torch.equal(y8.float(), torch.clamp(torch.round(y32 / torch.tensor(0.05, device=dev)), -128, 127))
    assert torch.equal(plain(), v)
    fx.flexiq_check_status()


@pytest.mark.parametrize("bn", [256, 192, 128, 64])
@pytest.mark.parametrize("K,G,ratio", [(512, 16, 0.5), (448, 64, 0.5), (1024, 16, 0.9), (1024, 32, 0.25), (256, 16, 1.0), (64, 16, 0.5)])
def test_linear(dev, bn, K, G, ratio):
    M, N = 20011, 528
    L = make(dev, K, N, G, K + bn)
    L.set_lowbit_path(fx.LOWBIT_PACKED_U4)
    L.set_lowbit_ratio(ratio)
    fx.flexiq_force_tile(1, bn)
    try:
        x4, x8, _ = L.quantize_lower(torch.randn(M, K, device=dev), 0.03)
        compare(lambda act, mode, **kw: L.mixed_gemm_act(x4, x8, M, 0.03, act, mode, **kw), lambda: L.mixed_gemm(x4, x8, M, 0.03, 1.0, fx.OUT_DEQUANT_F32), (M, N), dev, bn)
    finally:
        fx.flexiq_force_tile(0, 0)
    L.close()


@pytest.mark.parametrize("Nb,H,W,C,N,R,G", [(33, 59, 12, 448, 416, 1, 64), (33, 28, 31, 128, 544, 3, 16), (20, 33, 29, 256, 512, 3, 32)])
def test_conv(dev, Nb, H, W, C, N, R, G):
    L = make(dev, C, N, G, C + N, conv=(R, 1, R // 2))
    L.set_lowbit_path(fx.LOWBIT_PACKED_U4)
    L.set_lowbit_ratio(0.5)
    x4, x8, _ = L.quantize_lower(torch.randn(Nb, H, W, C, device=dev), 0.03)
    compare(lambda act, mode, **kw: L.mixed_conv_act(x4, x8, Nb, H, W, 0.03, act, mode, **kw), lambda: L.mixed_conv(x4, x8, Nb, H, W, 0.03, 1.0, fx.OUT_DEQUANT_F32), (Nb, H, W, N), dev, C)
    L.close()
