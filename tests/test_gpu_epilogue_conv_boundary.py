"""The fused boundary with an activation behind convolutions of every kind, in both orders, at odd numbers of 16-channel chunks, and with
many tiles a block; and the epilogue's calls without the native marshalling."""
import numpy as np
import pytest
import torch

import helpers
from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import calib, inputs
from test_gpu_epilogue_ops import ACTS, MODE, TYPES, mk, residual

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# plain 1x1, im2col (a stride; a filter wider than three columns), halo patches, streamed patches (one image and several side by side), each with
# few tiles and with several a block
@pytest.mark.parametrize("Nb,H,C,Cmid,R,stride", [(2, 14, 128, 272, 1, 1), (60, 28, 64, 80, 1, 1), (3, 28, 64, 144, 3, 2), (40, 56, 64, 48, 3, 2), (2, 28, 64, 112, 3, 1),
                                                  (60, 28, 64, 48, 3, 1), (3, 9, 64, 16, 3, 1), (4, 14, 256, 208, 3, 1), (48, 28, 160, 112, 3, 1), (5, 7, 256, 144, 3, 1),
                                                  (90, 7, 256, 48, 3, 1), (2, 30, 64, 80, 5, 1)])
def test_both_orders(dev, Nb, H, C, Cmid, R, stride):
    a = inputs.resnet_conv("a", Nb, H, C, Cmid, R, seed=H + C, stride=stride)
    P = (H + 2 * a.pad - R) // stride + 1
    pa, sga, _, _ = helpers.prepare_conv(a)
    rng = np.random.default_rng(H * C + Cmid)
    pb = rng.permutation(Cmid // 16).astype(np.int32)
    A = mk(a, dev, pa, sga, conv=True)
    Wp, wsp, bp = calib.permute_outputs_for_next(torch.from_numpy(a.Wq), torch.from_numpy(a.w_scale), torch.from_numpy(a.bias), pb, 16, conv=True)
    Ap = fx.Layer(Wp.to(dev), wsp.to(dev), bp.to(dev), pa, sga, a.G, conv=(a.stride, a.pad))
    B = fx.Layer(torch.zeros(Cmid, 32, dtype=torch.int8, device=dev), torch.ones(32, device=dev), None, pb, rng.integers(0, 5, Cmid // 16).astype(np.uint8), 16)
    x = torch.from_numpy(a.X).to(dev)
    n = Nb * P * P
    for i, (ra, rb) in enumerate([(0.5, 0.75), (0.0, 1.0), (1.0, 0.0)]):
        for L in (A, Ap):
            L.set_lowbit_ratio(ra)
        B.set_lowbit_ratio(rb)
        x4, x8, _ = A.quantize_lower(x, a.x_scale)
        for act in (ACTS if i == 0 else ACTS[i:4:2]):
            y = A.mixed_conv_act(x4, x8, Nb, H, H, a.x_scale, act, fx.OUT_DEQUANT_F32)
            two = B.quantize_lower(y, a.y_scale)[0][:n * Cmid].clone()
            for L, order in ((A, fx.ORDER_ORIGINAL), (Ap, fx.ORDER_NEXT_SLAB)):
                for _ in range(2):
                    slab, guard = helpers.with_guard(torch, (n * Cmid,), torch.uint8, dev)
                    assert L.mixed_conv_act_to_slab(x4, x8, Nb, H, H, a.x_scale, B, a.y_scale, act, slab=slab, out_order=order) is slab
                    torch.cuda.synchronize()
                    guard()
                    assert torch.equal(slab, two)
    fx.flexiq_check_status()
    for L in (A, Ap, B):
        L.close()


def without_native(*layers):
    for L in layers:
        L._calls = None


def test_linear_without_native_marshalling(dev):
    c = inputs.ranged_linear("c", 300, 256, 272, 16, seed=5, group_structured=True)
    perm, sxg, _, _ = helpers.prepare_linear(c)
    b = inputs.ranged_linear("b", 8, 272, 32, 16, seed=6, group_structured=True)
    A, B = mk(c, dev, perm, sxg), mk(b, dev, *helpers.prepare_linear(b)[:2])
    for L in (A, B):
        L.set_lowbit_ratio(0.5)
    x4, x8, _ = A.quantize_lower(torch.from_numpy(c.X).to(dev), c.x_scale)
    x = torch.randn(300, 256, device=dev)

    def calls():
        out = []
        for t in TYPES:
            r = residual((300, 272), t, dev, 3)
            out.append(A.mixed_gemm_act(x4, x8, 300, c.x_scale, fx.ACT_SILU, MODE[t], residual=r, residual_order=fx.RESIDUAL_BEFORE_ACT))
            out.append(A.mixed_gemm_act(x4, x8, 300, c.x_scale, fx.ACT_GELU, fx.OUT_REQUANT_I8, y_scale=c.y_scale, residual=r))
            assert A.mixed_gemm_act(x4, x8, 300, c.x_scale, fx.ACT_GELU, MODE[t], residual=r, Y=r) is r
            out.append(r)
        out.append(A.mixed_gemm_act_to_slab(x4, x8, 300, c.x_scale, B, 0.05, fx.ACT_GELU)[:300 * 272].clone())
        out.append(A.mixed_gemm_act_to_slab(x4, x8, 300, c.x_scale, B, 0.05, fx.ACT_SILU, slab=torch.empty(300 * 272, dtype=torch.uint8, device=dev)))
        out.append(A.group_norm_to_slab(x, 1, None, None, 0.03, act=fx.ACT_RELU, slab=torch.empty(300 * 256, dtype=torch.uint8, device=dev)))
        assert A.mixed_gemm_act(x4, x8, 0, c.x_scale, fx.ACT_GELU, fx.OUT_DEQUANT_F16).shape == (0, 272)
        return out
    want = calls()
    without_native(A, B)
    assert all(torch.equal(p, q) for p, q in zip(calls(), want, strict=True))
    for L in (A, B):
        L.close()


def test_conv_without_native_marshalling(dev):
    c = inputs.resnet_conv("c", 3, 14, 64, 112, 3, seed=5)
    A = mk(c, dev, *helpers.prepare_conv(c)[:2], conv=True)
    B = fx.Layer(torch.zeros(112, 32, dtype=torch.int8, device=dev), torch.ones(32, device=dev), None, np.arange(7, dtype=np.int32)[::-1].copy(), np.full(7, 2, np.uint8), 16)
    for L in (A, B):
        L.set_lowbit_ratio(0.5)
    x4, x8, _ = A.quantize_lower(torch.from_numpy(c.X).to(dev), c.x_scale)

    def calls():
        out = []
        for t in TYPES:
            r = residual((3, 14, 14, 112), t, dev, 3)
            out.append(A.mixed_conv_act(x4, x8, 3, 14, 14, c.x_scale, fx.ACT_RELU, MODE[t], residual=r, residual_order=fx.RESIDUAL_BEFORE_ACT))
            out.append(A.mixed_conv_act(x4, x8, 3, 14, 14, c.x_scale, fx.ACT_GELU_TANH, fx.OUT_REQUANT_I8, y_scale=c.y_scale, residual=r))
        out.append(A.mixed_conv_act_to_slab(x4, x8, 3, 14, 14, c.x_scale, B, 0.05, fx.ACT_GELU)[:588 * 112].clone())
        assert A.mixed_conv_act(x4, x8, 0, 14, 14, c.x_scale, fx.ACT_GELU, fx.OUT_DEQUANT_F16).shape == (0, 14, 14, 112)
        return out
    want = calls()
    without_native(A, B)
    got = calls()
    assert all(p.shape == q.shape and torch.equal(p, q) for p, q in zip(got, want, strict=True))
    for L in (A, B):
        L.close()


def test_the_same_bits_every_time(dev):
    """A pre-norm block's MLP half over many tiles a block, several times in a row with nothing waited for."""
    M = 12608
    a = inputs.ranged_linear("a", 64, 384, 1536, 16, seed=31, group_structured=True)
    b = inputs.ranged_linear("b", 64, 1536, 384, 16, seed=32, group_structured=True)
    A, B = (mk(c, dev, *helpers.prepare_linear(c)[:2]) for c in (a, b))
    for L in (A, B):
        L.set_lowbit_ratio(0.5)
    x = torch.randn(M, 384, device=dev).half()
    gamma, beta = torch.randn(384, device=dev), torch.randn(384, device=dev)

    def mlp(after=lambda: None):
        s1 = A.group_norm_to_slab(x, 1, gamma, beta, 0.03)
        after()
        s2 = A.mixed_gemm_act_to_slab(s1, None, M, 0.03, B, 0.05, fx.ACT_GELU)
        after()
        y = B.mixed_gemm_act(s2, None, M, 0.05, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=x)
        after()
        return y
    want = mlp(torch.cuda.synchronize)
    for y in [mlp() for _ in range(40)]:
        assert torch.equal(y, want)
    for L in (A, B):
        L.close()
