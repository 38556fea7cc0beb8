"""Activation and residual in the epilogue of a layer, against plain 64-bit forms.

v, the layer's de-quantized value, is compared with the oracle's accumulators; what follows it is derived from the GPU's own v (the
DEQUANT_F32 output of the plain call), so that the tolerances only hold what the new arithmetic may add:
  activation   at most 2^-21 |v| (the documented bound; ReLU and none are exact)
  additions    one rounding each, 2^-24 relative to the sum
  outputs      fp16 2^-11 (2^-25 below its normal range), bf16 2^-8, fp32 exact
A residual added before the activation shifts its argument by the addition's rounding, which a slope of at most 1.13 passes on."""
import numpy as np
import pytest
import torch

import helpers
import oracle
from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import calib, inputs

pytestmark = pytest.mark.gpu

ACTS = [fx.ACT_NONE, fx.ACT_RELU, fx.ACT_GELU, fx.ACT_GELU_TANH, fx.ACT_SILU]
HALF = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
MODE = {torch.float32: fx.OUT_DEQUANT_F32, torch.float16: fx.OUT_DEQUANT_F16, torch.bfloat16: fx.OUT_DEQUANT_BF16}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def act64(act, v):
    v = v.double()
    if act == fx.ACT_RELU:
        return v.clamp(min=0)
    if act == fx.ACT_GELU:
        return v * torch.special.ndtr(v)
    if act == fx.ACT_GELU_TANH:
        return v * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (v + 0.044715 * v ** 3))
    if act == fx.ACT_SILU:
        return v * torch.sigmoid(v)
    return v


def check(y, v, act, res, first):
    """y against the definition in 64 bits from the fp32 v."""
    r = None if res is None else res.double()
    a = v.double() if r is None or not first else v.double() + r
    want = act64(act, a)
    tol = torch.zeros_like(want) if act in (fx.ACT_NONE, fx.ACT_RELU) else 2.0 ** -21 * a.abs()
    if r is not None and first:
        tol = tol + 1.13 * 2.0 ** -24 * a.abs()
    if r is not None and not first:
        want = want + r
        tol = tol + 2.0 ** -24 * want.abs()
    tol = tol * 1.001 + HALF[y.dtype] * (want.abs() + tol) + (2.0 ** -25 if y.dtype == torch.float16 else 0.0) + 1e-40
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), (act, y.dtype, first, float((err - tol).max()), float(err.max()))


def mk(case, dev, perm, sxg, conv=False):
    return fx.Layer(torch.from_numpy(case.Wq).to(dev), torch.from_numpy(case.w_scale).to(dev), torch.from_numpy(case.bias).to(dev), perm, sxg, case.G,
                    conv=(case.stride, case.pad) if conv else None)


def residual(shape, dtype, dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * 2).to(dtype)


def all_forms(call, v, y_scale, dev, seed, act_to_slab=None):
    """Every activation, residual type and order, and output of one layer call: `call(act, mode, **kw)`."""
    for i, act in enumerate(ACTS):
        for j, (rt, first) in enumerate([(None, False), (torch.float16, False), (torch.float32, True), (torch.bfloat16, False), (torch.float32, False), (torch.float16, True)]):
            res = None if rt is None else residual(v.shape, rt, dev, seed + j)
            kw = {} if res is None else {"residual": res, "residual_order": fx.RESIDUAL_BEFORE_ACT if first else fx.RESIDUAL_AFTER_ACT}
            y32, guard = helpers.with_guard(torch, v.shape, torch.float32, dev)
            call(act, fx.OUT_DEQUANT_F32, Y=y32, **kw)
            torch.cuda.synchronize()
            guard()
            check(y32, v, act, res, first)
            t = TYPES[1 + (i + j) % 2]
            y16, guard = helpers.with_guard(torch, v.shape, t, dev)
            call(act, MODE[t], Y=y16, **kw)
            torch.cuda.synchronize()
            guard()
            assert torch.equal(y16, y32.to(t))          # the same value, rounded once more
            y8 = call(act, fx.OUT_REQUANT_I8, y_scale=y_scale, **kw)
            q = np.clip(np.rint(y32.cpu().numpy() / np.float32(y_scale)), -128, 127).astype(np.int8)
            assert np.array_equal(y8.cpu().numpy(), q)
    fx.flexiq_check_status()


def linear(dev, M, K, N, G, ratios, seed, path=fx.LOWBIT_MASKED_I8):
    c = inputs.ranged_linear("c", M, K, N, G, seed=seed, group_structured=True)
    perm, sxg, sxs, sw = helpers.prepare_linear(c)
    L = mk(c, dev, perm, sxg)
    L.set_lowbit_path(path)
    q = oracle.quantize(c.X, c.x_scale)
    for ratio in ratios:
        L.set_lowbit_ratio(ratio)
        x4, x8, _ = L.quantize_lower(torch.from_numpy(c.X).to(dev), c.x_scale)
        v = L.mixed_gemm(x4, x8, M, c.x_scale, 1.0, fx.OUT_DEQUANT_F32)
        acc = oracle.mixed_gemm_acc(q, c.Wq, G, perm, sxs, sw, oracle.n_low(ratio, K // G))
        want = acc.astype(np.float64) * (np.float64(np.float32(c.x_scale)) * c.w_scale.astype(np.float64)) + c.bias
        scale = np.abs(acc * (c.x_scale * c.w_scale.astype(np.float64))) * 2.0 ** -22 + np.abs(want) * 2.0 ** -23
        assert bool((np.abs(v.cpu().numpy() - want) <= scale).all())
        all_forms(lambda act, mode, **kw: L.mixed_gemm_act(x4, x8, M, c.x_scale, act, mode, **kw), v, c.y_scale, dev, seed)
    L.close()


@pytest.mark.parametrize("M,K,N,G", [(1, 64, 16, 16), (197, 384, 384, 16), (300, 256, 272, 16), (129, 128, 64, 32), (515, 192, 400, 64),
                                     (260, 1280, 112, 16), (1000, 720, 1104, 16), (2500, 768, 512, 16)])
def test_linear(dev, M, K, N, G):
    linear(dev, M, K, N, G, [0.5] if M > 200 else [0.0, 0.3, 1.0], seed=M + N)


@pytest.mark.parametrize("cg,bn", [(1, 64), (1, 128), (1, 192), (1, 256), (2, 128), (2, 192), (2, 256)])
def test_every_tile_shape(dev, cg, bn):
    fx.flexiq_force_tile(cg, bn)
    try:
        linear(dev, 700, 256, 720, 16, [0.5], seed=cg * 1000 + bn)
        linear(dev, 150, 1280, 80, 16, [0.5], seed=cg * 1000 + bn + 1)
    finally:
        fx.flexiq_force_tile(0, 0)


def test_packed_path(dev):
    linear(dev, 300, 256, 272, 16, [0.0, 0.5, 1.0], seed=77, path=fx.LOWBIT_PACKED_U4)


# plain 1x1, im2col (strides; a filter wider than three columns), halo patches, streamed patches (one and several images side by side)
@pytest.mark.parametrize("Nb,H,C,Cout,R,stride", [(2, 14, 128, 272, 1, 1), (3, 28, 64, 128, 3, 2), (2, 28, 64, 64, 3, 1), (3, 9, 64, 112, 3, 1),
                                                  (4, 14, 256, 256, 3, 1), (5, 7, 256, 144, 3, 1), (2, 30, 64, 64, 5, 1)])
def test_conv(dev, Nb, H, C, Cout, R, stride):
    c = inputs.resnet_conv("c", Nb, H, C, Cout, R, seed=H + C, stride=stride)
    perm, sxg, _, _ = helpers.prepare_conv(c)
    L = mk(c, dev, perm, sxg, conv=True)
    L.set_lowbit_ratio(0.5)
    x4, x8, _ = L.quantize_lower(torch.from_numpy(c.X).to(dev), c.x_scale)
    v = L.mixed_conv(x4, x8, Nb, H, H, c.x_scale, 1.0, fx.OUT_DEQUANT_F32)      # compared with the oracle by the parity tests
    all_forms(lambda act, mode, **kw: L.mixed_conv_act(x4, x8, Nb, H, H, c.x_scale, act, mode, **kw), v, c.y_scale, dev, H + Cout)
    L.close()


@pytest.mark.parametrize("N", [16, 48, 272, 528, 560])
def test_boundary_of_many_tiles_with_a_narrow_last_one(dev, N):
    """An odd number of 16-channel chunks, so that a warp stages one chunk in one tile and the next chunk in the next: many tiles a block, hardly
    any work between them, several times."""
    rng = np.random.default_rng(N)
    M, K = 24000, 64
    A = fx.Layer(torch.from_numpy(rng.integers(-127, 128, (K, N)).astype(np.int8)).to(dev), torch.full((N,), 1e-3, device=dev), torch.randn(N, device=dev),
                 rng.permutation(K // 16).astype(np.int32), rng.integers(0, 5, K // 16).astype(np.uint8), 16)
    B = fx.Layer(torch.from_numpy(rng.integers(-127, 128, (N, 32)).astype(np.int8)).to(dev), torch.ones(32, device=dev), None,
                 rng.permutation(N // 16).astype(np.int32), rng.integers(0, 5, N // 16).astype(np.uint8), 16)
    for L in (A, B):
        L.set_lowbit_ratio(0.5)
    x4, x8, _ = A.quantize_lower(torch.randn(M, K, device=dev), 0.03)
    for act in (fx.ACT_NONE, fx.ACT_SILU):
        y = A.mixed_gemm_act(x4, x8, M, 0.03, act, fx.OUT_DEQUANT_F32)
        two = B.quantize_lower(y, 0.02)[0][:M * N].view(torch.uint8).view(M, N).clone()
        for _ in range(4):
            slab, guard = helpers.with_guard(torch, (M, N), torch.uint8, dev)
            A.mixed_gemm_act_to_slab(x4, x8, M, 0.03, B, 0.02, act, slab=slab)
            torch.cuda.synchronize()
            guard()
            assert torch.equal(slab, two)
    for L in (A, B):
        L.close()


@pytest.mark.parametrize("M,K,N1,G1,G2", [(300, 256, 272, 16, 16), (129, 128, 64, 16, 32), (1, 64, 16, 16, 16), (1000, 384, 1024, 16, 64), (260, 1280, 112, 16, 16)])
def test_boundary_equals_the_two_calls(dev, M, K, N1, G1, G2):
    a = inputs.ranged_linear("a", M, K, N1, G1, seed=M, group_structured=True)
    b = inputs.ranged_linear("b", 64, N1, 32, G2, seed=M + 1, group_structured=True)
    pa, sga, _, _ = helpers.prepare_linear(a)
    pb, sgb, _, _ = helpers.prepare_linear(b, np.random.default_rng(M).integers(0, 5, N1 // G2).astype(np.uint8))
    A, B = mk(a, dev, pa, sga), mk(b, dev, pb, sgb)
    Wp, wsp, bp = calib.permute_outputs_for_next(torch.from_numpy(a.Wq), torch.from_numpy(a.w_scale), torch.from_numpy(a.bias), pb, G2)
    Ap = fx.Layer(Wp.to(dev), wsp.to(dev), bp.to(dev), pa, sga, G1)
    for ra, rb in [(0.0, 0.0), (0.5, 0.5), (1.0, 0.25), (0.25, 1.0)]:
        for L in (A, Ap):
            L.set_lowbit_ratio(ra)
        B.set_lowbit_ratio(rb)
        x4, x8, _ = A.quantize_lower(torch.from_numpy(a.X).to(dev), a.x_scale)
        for act in ACTS:
            # scales of both quotient forms: the second one's significand lies next to a multiple of 2^17
            for xs in (a.y_scale, float(np.float32((2 ** 23 + 2 ** 17 + 3) * 2.0 ** -28)) * max(1.0, a.y_scale)):
                y = A.mixed_gemm_act(x4, x8, M, a.x_scale, act, fx.OUT_DEQUANT_F32)
                two = B.quantize_lower(y, xs)[0][:M * N1].view(M, N1).clone()
                slab, guard = helpers.with_guard(torch, (M, N1), torch.uint8, dev)
                A.mixed_gemm_act_to_slab(x4, x8, M, a.x_scale, B, xs, act, slab=slab)
                torch.cuda.synchronize()
                guard()
                assert torch.equal(slab, two)
                slab, guard = helpers.with_guard(torch, (M, N1), torch.uint8, dev)
                Ap.mixed_gemm_act_to_slab(x4, x8, M, a.x_scale, B, xs, act, slab=slab, out_order=fx.ORDER_NEXT_SLAB)
                torch.cuda.synchronize()
                guard()
                assert torch.equal(slab, two)
    fx.flexiq_check_status()
    for L in (A, B, Ap):
        L.close()


@pytest.mark.parametrize("Nb,H,C,Cmid,R,stride", [(2, 14, 128, 64, 3, 1), (3, 28, 64, 128, 3, 2), (2, 14, 128, 256, 1, 1), (4, 14, 256, 256, 3, 1)])
def test_conv_boundary_equals_the_two_calls(dev, Nb, H, C, Cmid, R, stride):
    a = inputs.resnet_conv("a", Nb, H, C, Cmid, R, seed=H + C, stride=stride)
    P = (H + 2 * a.pad - R) // stride + 1
    b = inputs.resnet_conv("b", Nb, P, Cmid, 64, 3, seed=H + C + 1)
    pa, sga, _, _ = helpers.prepare_conv(a)
    pb, sgb, _, _ = helpers.prepare_conv(b, np.random.default_rng(H * C).integers(0, 5, Cmid // b.G).astype(np.uint8))
    A, B = mk(a, dev, pa, sga, conv=True), mk(b, dev, pb, sgb, conv=True)
    A.set_lowbit_ratio(0.5)
    B.set_lowbit_ratio(0.75)
    x4, x8, _ = A.quantize_lower(torch.from_numpy(a.X).to(dev), a.x_scale)
    n = Nb * P * P * Cmid
    for act in ACTS:
        y = A.mixed_conv_act(x4, x8, Nb, H, H, a.x_scale, act, fx.OUT_DEQUANT_F32)
        two = B.quantize_lower(y, a.y_scale)[0][:n].clone()
        slab, guard = helpers.with_guard(torch, (n,), torch.uint8, dev)
        A.mixed_conv_act_to_slab(x4, x8, Nb, H, H, a.x_scale, B, a.y_scale, act, slab=slab)
        torch.cuda.synchronize()
        guard()
        assert torch.equal(slab, two)
    B.mixed_conv(slab, None, Nb, P, P, a.y_scale, 1.0, fx.OUT_DEQUANT_F32)      # the handle knows the slab's ratio
    fx.flexiq_check_status()
    A.close()
    B.close()


def small(dev, M=200, K=128, N=96):
    c = inputs.ranged_linear("s", M, K, N, 16, seed=3, group_structured=True)
    perm, sxg, _, _ = helpers.prepare_linear(c)
    L = mk(c, dev, perm, sxg)
    L.set_lowbit_ratio(0.5)
    x4, x8, _ = L.quantize_lower(torch.from_numpy(c.X).to(dev), c.x_scale)
    return c, L, x4, x8


@pytest.mark.parametrize("t", TYPES)
def test_residual_in_place_and_at_any_alignment(dev, t):
    for M, N in ((200, 96), (1500, 400)):
        c, L, x4, x8 = small(dev, M, 128, N)
        r = residual((M, N), t, dev, 9)
        want = L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_GELU, MODE[t], residual=r)
        mine = r.clone()
        assert L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_GELU, MODE[t], residual=mine, Y=mine) is mine
        assert torch.equal(mine, want)
        pad = 16 // r.element_size()                     # sixteen bytes past a 32-byte boundary
        odd = torch.empty(M * N + pad, dtype=t, device=dev)[pad:].view(M, N)
        odd.copy_(r)
        assert odd.data_ptr() % 32 == 16
        assert torch.equal(L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_GELU, MODE[t], residual=odd), want)
        L.close()


def test_special_values(dev):
    """Infinities and NaNs reach the epilogue through the bias and the residual."""
    c, L, x4, x8 = small(dev)
    bias = torch.from_numpy(c.bias).clone()
    bias[0], bias[1], bias[2], bias[3], bias[4] = float("inf"), float("-inf"), float("nan"), -3e38, 3e38
    perm, sxg, _, _ = helpers.prepare_linear(c)
    S = fx.Layer(torch.from_numpy(c.Wq).to(dev), torch.from_numpy(c.w_scale).to(dev), bias.to(dev), perm, sxg, 16)
    S.set_lowbit_ratio(0.5)
    M, inf = c.M, float("inf")
    for act, low in ((fx.ACT_NONE, -inf), (fx.ACT_RELU, 0.0), (fx.ACT_GELU, 0.0), (fx.ACT_GELU_TANH, 0.0), (fx.ACT_SILU, 0.0)):
        y = S.mixed_gemm_act(x4, x8, M, c.x_scale, act, fx.OUT_DEQUANT_F32)
        assert bool((y[:, 0] == inf).all()) and bool((y[:, 1] == low).all()) and bool(y[:, 2].isnan().all())
        assert bool(((y[:, 3] == 0.0) if act != fx.ACT_NONE else (y[:, 3] < -2e38)).all()) and bool((y[:, 4] > 2e38).all())
        assert not bool(y[:, 5:].isnan().any())
        q = S.mixed_gemm_act(x4, x8, M, c.x_scale, act, fx.OUT_REQUANT_I8, y_scale=0.1)
        assert bool((q[:, 0] == 127).all()) and bool((q[:, 1] == (-128 if act == fx.ACT_NONE else 0)).all()) and bool((q[:, 2] == 127).all())
    r = residual((M, c.N), torch.float16, dev, 1)
    r[5] = -inf
    r[6, 7] = float("nan")
    y = L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_F16, residual=r)
    assert bool((y[5] == -inf).all()) and bool(y[6, 7].isnan()) and int(y.isnan().sum()) == 1
    y = L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_F16, residual=r, residual_order=fx.RESIDUAL_BEFORE_ACT)
    assert bool((y[5] == 0).all()) and bool(y[6, 7].isnan()) and int(y.isnan().sum()) == 1
    L.close()
    S.close()


def test_activations_over_their_range(dev):
    """Each activation over arguments of every magnitude, through a layer whose weights are zero and whose residual is the argument."""
    N, M = 256, 4096
    Z = fx.Layer(torch.zeros(64, N, dtype=torch.int8, device=dev), torch.ones(N, device=dev), None, np.arange(4, dtype=np.int32), np.zeros(4, np.uint8), 16)
    x4 = torch.zeros(M * 64, dtype=torch.uint8, device=dev)
    x = torch.linspace(-1, 1, M * N // 2, device=dev, dtype=torch.float64)
    v = torch.cat([40 * x ** 3, torch.sign(x) * 10 ** (-30 + 34 * x.abs())]).float().view(M, N)
    for act in ACTS:
        y = Z.mixed_gemm_act(x4, None, M, 1.0, act, fx.OUT_DEQUANT_F32, residual=v, residual_order=fx.RESIDUAL_BEFORE_ACT)
        check(y, v, act, None, False)
    Z.close()


def test_empty_and_refused(dev):
    c, L, x4, x8 = small(dev)
    M, N = c.M, c.N
    assert L.mixed_gemm_act(x4, x8, 0, c.x_scale, fx.ACT_GELU, fx.OUT_DEQUANT_F16).shape == (0, N)
    r = residual((M, N), torch.float16, dev, 1)

    def refused(call, code=fx.ERR_INVALID_ARG):
        with pytest.raises(fx.FlexiqError) as e:
            call()
        assert e.value.code == code
    args = (x4, x8, M, c.x_scale)
    refused(lambda: L.mixed_gemm_act(*args, 5, fx.OUT_DEQUANT_F16))
    refused(lambda: L.mixed_gemm_act(*args, -1, fx.OUT_DEQUANT_F16))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_ACC_I32))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, 3))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_REQUANT_I8, y_scale=0.0))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=r, residual_order=2))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=r[:-1]))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=r.t().contiguous().t()))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=r.cpu()))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=r.to(torch.int8)))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, Y=r.float()))
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_BF16, residual=r, Y=r.view(torch.bfloat16)))     # one memory, two types
    refused(lambda: L.mixed_gemm_act(x4, x8, -1, c.x_scale, fx.ACT_NONE, fx.OUT_DEQUANT_F16))
    off = torch.empty(M * N + 1, dtype=torch.float16, device=dev)[1:].view(M, N)
    refused(lambda: L.mixed_gemm_act(*args, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=off))
    refused(lambda: L.mixed_gemm_act_to_slab(*args, L, 0.1, fx.ACT_GELU))                 # 96 outputs into 128 inputs
    b = inputs.ranged_linear("b", 8, N, 16, 16, seed=6)
    pb, sgb, _, _ = helpers.prepare_linear(b)
    B = mk(b, dev, pb, sgb)
    refused(lambda: L.mixed_gemm_act_to_slab(*args, B, 0.0, fx.ACT_GELU))
    refused(lambda: L.mixed_gemm_act_to_slab(*args, B, 0.1, 9))
    refused(lambda: L.mixed_gemm_act_to_slab(*args, B, 0.1, fx.ACT_GELU, out_order=5))
    refused(lambda: L.mixed_gemm_act_to_slab(*args, B, 0.1, fx.ACT_GELU, slab=torch.empty(M * N - 1, dtype=torch.uint8, device=dev)))
    refused(lambda: L.mixed_conv_act(x4, x8, 1, 4, 4, c.x_scale, fx.ACT_NONE, fx.OUT_DEQUANT_F16))
    B.set_lowbit_path(fx.LOWBIT_PACKED_U4)
    refused(lambda: L.mixed_gemm_act_to_slab(*args, B, 0.1, fx.ACT_GELU), fx.ERR_UNSUPPORTED)
    B.close()
    L.close()


def test_other_stream_and_graph(dev):
    """Eager on a side stream, and captured with the plain call of the same scales: one graph, replayed on changed inputs."""
    c, L, x4, x8 = small(dev, 700, 256, 512)
    M = c.M
    r = residual((M, c.N), torch.bfloat16, dev, 4)
    want = L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_BF16, residual=r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = L.mixed_gemm_act(x4, x8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_BF16, residual=r)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)
    X = torch.from_numpy(c.X).to(dev)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a4, a8, _ = L.quantize_lower(X, c.x_scale)
        gy = L.mixed_gemm_act(a4, a8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_BF16, residual=r)
        gp = L.mixed_gemm(a4, a8, M, c.x_scale, 1.0, fx.OUT_DEQUANT_BF16)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(gy, want)
    X.mul_(0.5)
    r.mul_(-1)
    g.replay()
    torch.cuda.synchronize()
    got = gy.clone()
    assert torch.equal(gp, L.mixed_gemm(a4, a8, M, c.x_scale, 1.0, fx.OUT_DEQUANT_BF16))
    assert torch.equal(got, L.mixed_gemm_act(a4, a8, M, c.x_scale, fx.ACT_SILU, fx.OUT_DEQUANT_BF16, residual=r)) and not torch.equal(got, want)
    L.close()


def test_offsets_beyond_32_bits(dev):
    """Residual and output of more than 2^32 bytes, updated in place; rows at the end and around the mark against a call on those rows alone."""
    K, N = 64, 1040
    M = (1 << 32) // (4 * N) + 50_021
    W = torch.randint(-100, 100, (K, N), dtype=torch.int8, device=dev)
    L = fx.Layer(W, torch.full((N,), 0.01, device=dev), None, np.arange(4, dtype=np.int32), np.zeros(4, np.uint8), 16)
    x = torch.randint(-100, 100, (M, K), dtype=torch.int8, device=dev)
    r = torch.randn(M, N, device=dev)
    mark = (1 << 32) // (4 * N)
    parts = [slice(0, 300), slice(mark - 200, mark + 300), slice(M - 333, M)]
    wants = [L.mixed_gemm_act(x[p].contiguous(), None, p.stop - p.start, 0.02, fx.ACT_GELU, fx.OUT_DEQUANT_F32, residual=r[p].contiguous()) for p in parts]
    L.mixed_gemm_act(x, None, M, 0.02, fx.ACT_GELU, fx.OUT_DEQUANT_F32, residual=r, Y=r)
    for p, w in zip(parts, wants):
        assert torch.equal(r[p], w)
    fx.flexiq_check_status()
    L.close()
