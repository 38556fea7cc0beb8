"""Group normalisation of channels-last tensors against its definition in 64 bits.

Tolerance, from the fp32 arithmetic the documentation promises (u = 2^-24; x the group's values, d = x - mean, E a mean over the group):
  mean   sums of at most 24 roundings in a row:  32 u E|x|  (which also covers the rounding of beta - mean * scale)
  scale  1 / sqrt(var + eps): sums of squares of at most 64 roundings, the square root and the quotient: 64 u relative, on |d| scale
  rest   4 u (|y| + |beta|)
  activation  2^-21 of its argument, and a slope of at most 1.13; output fp16 2^-11 (2^-25 below its normal range), bf16 2^-8."""
import numpy as np
import pytest
import torch

import helpers
import oracle
from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import inputs
from test_gpu_epilogue_ops import ACTS, HALF, TYPES, act64, mk

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


def draw(shape, dtype, dev, seed, mean=1.0, spread=1.0):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    C = shape[-1]
    x = torch.randn(shape, generator=g, device=dev) * (0.25 + 1.75 * torch.rand(C, generator=g, device=dev)) * spread + mean * torch.randn(C, generator=g, device=dev)
    return x.to(dtype), 1 + 0.3 * torch.randn(C, generator=g, device=dev), 0.3 * torch.randn(C, generator=g, device=dev)


def want_and_tolerance(x, groups, gamma, beta, eps, act):
    shape, C = x.shape, x.shape[-1]
    g = x.double().reshape(shape[0], -1, groups, C // groups)
    gm = torch.ones(C, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    bt = torch.zeros(C, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    mean = g.mean((1, 3), keepdim=True)
    d = g - mean
    rstd = ((d * d).mean((1, 3), keepdim=True) + eps).rsqrt()
    full = lambda t: t.expand_as(g).reshape(shape)      # noqa: E731
    scale = full(rstd) * gm.abs()
    pre = (d * rstd).reshape(shape) * gm + bt
    tol = scale * (32 * U * full(g.abs().mean((1, 3), keepdim=True)) + 64 * U * d.reshape(shape).abs()) + 4 * U * (pre.abs() + bt.abs())
    if act in (fx.ACT_NONE, fx.ACT_RELU):
        return act64(act, pre), tol
    return act64(act, pre), 1.13 * tol + 2.0 ** -21 * (pre.abs() + tol)


def check(y, want, tol):
    tol = tol * 1.001 + HALF[y.dtype] * (want.abs() + tol) + (2.0 ** -25 if y.dtype == torch.float16 else 0.0) + 1e-40
    err = (y.double() - want).abs()
    assert bool((err <= tol).all()), (y.dtype, float((err / tol).max()), float(err.max()))


def run(x, groups, gamma, beta, act, out, dev, eps=1e-5):
    y, guard = helpers.with_guard(torch, tuple(x.shape), out, dev)
    before = x.clone()
    assert fx.group_norm(x, groups, gamma, beta, eps, act, out, Y=y) is y
    torch.cuda.synchronize()
    guard()
    assert torch.equal(x, before)
    check(y, *want_and_tolerance(x, groups, gamma, beta, eps, act))
    again = fx.group_norm(x, groups, gamma, beta, eps, act, out)
    assert torch.equal(again.view(torch.uint8), y.view(torch.uint8))      # the same bits every time
    return y


# images, positions, channels, groups: one position, one channel a group, groups that cut 16-byte pieces (3, 10, 12, 20 channels), rows
# that are no multiple of 16 bytes (30, 33, 77 channels), one group over everything, images of many and of very many positions
SHAPES = [(1, 1, 16, 1), (3, 1, 768, 1), (197, 1, 384, 1), (5, 1, 1000, 4), (1, 1, 4096, 1), (70, 1, 17, 1), (2, 1, 9000, 2), (1, 1, 32, 32),
          (1, 49, 512, 32), (32, 49, 64, 32), (3, 9, 96, 32), (2, 100, 320, 32), (2, 81, 640, 32), (1, 1000, 48, 4), (7, 3, 30, 5), (2, 50, 33, 11),
          (1, 2, 77, 1), (4, 197, 768, 1), (2, 64, 2056, 8), (1, 60, 5000, 2), (3, 3136, 64, 32), (1, 4097, 128, 8), (2, 2, 64, 64), (9, 1023, 24, 2),
          (1, 16384, 128, 32), (1, 70001, 16, 4), (2, 30000, 40, 8), (1, 40000, 12, 3), (1, 9001, 6, 2), (500, 4, 64, 8), (1, 300, 8224, 32),
          (1, 66000, 128, 32), (1, 90001, 64, 1), (700, 49, 128, 32), (4100, 3, 192, 12), (40, 49, 2048, 32), (24, 784, 256, 32), (3, 900, 1280, 32), (2, 12544, 64, 32),
          (40, 1024, 320, 32)]


@pytest.mark.parametrize("Nb,P,C,groups", SHAPES)
def test_shapes_and_types(dev, Nb, P, C, groups):
    for i, t in enumerate(TYPES):
        x, gamma, beta = draw((Nb, P, C), t, dev, seed=Nb + P + C + i)
        for out in (t, TYPES[(i + 1) % 3]):
            run(x, groups, gamma, beta, ACTS[(i + P + (out == t)) % 5], out, dev)
    run(x, groups, None, None, fx.ACT_NONE, torch.float32, dev)
    run(x, groups, gamma, None, fx.ACT_SILU, torch.bfloat16, dev)
    run(x, groups, None, beta, fx.ACT_GELU, torch.float16, dev)


def test_every_activation_and_type(dev):
    for shape, groups in (((6, 144, 64), 8), ((300, 1, 384), 1), ((1, 20000, 64), 16)):
        for t in TYPES:
            x, gamma, beta = draw(shape, t, dev, seed=shape[1])
            for act in ACTS:
                for out in TYPES:
                    run(x, groups, gamma, beta, act, out, dev)


@pytest.mark.parametrize("Nb,P,C,groups", [(4, 1, 768, 1), (2, 49, 64, 8), (2, 3136, 64, 32), (1, 30000, 32, 4), (2, 50, 30, 5)])
def test_mean_far_from_zero(dev, Nb, P, C, groups):
    """The deviation a thousandth of the mean: a variance from the difference of two sums would be lost."""
    x, gamma, beta = draw((Nb, P, C), torch.float32, dev, seed=P, mean=0.0, spread=0.02)
    run(x + 20.0, groups, gamma, beta, fx.ACT_NONE, torch.float32, dev, eps=1e-8)
    first = x.clone()
    first[:, 0] += 1000.0       # an outlier in front
    run(first, groups, gamma, beta, fx.ACT_NONE, torch.float32, dev)


@pytest.mark.parametrize("Nb,P,C,groups", [(4, 1, 768, 1), (3, 49, 64, 8), (2, 3136, 64, 32), (1, 30000, 32, 4), (2, 50, 30, 5)])
def test_constant_and_special_values(dev, Nb, P, C, groups):
    x = torch.full((Nb, P, C), 3.0, dtype=torch.float16, device=dev)
    gamma, beta = torch.full((C,), 2.0, device=dev), torch.linspace(-1, 1, C, device=dev)
    y = fx.group_norm(x, groups, gamma, beta, out_dtype=torch.float32)
    assert bool(((y - beta).abs() <= 1e-5).all())
    # an infinity or a NaN spoils its own group and no other
    x, gamma, beta = draw((Nb, P, C), torch.float16, dev, seed=4)
    clean = fx.group_norm(x, groups, gamma, beta)
    cpg = C // groups
    for bad in (float("inf"), float("nan")):
        z = x.clone()
        z[0, P // 2, C - 1] = bad
        y = fx.group_norm(z, groups, gamma, beta)
        assert bool(y[0, :, C - cpg:].isnan().all())
        y[0, :, C - cpg:] = clean[0, :, C - cpg:]
        assert torch.equal(y, clean)
    # gamma and beta pass theirs on
    gamma = gamma.clone()
    gamma[1] = float("nan")
    y = fx.group_norm(x, groups, gamma, beta)
    assert bool(y[..., 1].isnan().all()) and int(y.isnan().sum()) == Nb * P


def test_in_place_views_and_shapes(dev):
    for shape, groups in (((2, 14, 14, 64), 8), ((50, 384), 1), ((1, 3, 100, 90, 32), 4)):
        for t in TYPES:
            x, gamma, beta = draw(shape, t, dev, seed=1)
            want = fx.group_norm(x, groups, gamma, beta, act=fx.ACT_SILU)
            assert want.shape == x.shape and want.dtype == t
            mine = x.clone()
            assert fx.group_norm(mine, groups, gamma, beta, act=fx.ACT_SILU, Y=mine) is mine
            assert torch.equal(mine, want)
            pad = 16 // x.element_size()                 # sixteen bytes past a 32-byte boundary
            odd = torch.empty(x.numel() + pad, dtype=t, device=dev)[pad:].view(shape)
            odd.copy_(x)
            assert odd.data_ptr() % 32 == 16
            assert torch.equal(fx.group_norm(odd, groups, gamma, beta, act=fx.ACT_SILU, Y=odd), want)


@pytest.mark.parametrize("Nb,P,C,groups,G", [(300, 1, 384, 1, 16), (1, 1, 64, 1, 16), (77, 1, 1024, 4, 32), (9, 1, 4096, 1, 16), (2, 196, 128, 32, 16), (3, 49, 512, 32, 64),
                                             (1, 3136, 64, 32, 16), (2, 100, 320, 32, 16), (1, 20000, 64, 8, 16), (5, 7, 48, 3, 16), (3, 2, 144, 9, 16)])
def test_slab_equals_the_two_calls(dev, Nb, P, C, groups, G):
    rng = np.random.default_rng(P + C)
    perm = rng.permutation(C // G).astype(np.int32)
    W = torch.from_numpy(rng.integers(-127, 128, (C, 32)).astype(np.int8)).to(dev)
    L = fx.Layer(W, torch.ones(32, device=dev), None, perm, rng.integers(0, 5, C // G).astype(np.uint8), G)
    for t in TYPES:
        x, gamma, beta = draw((Nb, P, C), t, dev, seed=P + 1)
        for ratio, act in ((0.0, fx.ACT_NONE), (0.5, fx.ACT_SILU), (0.3, fx.ACT_GELU), (1.0, fx.ACT_RELU)):
            L.set_lowbit_ratio(ratio)
            # scales of both quotient forms: the second one's significand lies next to a multiple of 2^17
            for xs in (float(np.float32(0.021)), float(np.float32((2 ** 23 + 2 ** 17 + 3) * 2.0 ** -29))):
                y = fx.group_norm(x, groups, gamma, beta, act=act, out_dtype=torch.float32)
                two = L.quantize_lower(y, xs)[0][:Nb * P * C].clone()
                slab, guard = helpers.with_guard(torch, (Nb * P * C,), torch.uint8, dev)
                assert L.group_norm_to_slab(x, groups, gamma, beta, xs, act=act, slab=slab) is slab
                torch.cuda.synchronize()
                guard()
                assert torch.equal(slab, two)
    z = x.clone()
    z.view(-1)[0] = float("nan")
    y = fx.group_norm(z, groups, gamma, beta, out_dtype=torch.float32)
    assert torch.equal(L.group_norm_to_slab(z, groups, gamma, beta, 0.02)[:Nb * P * C], L.quantize_lower(y, 0.02, slabs=(torch.empty_like(slab), None))[0])
    L.close()


def test_slab_in_use(dev):
    """The slab belongs to the ratio in force, and the layer's GEMM takes it."""
    c = inputs.ranged_linear("n", 300, 256, 48, 16, seed=2, group_structured=True)
    perm, sxg, _, _ = helpers.prepare_linear(c)
    L = mk(c, dev, perm, sxg)
    x, gamma, beta = draw((300, 256), torch.float16, dev, seed=8)
    L.set_lowbit_ratio(0.3)
    slab = L.group_norm_to_slab(x, 1, gamma, beta, 0.03)
    y = L.mixed_gemm(slab, None, 300, 0.03, 1.0, fx.OUT_DEQUANT_F32)
    q = oracle.quantize(fx.group_norm(x, 1, gamma, beta, out_dtype=torch.float32).cpu().numpy(), 0.03)
    perm, sxg, sxs, sw = helpers.prepare_linear(c)
    acc = oracle.mixed_gemm_acc(q, c.Wq, 16, perm, sxs, sw, oracle.n_low(0.3, 16))
    assert np.allclose(y.cpu().numpy(), oracle.epilogue_f32(acc, 0.03, c.w_scale, c.bias), rtol=1e-6, atol=0)
    L.set_lowbit_ratio(0.5)
    with pytest.raises(fx.FlexiqError):
        L.mixed_gemm(slab, None, 300, 0.03, 1.0, fx.OUT_DEQUANT_F32)
    L.close()


def test_refused(dev):
    x, gamma, beta = draw((4, 9, 64), torch.float16, dev, seed=8)

    def refused(call, code=fx.ERR_INVALID_ARG):
        with pytest.raises(fx.FlexiqError) as e:
            call()
        assert e.value.code == code
    refused(lambda: fx.group_norm(x, 7, gamma, beta))
    refused(lambda: fx.group_norm(x, 0, gamma, beta))
    refused(lambda: fx.group_norm(x, 8, gamma, beta, eps=0.0))
    refused(lambda: fx.group_norm(x, 8, gamma, beta, act=7))
    refused(lambda: fx.group_norm(x, 8, gamma.half(), beta))
    refused(lambda: fx.group_norm(x, 8, gamma, beta[:-1]))
    refused(lambda: fx.group_norm(x, 8, gamma.cpu(), beta))
    refused(lambda: fx.group_norm(x.transpose(0, 1), 8, gamma, beta))
    refused(lambda: fx.group_norm(x[0, 0], 8, gamma, beta))
    refused(lambda: fx.group_norm(x, 8, gamma, beta, Y=x.float(), out_dtype=torch.float16))
    refused(lambda: fx.group_norm(x, 8, gamma, beta, Y=x.view(torch.bfloat16)))
    refused(lambda: fx.group_norm(x, 8, gamma, beta, Y=x[:2]))
    refused(lambda: fx.group_norm(x.to(torch.float64), 8, gamma, beta))
    off = torch.empty(x.numel() + 1, dtype=torch.float16, device=dev)[1:].view(x.shape)
    refused(lambda: fx.group_norm(off, 8, gamma, beta))
    assert fx.group_norm(x[:0], 8, gamma, beta).shape == (0, 9, 64)
    assert fx.group_norm(x[:, :0].contiguous(), 8, gamma, beta).shape == (4, 0, 64)
    L = fx.Layer(torch.zeros(64, 16, dtype=torch.int8, device=dev), torch.ones(16, device=dev), None, np.arange(4, dtype=np.int32), np.zeros(4, np.uint8), 16)
    refused(lambda: L.group_norm_to_slab(x[..., :32].contiguous(), 8, gamma[:32], beta[:32], 0.1))
    refused(lambda: L.group_norm_to_slab(x, 8, gamma, beta, 0.0))
    refused(lambda: L.group_norm_to_slab(x, 8, gamma, beta, 0.1, slab=torch.empty(x.numel() - 1, dtype=torch.uint8, device=dev)))
    L.set_lowbit_path(fx.LOWBIT_PACKED_U4)
    refused(lambda: L.group_norm_to_slab(x, 8, gamma, beta, 0.1), fx.ERR_UNSUPPORTED)
    L.close()


def test_without_native_marshalling(dev, monkeypatch):
    for shape, groups in (((4, 9, 64), 8), ((1, 20000, 64), 8)):
        x, gamma, beta = draw(shape, torch.float16, dev, seed=8)
        want = fx.group_norm(x, groups, gamma, beta, act=fx.ACT_SILU)
        with monkeypatch.context() as m:
            m.setattr(fx, "_native_calls", lambda: None)
            assert torch.equal(fx.group_norm(x, groups, gamma, beta, act=fx.ACT_SILU), want)


def test_streams_and_graphs(dev):
    """Two side streams at once, and graphs that are replayed together on different streams: no scratch is shared."""
    shapes = [((2, 20000, 64), 8), ((2, 3136, 64), 32), ((500, 1, 768), 1)]
    for shape, groups in shapes:
        xs = [draw(shape, torch.bfloat16, dev, seed=s) for s in (1, 2)]
        wants = [fx.group_norm(x, groups, g, b, act=fx.ACT_SILU) for x, g, b in xs]
        streams = [torch.cuda.Stream() for _ in xs]
        torch.cuda.synchronize()
        outs, graphs = [None, None], []
        for _ in range(3):
            for i, (x, g, b) in enumerate(xs):
                with torch.cuda.stream(streams[i]):
                    outs[i] = fx.group_norm(x, groups, g, b, act=fx.ACT_SILU)
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, wants))
        held = []
        for x, g, b in xs:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held.append(fx.group_norm(x, groups, g, b, act=fx.ACT_SILU))
            graphs.append(graph)
        for _ in range(3):
            for h in held:
                h.zero_()
            torch.cuda.synchronize()
            for s, graph in zip(streams, graphs):
                with torch.cuda.stream(s):
                    graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o, w) for o, w in zip(held, wants))
        xs[0][0].mul_(-1)
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], fx.group_norm(xs[0][0], groups, xs[0][1], xs[0][2], act=fx.ACT_SILU))


@pytest.mark.parametrize("Nb,P,C,groups", [(1, 66000, 128, 32), (3, 30000, 64, 8), (24, 784, 256, 32), (600, 49, 128, 32), (500, 1, 768, 1)])
def test_calls_behind_one_another(dev, Nb, P, C, groups):
    """Kernels that begin before the ones in front of them have ended: the input rewritten before each call, the output normalised again in
    place, and nothing waited for in between, gives what a wait after every step gives."""
    x, gamma, beta = draw((Nb, P, C), torch.float16, dev, seed=11)
    other = torch.randn(Nb, P, C, device=dev).half()

    def steps(after):
        v, outs = x.clone(), []
        for i in range(6):
            v.add_(other, alpha=0.25)
            after()
            y = fx.group_norm(v, groups, gamma, beta, act=fx.ACT_SILU)
            after()
            fx.group_norm(y, groups, gamma, beta, Y=y)
            after()
            fx.group_norm(v, groups, None, beta, Y=v)
            after()
            outs.append(y)
        return outs + [v]

    want = steps(torch.cuda.synchronize)
    got = steps(lambda: None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_mlp_and_preactivation_chains(dev):
    """The operators in a row as a pre-norm block's MLP and as a pre-activation convolution block use them, against the same chain step by step
    through floating-point tensors."""
    a = inputs.ranged_linear("a", 300, 384, 512, 16, seed=21, group_structured=True)
    b = inputs.ranged_linear("b", 300, 512, 384, 16, seed=22, group_structured=True)
    A, B = (mk(c, dev, *helpers.prepare_linear(c)[:2]) for c in (a, b))
    x, gamma, beta = draw((300, 384), torch.float16, dev, seed=3)
    for ratio in (0.0, 0.3, 1.0):
        for L in (A, B):
            L.set_lowbit_ratio(ratio)
        s1 = A.group_norm_to_slab(x, 1, gamma, beta, 0.03)
        s2 = A.mixed_gemm_act_to_slab(s1, None, 300, 0.03, B, 0.05, fx.ACT_GELU)
        y = B.mixed_gemm_act(s2, None, 300, 0.05, fx.ACT_NONE, fx.OUT_DEQUANT_F16, residual=x)
        t4, t8, _ = A.quantize_lower(fx.group_norm(x, 1, gamma, beta, out_dtype=torch.float32), 0.03, slabs=(torch.empty_like(s1), torch.empty_like(s1)))
        h = A.mixed_gemm_act(t4, t8, 300, 0.03, fx.ACT_GELU, fx.OUT_DEQUANT_F32)
        u4, u8, _ = B.quantize_lower(h, 0.05, slabs=(torch.empty_like(s2), torch.empty_like(s2)))
        z = B.mixed_gemm_act(u4, u8, 300, 0.05, fx.ACT_NONE, fx.OUT_DEQUANT_F32) + x.float()
        assert torch.equal(y, z.half())
    A.close()
    B.close()
    c = inputs.resnet_conv("c", 3, 14, 64, 64, 3, seed=5)
    L = mk(c, dev, *helpers.prepare_conv(c)[:2], conv=True)
    L.set_lowbit_ratio(0.5)
    x, gamma, beta = draw((3, 14, 14, 64), torch.bfloat16, dev, seed=6)
    s = L.group_norm_to_slab(x, 16, gamma, beta, 0.02, act=fx.ACT_SILU)
    y = L.mixed_conv_act(s, None, 3, 14, 14, 0.02, fx.ACT_NONE, fx.OUT_DEQUANT_BF16, residual=x)
    n = fx.group_norm(x, 16, gamma, beta, act=fx.ACT_SILU, out_dtype=torch.float32)
    t4, t8, _ = L.quantize_lower(n, 0.02, slabs=(torch.empty_like(s), torch.empty_like(s)))
    z = L.mixed_conv(t4, t8, 3, 14, 14, 0.02, 1.0, fx.OUT_DEQUANT_F32) + x.float()
    assert torch.equal(y, z.bfloat16())
    L.close()
    fx.flexiq_check_status()


def test_offsets_beyond_32_bits(dev):
    """Tensors of more than 2^32 bytes, in place; one image larger than that; rows around the mark against a call on those alone."""
    x = torch.randn(9, 2 ** 21 + 77, 128, device=dev, dtype=torch.bfloat16)
    last = x[8:].clone()
    fx.group_norm(x, 32, act=fx.ACT_SILU, Y=x)
    check(x[8:], *want_and_tolerance(last, 32, None, None, 1e-5, fx.ACT_SILU))
    del x, last
    x = torch.randn(1, 2 ** 23 + 5, 256, device=dev, dtype=torch.bfloat16) + 1
    y = fx.group_norm(x, 32, act=fx.ACT_NONE)
    for g in (0, 17, 31):
        part = x[0, :, 8 * g:8 * g + 8].double()
        d = part - part.mean()
        ref = d / ((d * d).mean() + 1e-5).sqrt()
        assert float((y[0, :, 8 * g:8 * g + 8].double() - ref).abs().max()) < 0.03       # two bf16 steps of the largest value, about 6
    del x, y
    x = torch.randn(6_000_000, 768, device=dev, dtype=torch.float16)
    y = fx.group_norm(x, 1)
    for s in (slice(0, 100), slice(2 ** 32 // 1536 - 50, 2 ** 32 // 1536 + 50), slice(-100, None)):
        assert torch.equal(y[s], fx.group_norm(x[s].contiguous(), 1))
