"""Group normalisation where an image's pieces end with the image, where a thread has thousands of them, and where squares leave fp32.

Tolerances as in test_gpu_group_norm."""
import numpy as np
import pytest
import torch

import helpers
from paper_2510_02822_b200 import binding as fx
from test_gpu_group_norm import check, draw, run, want_and_tolerance

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def dev():
    return torch.device("cuda:0")


# On 148 SMs these images are cut in more pieces than their positions fill, the last full pair of them ending with the image.
@pytest.mark.parametrize("P,C,groups,t", [(6600, 512, 4, F16), (8712, 512, 32, BF16), (10920, 256, 32, F16), (9800, 320, 32, F16), (9604, 320, 32, BF16), (4000, 640, 1, F16),
                                          (6724, 192, 32, F32), (10270, 128, 32, F32), (33282, 128, 32, F16), (984, 435, 1, F16), (21316, 256, 32, F16)])
def test_pieces_that_end_with_the_image(dev, P, C, groups, t):
    x, gamma, beta = draw((1, P, C), t, dev, seed=P)
    run(x, groups, gamma, beta, fx.ACT_SILU, t, dev)
    y = run(x, groups, gamma, beta, fx.ACT_NONE, F32, dev)
    mine = x.clone()
    fx.group_norm(mine, groups, gamma, beta, act=fx.ACT_SILU, Y=mine)
    assert torch.equal(mine, fx.group_norm(x, groups, gamma, beta, act=fx.ACT_SILU))
    if C % 16 == 0:
        L = fx.Layer(torch.zeros(C, 16, dtype=torch.int8, device=dev), torch.ones(16, device=dev), None, np.arange(C // 16, dtype=np.int32), np.full(C // 16, 2, np.uint8), 16)
        L.set_lowbit_ratio(0.5)
        two = L.quantize_lower(y, 0.02)[0][:P * C].clone()
        assert torch.equal(L.group_norm_to_slab(x, groups, gamma, beta, 0.02, slab=torch.empty(P * C, dtype=torch.uint8, device=dev)), two)
        L.close()


def test_every_length_of_an_image(dev):
    """One image of every length around the cuts, scalar and wide, by its sum of squares: NaN anywhere would show."""
    for C, groups, t, lengths in ((512, 32, F16, range(6500, 6720, 7)), (128, 1, F32, range(10200, 10360, 5)), (435, 1, F16, range(900, 1060, 4))):
        x, _, _ = draw((1, max(lengths), C), t, dev, seed=C)
        for P in lengths:
            y = fx.group_norm(x[:, :P], groups, out_dtype=F32)
            assert abs(float(y.double().square().mean()) - 1) < 1e-4


@pytest.mark.parametrize("P,C,groups,t", [(65539, 64, 32, F32), (131075, 64, 8, BF16), (65539, 64, 4, F32)])
def test_an_outlier_in_front_of_a_long_image(dev, P, C, groups, t):
    """Thousands of values a thread, the first of them far from all others: as many images as let a block take a whole one."""
    x = torch.randn(296, P, C, device=dev, dtype=t)
    x[:, 0, ::C // groups] = 30000.0
    y = fx.group_norm(x, groups, out_dtype=t)
    for i in (0, 100, 295):
        check(y[i:i + 1], *want_and_tolerance(x[i:i + 1], groups, None, None, 1e-5, fx.ACT_NONE))


# the three ways of cutting an image, in pieces of one group and of several, wide and scalar
KINDS = [(40, 1, 768, 1), (3, 1, 3000, 1), (6, 1, 77, 1), (3, 49, 64, 8), (2, 3136, 64, 32), (2, 50, 30, 5), (2, 64, 2056, 8), (1, 30000, 32, 4), (2, 40000, 64, 32), (1, 40000, 12, 3),
         (1, 984, 435, 1), (1, 66000, 128, 32)]


@pytest.mark.parametrize("Nb,P,C,groups", KINDS)
def test_squares_beyond_fp32(dev, Nb, P, C, groups):
    """Deviations whose squares leave fp32: the variance is infinite, and what is normalised is zero.  Both where the values of a channel differ and
    where only the channels of a group do."""
    beta = torch.linspace(-2, 2, C, device=dev)
    want = beta.expand(Nb, P, C)
    g = torch.Generator(device=dev)
    g.manual_seed(P + C)
    sign = (torch.randint(0, 2, (Nb, P, C), generator=g, device=dev) * 2 - 1).float()
    sign[..., 0::C // groups], sign[..., 1::C // groups] = 1.0, -1.0          # (no group of one sign alone)
    for t in (F32, BF16):
        for x in (sign, sign[:1, :1].expand(Nb, P, C)):
            y = fx.group_norm((x * 2.0 ** 66).to(t).contiguous(), groups, None, beta, out_dtype=F32)
            assert torch.equal(y, want)


@pytest.mark.parametrize("C,groups", [(64, 8), (64, 32)])
def test_squares_beyond_fp32_where_all_means_agree(dev, C, groups):
    """As many images as let a block take a whole one of 4096 positions, sixteen side by side: the first eight pieces of every thread are 2^66, the
    next eight its negative, and so on.  Each thread's distances from its first pieces' mean have a sum and squares that cancel but for infinities."""
    x = torch.where(torch.arange(4096, device=dev) // 128 % 2 == 0, 2.0 ** 66, -2.0 ** 66)[None, :, None].expand(296, 4096, C).contiguous()
    beta = torch.linspace(-2, 2, C, device=dev)
    y = fx.group_norm(x, groups, None, beta)
    assert torch.equal(y, beta.expand(296, 4096, C))
