"""Refusals of the operators between the quantized layers that need no device."""
import ctypes as C

import pytest
import torch

from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import build as fxbuild


@pytest.fixture(scope="module")
def lib():
    fxbuild.build_library()
    return fx.lib()


P16 = C.c_void_p(4096)      # never dereferenced: the checks come first
ODD = C.c_void_p(4100)


def test_dead_handles(lib):
    assert lib.flexiq_mixed_gemm_act(None, None, None, None, 1, 1.0, 1.0, 0, None, 0, 0, 2, None, None) == fx.ERR_INVALID_ARG
    assert lib.flexiq_mixed_conv_act(None, None, None, None, 1, 1, 1, 1.0, 1.0, 0, None, 0, 0, 2, None, None) == fx.ERR_INVALID_ARG
    assert lib.flexiq_mixed_gemm_act_to_slab(None, None, None, None, 1, 1.0, None, 1.0, 0, 0, None, None) == fx.ERR_INVALID_ARG
    assert lib.flexiq_mixed_conv_act_to_slab(None, None, None, None, 1, 1, 1, 1.0, None, 1.0, 0, 0, None, None) == fx.ERR_INVALID_ARG
    assert lib.flexiq_group_norm_to_slab(None, P16, 0, 1, 1, 1, None, None, 1e-5, 0, 1.0, P16, None, None) == fx.ERR_INVALID_ARG
    assert "handle" in fx.last_error()


@pytest.mark.parametrize("change, message", [
    (dict(x_dtype=3), "x_dtype"), (dict(x_dtype=-1), "x_dtype"), (dict(y_dtype=3), "y_dtype"), (dict(Nb=-1), "Nb"), (dict(P=-1), "P = -1"),
    (dict(C=0), "multiple"), (dict(groups=0), "multiple"), (dict(groups=3), "multiple"), (dict(groups=64), "multiple"), (dict(Nb=1 << 40, P=1 << 30), "64 bits"),
    (dict(act=5), "act"), (dict(act=-1), "act"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(X=None), "NULL"), (dict(Y=None), "NULL"), (dict(X=ODD), "aligned"), (dict(Y=ODD), "aligned"), (dict(gamma=ODD), "aligned"), (dict(beta=ODD), "aligned"),
    (dict(y_dtype=1, Y=P16), "same type")])
def test_group_norm_arguments(lib, change, message):
    a = dict(X=P16, x_dtype=0, Nb=2, P=4, C=32, groups=4, gamma=None, beta=None, eps=1e-5, act=0, y_dtype=0, Y=C.c_void_p(8192), scratch=None, stream=None)
    a.update(change)
    assert lib.flexiq_group_norm(*a.values()) == fx.ERR_INVALID_ARG
    assert message in fx.last_error()


def test_group_norm_nothing_to_do(lib):
    assert lib.flexiq_group_norm(None, 0, 0, 4, 32, 4, None, None, 1e-5, 0, 0, None, None, None) == fx.OK
    assert lib.flexiq_group_norm(None, 0, 4, 0, 32, 4, None, None, 1e-5, 0, 0, None, None, None) == fx.OK


def test_scratch_size(lib):
    assert fx.flexiq_group_norm_scratch(fx.DTYPE_F16, 1, 49, 512, 32) == 0 and fx.flexiq_group_norm_scratch(fx.DTYPE_F16, 0, 1 << 20, 64, 32) == 0
    assert fx.flexiq_group_norm_scratch(fx.DTYPE_F16, 3, 1 << 20, 64, 32) >= 3 * 32 * 8
    for bad in [(3, 1, 1, 32, 4), (0, -1, 1, 32, 4), (0, 1, 1, 32, 5), (0, 1, 1, 0, 1)]:
        with pytest.raises(fx.FlexiqError):
            fx.flexiq_group_norm_scratch(*bad)
    assert lib.flexiq_group_norm_scratch(0, 1, 1, 32, 4, None) == fx.ERR_INVALID_ARG


def test_python_refusals(lib, monkeypatch):
    x = torch.zeros(2, 4, 32)
    for native in (fx._native_calls, lambda: None):
        monkeypatch.setattr(fx, "_native_calls", native)
        for bad in (lambda: fx.group_norm(x, 4), lambda: fx.group_norm(x, 4, out_dtype=torch.int8), lambda: fx.group_norm(x.int(), 4)):
            with pytest.raises(fx.FlexiqError) as e:
                bad()
            assert e.value.code == fx.ERR_INVALID_ARG
