"""xpress_linear without a GPU: refusals of the C entry and of the binding, and every
compiled variant launched by some call, on the stand-in for the CUDA runtime."""
import ctypes as C
import itertools

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD
from test_head_variants import _all_launched, _library

torch = pytest.importorskip("torch")
BAD, UNS, WSP, OK = X.XPRESS_ERR_INVALID_ARG, X.XPRESS_ERR_UNSUPPORTED, X.XPRESS_ERR_WORKSPACE, X.XPRESS_OK


@pytest.fixture(scope="module")
def lib():
    BLD.build()
    return X.load()


def _args(**kw):
    # addresses are never followed: the checks come first
    g = X.XpressLinearArgs(M=3, N=100, K=256, out_dtype=X.XPRESS_BF16, act=X.XPRESS_ACT_SILU, x=4096, ldx=256, w=4096, ldw=256,
                           bias=4096, residual=4096, ldr=100, out=4096, ldo=100)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("kw, want", [
    (dict(x=None), BAD), (dict(w=None), BAD), (dict(out=None), BAD), (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD),
    (dict(ldx=255), BAD), (dict(ldx=260), BAD), (dict(ldw=248), BAD), (dict(ldw=260), BAD), (dict(x=4104), BAD),
    (dict(w=4104), BAD), (dict(ldo=99), BAD), (dict(ldr=99), BAD), (dict(out=4097), BAD), (dict(bias=4097), BAD),
    (dict(residual=4097), BAD), (dict(out_dtype=X.XPRESS_F32, out=4098), BAD), (dict(out_dtype=X.XPRESS_F32, residual=4098), BAD),
    (dict(out_dtype=5), UNS), (dict(act=3), UNS), (dict(act=-2), UNS), (dict(K=(1 << 24) + 8, ldx=1 << 25, ldw=1 << 25), UNS),
    (dict(M=(1 << 30) + 1), UNS), (dict(N=(1 << 30) + 1, ldo=1 << 31, ldr=1 << 31), UNS), (dict(M=0), OK)])
def test_refusals(lib, kw, want):
    assert lib.xpress_linear(_args(**kw), 4096, 256, None) == want


def test_workspace_refusals(lib):
    size = lib.xpress_linear_workspace_size()
    for ws, n in ((None, size), (4096, size - 1), (4096 + 16, size)):
        assert lib.xpress_linear(_args(), ws, n, None) == WSP
    assert lib.xpress_linear(None, 4096, size, None) == BAD


def test_the_refiner_refuses_no_activation(lib):
    """XPRESS_ACT_NONE is xpress_linear's only."""
    w = X.XpressWeights(4096, 151936, 256, 16, X.XPRESS_BF16, X.XPRESS_ACT_NONE, *[C.c_void_p(16)] * 8)
    assert lib.xpress_refiner_create(C.byref(w), None, C.byref(C.c_void_p())) == UNS


def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


@pytest.mark.parametrize("call", [
    lambda: X.linear(_bf(2, 16), _bf(5, 24), _bf(2, 5)),                               # K differs
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 6)),                               # out's shape
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(3, 5)),
    lambda: X.linear(_bf(2, 16).float(), _bf(5, 16), _bf(2, 5)),                       # x's type
    lambda: X.linear(_bf(2, 16), _bf(5, 16).half(), _bf(2, 5)),
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5).half()),
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5), bias=_bf(4)),
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5), bias=_bf(5).float()),
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5), residual=_bf(2, 5).float()),   # residual's type
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5), residual=_bf(2, 6)),
    lambda: X.linear(_bf(16, 2).t(), _bf(5, 16), _bf(2, 5)),                           # columns not contiguous
    lambda: X.linear(_bf(2, 16), _bf(5, 16), _bf(2, 5)),                               # device
])
def test_binding_refuses(lib, call):
    with pytest.raises(ValueError):
        call()


def test_variants(tmp_path):
    lib = _library(tmp_path, "linear", "linear_wide")
    lib.xpress_linear.argtypes = [C.POINTER(X.XpressLinearArgs), C.c_void_p, C.c_size_t, C.c_void_p]
    for dt, M, (N, K) in itertools.product((X.XPRESS_F32, X.XPRESS_BF16), (1, 16, 24, 50, 100, 200, 300, 2000),
                                           ((4096, 4096), (500, 16384), (38912, 520))):
        g = _args(out_dtype=dt, M=M, N=N, K=K, ldx=K, ldw=K, ldo=N, ldr=N)
        assert lib.xpress_linear(g, 4096, 256, None) == X.XPRESS_OK
    _all_launched(lib)


def test_in_place_needs_the_same_pitch(lib):
    """out over residual in rows of another pitch: an output would replace another row's residual."""
    assert lib.xpress_linear(_args(ldr=104), 4096, 256, None) == BAD
    assert lib.xpress_linear(_args(ldo=104), 4096, 256, None) == BAD
