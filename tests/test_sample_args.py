"""xpress_sample without a GPU: refusals of the C entry and of the binding, every compiled
variant launched by some call, and calls on several devices, on the stand-in for the CUDA
runtime."""
import ctypes as C
import itertools

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD
from test_head_variants import _all_launched, _library

torch = pytest.importorskip("torch")
BAD, UNS, OK = X.XPRESS_ERR_INVALID_ARG, X.XPRESS_ERR_UNSUPPORTED, X.XPRESS_OK


@pytest.fixture(scope="module")
def lib():
    BLD.build()
    return X.load()


def _args(**kw):
    # addresses are never followed: the checks come first
    g = X.XpressSampleArgs(n_seq=2, rows=3, V=1000, dtype=X.XPRESS_BF16, logits=4096, ld=1000, temperature=4096, top_k=4096,
                           top_p=4096, min_p=4096, u=4096, tokens=4096, out=8192, ldo=1000, mask_value=-8192.0)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("kw, want", [
    (dict(logits=None), BAD), (dict(temperature=None), BAD), (dict(tokens=None, out=None), BAD), (dict(u=None), BAD),
    (dict(n_seq=-1), BAD), (dict(rows=0), BAD), (dict(V=0), BAD), (dict(ld=999), BAD), (dict(ldo=999), BAD),
    (dict(logits=4097), BAD), (dict(out=4097), BAD), (dict(tokens=4098), BAD), (dict(u=4098), BAD), (dict(temperature=4097), BAD),
    (dict(top_k=4097), BAD), (dict(top_p=4097), BAD), (dict(min_p=4097), BAD), (dict(dtype=X.XPRESS_F32, logits=4098), BAD),
    (dict(dtype=3), UNS), (dict(V=(1 << 24) + 1, ld=1 << 25, ldo=1 << 25), UNS), (dict(n_seq=1 << 20, rows=1 << 8), UNS),
    (dict(n_seq=0), OK)])
def test_refusals(lib, kw, want):
    assert lib.xpress_sample(_args(**kw), None) == want


def test_null_argument_block(lib):
    assert lib.xpress_sample(None, None) == BAD


def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _f32(*shape):
    return torch.zeros(shape)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: X.sample(_bf(5, 8), _f32(2), out=_bf(5, 8), rows=2),                       # rows do not divide
    lambda: X.sample(_bf(4, 8), _f32(3), out=_bf(4, 8)),
    lambda: X.sample(_bf(4, 8), _f32(4), out=_f32(4, 8)),                              # out's type
    lambda: X.sample(_bf(4, 8).half(), _f32(4), out=_bf(4, 8).half()),
    lambda: X.sample(_bf(4, 8), _f32(4), tokens_out=_i32(4)),                          # no numbers
    lambda: X.sample(_bf(4, 8), _f32(4), u=_f32(3), tokens_out=_i32(4)),
    lambda: X.sample(_bf(4, 8), _f32(4), u=_f32(4), tokens_out=_i32(4).long()),
    lambda: X.sample(_bf(4, 8), _f32(4), out=_bf(4, 8), top_k=_f32(4)),
    lambda: X.sample(_bf(4, 8), _f32(4), out=_bf(4, 8), top_p=_f32(8)[::2]),
    lambda: X.sample(_bf(4, 8), _f32(2), out=_bf(4, 8), rows=2, min_p=_f32(4)),
    lambda: X.sample(_bf(8, 4).t(), _f32(4), out=_bf(4, 8)),                           # columns not contiguous
    lambda: X.sample(_bf(4, 8), _f32(4), out=_bf(4, 8))])                              # device
def test_binding_refuses(lib, call):
    with pytest.raises(ValueError):
        call()


def _fake(tmp_path):
    lib = _library(tmp_path, "sample")
    lib.xpress_sample.argtypes = [C.POINTER(X.XpressSampleArgs), C.c_void_p]
    return lib


def test_variants(tmp_path):
    lib = _fake(tmp_path)
    for dt, V in itertools.product((X.XPRESS_F32, X.XPRESS_BF16), (1000, 151936, 1 << 22)):
        assert lib.xpress_sample(_args(dtype=dt, V=V, ld=V, ldo=V), None) == OK
    _all_launched(lib)


@pytest.mark.parametrize("n, V, most", [(1, 151936, 8), (1, 100, 1), (600, 151936, 8), (600, 2000, 1), (1, 1 << 24, 8)])
def test_cluster_sizes(tmp_path, n, V, most):
    lib = _fake(tmp_path)
    for dev in (0, 1, 69, 0):
        lib.fake_use(dev)
        before = lib.fake_launches()
        assert lib.xpress_sample(_args(n_seq=n, rows=1, V=V, ld=V, ldo=V), None) == OK
        assert lib.fake_launches() == before + 1 and lib.fake_last_cluster() <= most


def test_in_place_needs_the_same_pitch(lib):
    """out over logits in rows of another pitch: a written row would replace another one's logits."""
    assert lib.xpress_sample(_args(out=4096, ldo=1008), None) == BAD
    assert lib.xpress_sample(_args(out=4096, ld=1001), None) == BAD
