"""Refusals of the 8-bit drafter head's entry points, without a GPU: the C ABI
returns before any CUDA call, the binding raises before the library is
called."""
import ctypes as C

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD

torch = pytest.importorskip("torch")
BAD, UNS, WSP, OK = X.XPRESS_ERR_INVALID_ARG, X.XPRESS_ERR_UNSUPPORTED, X.XPRESS_ERR_WORKSPACE, X.XPRESS_OK


@pytest.fixture(scope="module")
def lib():
    BLD.build()
    return X.load()


def _set(args, **kw):
    for k, v in kw.items():
        setattr(args, k, v)
    return args


def _norm(**kw):
    # addresses are never followed: the checks come first
    a = X.XpressNormArgs(rows=4, H=256, dtype=X.XPRESS_BF16, eps=1e-6, x=4096, ldx=256, residual=8192, ldr=256,
                         weight=4096, sum=8192, lds=256, y=4096, ldy=256, q=4096, ldq=256, scale=4096, ldscale=2)
    return _set(a, **kw)


@pytest.mark.parametrize("kw, want", [
    (dict(x=None), BAD), (dict(weight=None), BAD), (dict(rows=-1), BAD), (dict(H=0), BAD),
    (dict(sum=None, y=None, q=None), BAD), (dict(scale=None), BAD), (dict(ldx=255), BAD), (dict(ldr=255), BAD),
    (dict(lds=255), BAD), (dict(ldy=255), BAD), (dict(ldq=255), BAD), (dict(ldscale=1), BAD), (dict(x=4097), BAD),
    (dict(scale=4098), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(dtype=2), UNS),
    (dict(rows=0), OK)])
def test_norm_refusals(lib, kw, want):
    assert lib.xpress_rmsnorm(_norm(**kw), None) == want


def test_null_argument_blocks(lib):
    assert lib.xpress_rmsnorm(None, None) == BAD
    assert lib.xpress_matmul_fp8(None, None, 0, None) == BAD
    assert lib.xpress_process_logits(None, None, 0, None) == BAD


@pytest.mark.parametrize("kw, want", [
    (dict(W=None), BAD), (dict(q=None), BAD), (dict(scale=None), BAD), (dict(rows=-1), BAD), (dict(cols=0), BAD),
    (dict(ldw=255), BAD), (dict(ldq=255), BAD), (dict(W=4097), BAD), (dict(dtype=7), UNS),
    (dict(rows=2 ** 31 - 1, cols=2 ** 21, ldw=2 ** 21, ldq=2 ** 21), UNS), (dict(rows=0), OK)])
def test_quantize_refusals(lib, kw, want):
    a = dict(W=4096, dtype=X.XPRESS_BF16, rows=4, cols=256, ldw=256, q=4096, ldq=256, scale=4096)
    a.update(kw)
    assert lib.xpress_quantize_weight(*a.values(), None) == want


@pytest.mark.parametrize("kw, want", [
    (dict(a=None), BAD), (dict(w=None), BAD), (dict(a_scale=None), BAD), (dict(w_scale=None), BAD),
    (dict(out=None), BAD), (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(lda=200), BAD),
    (dict(lda=264), BAD), (dict(ldw=264), BAD), (dict(a=4104), BAD), (dict(w=4104), BAD), (dict(ldo=99), BAD),
    (dict(ld_a_scale=1), BAD), (dict(ld_w_scale=1), BAD), (dict(out=4097), BAD), (dict(out_dtype=5), UNS),
    (dict(K=65537, lda=65552, ldw=65552, ld_a_scale=513, ld_w_scale=513), UNS), (dict(M=0), OK)])
def test_matmul_refusals(lib, kw, want):
    g = X.XpressMatmulArgs(M=3, N=100, K=256, out_dtype=X.XPRESS_BF16, a=4096, lda=256, a_scale=4096, ld_a_scale=2,
                           w=4096, ldw=256, w_scale=4096, ld_w_scale=2, out=4096, ldo=100)
    assert lib.xpress_matmul_fp8(_set(g, **kw), 4096, 256, None) == want


def test_matmul_workspace_refusals(lib):
    g = X.XpressMatmulArgs(M=3, N=100, K=256, out_dtype=X.XPRESS_BF16, a=4096, lda=256, a_scale=4096, ld_a_scale=2,
                           w=4096, ldw=256, w_scale=4096, ld_w_scale=2, out=4096, ldo=100)
    size = lib.xpress_matmul_fp8_workspace_size()
    for ws, n in ((None, size), (4096, size - 1), (4096 + 16, size)):
        assert lib.xpress_matmul_fp8(g, ws, n, None) == WSP


def _logits(**kw):
    g = X.XpressLogitsArgs(n_seq=2, rows=3, V=1000, dtype=X.XPRESS_BF16, logits=4096, ld=1000, out=8192, ldo=1000,
                           argmax=4096, repetition=4096, history=4096, n_history=10, history_offsets=4096,
                           prompt_len=4096, draft=4096, ld_draft=2, bias_ids=4096, bias_values=4096, n_bias=4,
                           bias_offsets=4096, mask=4096, ld_mask=32, mask_rows=6, mask_row=4096, mask_value=-1e30)
    return _set(g, **kw)


@pytest.mark.parametrize("kw, want", [
    (dict(logits=None), BAD), (dict(out=None, argmax=None), BAD), (dict(n_seq=-1), BAD), (dict(rows=0), BAD),
    (dict(V=0), BAD), (dict(ld=999), BAD), (dict(ldo=999), BAD), (dict(history_offsets=None), BAD),
    (dict(n_history=-1), BAD), (dict(bias_values=None), BAD), (dict(bias_offsets=None), BAD), (dict(n_bias=-1), BAD),
    (dict(ld_draft=1), BAD), (dict(ld_mask=31), BAD), (dict(mask_rows=-1), BAD), (dict(logits=4097), BAD),
    (dict(history_offsets=4100), BAD), (dict(mask_row=4098), BAD), (dict(dtype=3), UNS), (dict(n_seq=65536), UNS),
    (dict(V=(1 << 24) + 1, ld=1 << 25, ldo=1 << 25, ld_mask=1 << 20), UNS), (dict(n_history=(1 << 30) + 1), UNS),
    (dict(n_bias=(1 << 30) + 1), UNS),
    (dict(n_seq=0), OK)])
def test_logits_refusals(lib, kw, want):
    size = 1 << 24
    assert lib.xpress_process_logits(_logits(**kw), 1 << 20, size, None) == want


def test_logits_workspace_refusals(lib):
    size = lib.xpress_process_logits_workspace_size(2, 3, 1000)
    assert size > 0 and lib.xpress_process_logits_workspace_size(0, 3, 1000) == 0
    for ws, n in ((None, size), (1 << 20, size - 1), ((1 << 20) + 16, size)):
        assert lib.xpress_process_logits(_logits(), ws, n, None) == WSP


# The binding's own checks, on CPU tensors (they are refused last, for their device).

def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _f32(*shape):
    return torch.zeros(shape)


def _q(*shape):
    return torch.zeros(shape, dtype=torch.float8_e4m3fn)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda: X.rmsnorm(_bf(4, 8), _bf(7), y_out=_bf(4, 8)),                             # weight's length
    lambda: X.rmsnorm(_bf(4, 8), _f32(8), y_out=_bf(4, 8)),                            # weight's type
    lambda: X.rmsnorm(_bf(4, 8), _bf(8), y_out=_f32(4, 8)),                            # output's type
    lambda: X.rmsnorm(_bf(4, 8), _bf(8), residual=_bf(3, 8), y_out=_bf(4, 8)),         # residual's shape
    lambda: X.rmsnorm(_bf(8, 4).t(), _bf(8), y_out=_bf(4, 8)),                         # columns not contiguous
    lambda: X.rmsnorm(_bf(4, 8), _bf(8), q_out=_q(4, 8)),                              # q without scales
    lambda: X.rmsnorm(_bf(4, 8).half(), _bf(8).half(), y_out=_bf(4, 8)),               # dtype
    lambda: X.rmsnorm(_bf(8), _bf(8), y_out=_bf(8)),                                   # rank
    lambda: X.rmsnorm(_bf(4, 8), _bf(8), y_out=_bf(4, 8)),                             # device
    lambda: X.quantize_weight(_bf(8)),
    lambda: X.quantize_weight(_bf(4, 8), _q(4, 9), _f32(1, 1)),
    lambda: X.quantize_weight(_bf(300, 8), _q(300, 8), _f32(3, 2)[:, :1]),             # scales not contiguous
    lambda: X.quantize_weight(_bf(4, 8), _q(4, 8), _f32(1, 1)),                        # device
    lambda: X.matmul_fp8(_q(2, 16), _f32(2, 1), _q(5, 32), _f32(1, 1), _bf(2, 5)),     # K differs
    lambda: X.matmul_fp8(_q(2, 16), _f32(2, 2), _q(5, 16), _f32(1, 1), _bf(2, 5)),     # scales' shape
    lambda: X.matmul_fp8(_q(2, 16), _f32(2, 1), _q(5, 16), _f32(1, 1), _bf(2, 6)),     # out's shape
    lambda: X.matmul_fp8(_bf(2, 16), _f32(2, 1), _q(5, 16), _f32(1, 1), _bf(2, 5)),    # a's type
    lambda: X.matmul_fp8(_q(2, 16), _f32(2, 1), _q(5, 16), _f32(1, 1), _bf(2, 5)),     # device
    lambda: X.process_logits(_bf(5, 8), _bf(5, 8), rows=2),                            # rows do not divide
    lambda: X.process_logits(_bf(4, 8), _f32(4, 8)),
    lambda: X.process_logits(_bf(4, 8), None, _i32(3)),
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), repetition=_f32(3)),
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), history=_i32(5)),                   # no offsets
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), history=_i32(5), history_offsets=_i32(5)),
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), rows=2, draft=_i32(2, 0)),          # too few draft tokens
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), bias_ids=_i32(5)),
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), mask=_i32(4, 2)),                   # words per row
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8), mask=_i32(4, 1), mask_row=_i32(3)),
    lambda: X.process_logits(_bf(4, 8), _bf(4, 8))])                                   # device
def test_binding_refuses(lib, call):
    with pytest.raises(ValueError):
        call()


def test_e4m3_rows_start_on_16_bytes():
    q = X.alloc_e4m3(3, 100, device="cpu")
    assert q.shape == (3, 100) and q.stride() == (112, 1)
