"""The 8-bit values of xpress_quantize_weight and xpress_rmsnorm, element by element:
e4m3 (nearest even) of the fp32 quotient of the value and the stored scale, over all
scales, on values that lie half way between two e4m3 values by design.

The quotient's reference is rounded to fp32 from 64 bits, which is the rounded quotient
of two fp32 numbers (53 bits hold more than twice 24)."""
import numpy as np
import pytest

import test_gpu_head as G

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
X = G.X                                          # the module's fixture


def _e4m3(v, s):
    return (v.double() / s.double()).float().to(torch.float8_e4m3fn).float()


def _spread(s, rows, cols):
    return s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def _midpoints():
    """What lies half way between neighbouring e4m3 values, in fp32 (5 bits)."""
    v = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    return ((v[1:] + v[:-1]) / 2).astype(np.float32)


@pytest.mark.parametrize("lo, hi", [(-126, -118), (-118, -100), (-100, -60), (-20, -2), (-2, 20), (90, 118)])
@pytest.mark.parametrize("cols", [512, 515])
def test_quantised_ties(X, cols, lo, hi):
    rng = np.random.Generator(np.random.PCG64(cols + lo + 200))
    rows, nr, nc = 1030, 9, -(-cols // 128)
    # scales of at most 16 bits, so that a midpoint times the scale is exact, and 448 times it
    s = np.ldexp(1 + rng.integers(0, 2 ** 15, (nr, nc)) / 2.0 ** 15, rng.integers(lo, hi, (nr, nc))).astype(np.float32)
    s[::2] = np.ldexp(1 + rng.integers(0, 16, s[::2].shape) / 16.0, rng.integers(lo, hi, s[::2].shape))
    big = np.repeat(np.repeat(s, 128, 0)[:rows], 128, 1)[:, :cols].astype(np.float64)
    W = (rng.choice(_midpoints(), (rows, cols)) * rng.choice([-1.0, 1.0], (rows, cols)) * big).astype(np.float32)
    near = rng.random((rows, cols)) < 0.2
    W[near] = np.nextafter(W[near], np.float32(0))
    W[::128, ::128] = (448 * s.astype(np.float64)).astype(np.float32)
    W = torch.from_numpy(W).cuda()
    q, sc = X.quantize_weight(W)
    assert torch.equal(sc, torch.from_numpy(s).cuda())
    want = _e4m3(W, _spread(sc, rows, cols))
    assert int((q.float() != want).sum()) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [512, 515])
@pytest.mark.parametrize("size", [1e-37, 1e-34, 1e-30, 0.02, 1e30])
def test_quantised_values(X, size, cols, dtype):
    W = (torch.randn((1030, cols), device="cuda", generator=G._gen(cols), dtype=torch.float64) * size).to(dtype)
    q, sc = X.quantize_weight(W)
    assert int((q.float() != _e4m3(W, _spread(sc, 1030, cols))).sum()) == 0


@pytest.mark.parametrize("H", [512, 514, 515, 20001])
@pytest.mark.parametrize("size", [1e-36, 1e-33, 1.0, 1e30])
def test_normed_values(X, size, H):
    """From the stored y, which in fp32 is the y that the scales and q are made of."""
    x = torch.randn((200, H), device="cuda", generator=G._gen(H))
    w = torch.full((H,), size, device="cuda")
    y, q, s = torch.empty_like(x), X.alloc_e4m3(200, H), torch.empty((200, -(-H // 128)), device="cuda")
    X.rmsnorm(x, w, 1e-6, y_out=y, q_out=q, scale_out=s)
    assert int((q.float() != _e4m3(y, s.repeat_interleave(128, 1)[:, :H])).sum()) == 0
