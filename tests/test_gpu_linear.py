"""xpress_linear on the GPU against its definition in 64 bits: sizes that fit no tile,
every split of K, types, strides, in place, on other streams and in captured graphs.

Tolerances, before the output's rounding: products of two bf16 are exact in fp32; a sum
of K of them in any order, an addition that may truncate off by 2^-23, is off by at most
K 2^-23 sum |x w|.  Every activation's slope is below 1.13.  The bias, the residual and
the activation's own steps round 2^-24 of what they add; SiLU for bf16 outputs takes the
fast exponential (2^-21 + |t| 2^-22 of the result) and a division 2 ulp off, GELU erfc 4
ulp off.  The output's rounding is eps / 2 of the value."""
import math

import pytest
import torch

from paper_2608_02438_gb300 import binding as X

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
NONE, SILU, GELU, RELU = X.XPRESS_ACT_NONE, X.XPRESS_ACT_SILU, X.XPRESS_ACT_GELU, X.XPRESS_ACT_RELU


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_02438_gb300 import build as BLD
    BLD.build()
    yield
    assert X.matmul_fp8_status() == X.XPRESS_OK


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def operand(rows, cols, g, scale=1.0, pad=0):
    t = torch.empty((rows, -(-cols // 8) * 8 + pad), dtype=BF16, device="cuda")
    t.fill_(float("nan"))                                     # the padding is never used
    t[:, :cols] = (torch.randn((rows, cols), device="cuda", generator=g) * scale).to(BF16)
    return t[:, :cols]


def like(rows, cols, dt, pad=0):
    return torch.full((rows, cols + pad), 7.0, dtype=dt, device="cuda")[:, :cols]


def activation(act, t):
    if act == SILU:
        return t / (1.0 + torch.exp(-t))
    if act == GELU:
        return 0.5 * t * torch.erfc(-t / math.sqrt(2.0))
    return t.clamp(min=0.0) if act == RELU else t


def check(out, x, w, bias=None, act=NONE, residual=None):
    xd, wd = x.double(), w.double()
    t = xd @ wd.t()
    mag = xd.abs() @ wd.abs().t()
    if bias is not None:
        t = t + bias.double()
        mag = mag + bias.double().abs()
    a = activation(act, t)
    want = a if residual is None else a + residual.double()
    tol = 1.13 * (x.shape[1] + 2) * 2.0 ** -23 * mag
    if act == SILU:
        tol = tol + (2.0 ** -20 + (1.0 + t.abs()) * 2.0 ** -22) * a.abs()
    if act == GELU:
        tol = tol + 2.0 ** -20 * a.abs()
    if residual is not None:
        tol = tol + 2.0 ** -23 * (a.abs() + residual.double().abs())
    tol = (tol + torch.finfo(out.dtype).eps / 2 * (want.abs() + tol)).clamp(min=2.0 ** -126)
    bad = ~((out.double() - want).abs() <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0].tolist()}, " \
                                f"worst {float(((out.double() - want).abs() / tol).max()):.3g} of the tolerance"


def one(M, N, K, dt=BF16, bias=True, act=SILU, residual=True, pad=0, opad=0, seed=1):
    g = _gen(seed)
    x, w = operand(M, K, g, 1.0, opad), operand(N, K, g, 1.5 / math.sqrt(K), opad)
    b = (0.3 * torch.randn(N, device="cuda", generator=g)).to(BF16) if bias else None
    out, res = like(M, N, dt, pad), None
    if residual:
        res = like(M, N, dt, pad)
        res.normal_(0.0, 2.0, generator=g)
    assert X.linear(x, w, out, bias=b, act=act, residual=res) == X.XPRESS_OK
    check(out, x, w, b, act, res)
    if pad and M > 1:                                         # what lies between the rows stays
        assert bool((out.as_strided((M - 1, pad), (out.stride(0), 1), N) == 7.0).all())
    return x, w, b, out, res


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 300, 513, 700])
@pytest.mark.parametrize("N, K", [(384, 512), (517, 328), (2083, 1000)])
def test_rows(M, N, K):
    one(M, N, K)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("K", [1, 7, 8, 63, 64, 65, 127, 128, 129, 192, 4096, 4104, 5000])
def test_depths(M, K):
    one(M, 200, K, dt=F32)


@pytest.mark.parametrize("M", [1, 20, 100, 260])
@pytest.mark.parametrize("N", [1, 2, 7, 127, 128, 129, 255, 256, 257, 4096])
def test_columns(M, N):
    one(M, N, 320)


@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("act", [NONE, SILU, GELU, RELU])
@pytest.mark.parametrize("bias, residual", [(False, False), (True, False), (False, True), (True, True)])
def test_epilogues(M, dt, act, bias, residual):
    one(M, 328, 256, dt, bias, act, residual)


@pytest.mark.parametrize("M", [3, 70, 200, 1100])
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad", [1, 3, 4, 8])
def test_padded_rows(M, dt, pad):
    one(M, 520, 200, dt, pad=pad, opad=24)


@pytest.mark.parametrize("M, N, K", [
    (1, 4096, 4096), (16, 1024, 16384), (8, 128, 65536), (30, 512, 8192), (60, 700, 8192), (128, 1000, 4096), (100, 300, 16384),  # few rows, K split
    (512, 4096, 16384), (256, 256, 16384), (300, 700, 8192), (1000, 1030, 4096),                                                   # pairs, K split
    (16, 38912, 512), (100, 38912, 256), (2048, 8192, 512), (3000, 5000, 256)])                                                    # many tiles
@pytest.mark.parametrize("dt", [BF16, F32])
def test_plans(M, N, K, dt):
    one(M, N, K, dt)


def test_a_bias_that_starts_anywhere():
    g = _gen(3)
    for M in (5, 300):
        x, w = operand(M, 256, g), operand(520, 256, g, 0.1)
        b = torch.randn(521, device="cuda", generator=g).to(BF16)[1:]
        out = like(M, 520, BF16)
        X.linear(x, w, out, bias=b, act=RELU)
        check(out, x, w, b, RELU)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("K", [512, 16384])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_in_place_on_the_residual(M, K, dt):
    g = _gen(4)
    x, w = operand(M, K, g), operand(600, K, g, 1.0 / math.sqrt(K))
    res = torch.randn((M, 600), device="cuda", generator=g).to(dt)
    out = res.clone()
    X.linear(x, w, out, act=SILU, residual=out)
    check(out, x, w, None, SILU, res)


def test_no_rows():
    w = operand(64, 64, _gen(5))
    out = like(0, 64, BF16)
    assert X.linear(w[:0], w, out) == X.XPRESS_OK


@pytest.mark.parametrize("M", [2, 300])
@pytest.mark.parametrize("act", [NONE, SILU, GELU, RELU])
def test_infinities_and_nans_stay_in_their_places(M, act):
    """A NaN or an infinity of x reaches its row, of w its column, of the residual its place."""
    g = _gen(6)
    x, w, res = operand(M, 128, g), operand(300, 128, g), like(M, 300, F32)
    res.normal_(0.0, 1.0, generator=g)
    x[0, 5] = float("nan")
    w[7, 100] = float("inf")
    res[1, 9] = float("-inf")
    out = like(M, 300, F32)
    X.linear(x, w, out, act=act, residual=res)
    assert bool(out[0].isnan().all()) and float(out[1, 9]) == float("-inf")
    t = activation(act, x.double() @ w.double().t()) + res.double()
    assert bool((out[1:, 7].isinf() | out[1:, 7].isnan() | (t[1:, 7] == out[1:, 7].double())).all())
    rest = torch.ones((M, 300), dtype=torch.bool, device="cuda")
    rest[0], rest[:, 7], rest[1, 9] = False, False, False
    assert bool(out[rest].isfinite().all())


@pytest.mark.parametrize("act", [SILU, GELU, RELU])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_activations_over_their_range(act, dt):
    """One product per output, so that the sum is exact: the activations from far negative to far positive."""
    t = torch.cat([torch.linspace(-100.0, 100.0, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3e38, -3e38])])
    w = torch.zeros((t.numel(), 8), dtype=BF16, device="cuda")
    w[:, 0] = t.to(BF16).cuda()
    x = torch.zeros((1, 8), dtype=BF16, device="cuda")
    x[0, 0] = 1.0
    out = like(1, t.numel(), dt)
    X.linear(x, w, out, act=act)
    check(out, x, w, None, act)


@pytest.mark.parametrize("M, N, K", [(1, 4096, 4096), (300, 700, 8192), (2000, 3000, 512)])
def test_calls_repeat_bit_for_bit(M, N, K):
    x, w, b, out, res = one(M, N, K, F32)
    for _ in range(5):
        again = torch.empty_like(out)
        X.linear(x, w, again, bias=b, act=SILU, residual=res)
        assert torch.equal(out, again)


def test_streams_and_graphs():
    g = _gen(8)
    cases = [(M, operand(M, 1024, g), operand(500, 1024, g, 0.03), like(M, 500, BF16)) for M in (1, 50, 400)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _, x, w, out in cases:
        X.linear(x, w, out, act=GELU, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for _, x, w, out in cases:
        check(out, x, w, None, GELU)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _, x, w, out in cases:
            X.linear(x, w, out, act=GELU)
    for _, x, w, out in cases:
        x.normal_(0.0, 1.0, generator=g)
        out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for _, x, w, out in cases:
        check(out, x, w, None, GELU)


def test_a_block_of_two_products():
    """x + W2 act(W1 x + b1) + b2, the second product reading what the first wrote."""
    g = _gen(9)
    for M in (1, 16, 700):
        x = operand(M, 512, g)
        w1, w2 = operand(2048, 512, g, 0.05), operand(512, 2048, g, 0.03)
        b1, b2 = (torch.randn(n, device="cuda", generator=g).to(BF16) for n in (2048, 512))
        mid, out = like(M, 2048, BF16), like(M, 512, BF16)
        X.linear(x, w1, mid, bias=b1, act=GELU)
        X.linear(mid, w2, out, bias=b2, residual=x)
        check(mid, x, w1, b1, GELU)
        check(out, mid, w2, b2, NONE, x)
