"""GPU tests of the 8-bit drafter head: xpress_rmsnorm, xpress_quantize_weight
and xpress_matmul_fp8 against their definitions in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, the unit roundoff of fp32):
  norm    t is one rounding; the sum of squares is a tree over at most 40
          roundings per path, halved by the root; root, quotient and the two
          products add 4: |y - y64| <= 32 u |y64|, plus half a bf16 ulp of the
          larger of the two (2^(floor(log2 |y|) - 8)) where stored in bf16.  The same 32 u for the scale.
  q       |q - y64 / scale64| <= half the e4m3 spacing there + 2^-18 relative
          (the errors of y and the scale)
  product products of two e4m3 values are exact in fp32; 128 sums per K block
          (taken as truncating, 2 u each), the scales' product, and one FMA per
          K block: |out - out64| <= (128 + KB + 2) 2 u sum |terms|, plus half an
          ulp of the output type.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02438_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _padded(rows, cols, dtype, pad, off=0):
    """[rows, cols] inside a wider, NaN-filled matrix, starting `off` elements into a row."""
    t = torch.full((rows, off + cols + pad), float("nan"), dtype=dtype, device="cuda")
    return t, t[:, off:off + cols]


def _half_ulp(v, dtype):
    """Half the spacing of the storage type at v (0 for fp32, whose rounding is counted in u)."""
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -126))) - 8) if dtype is BF16 else 0.0


def _half_ulp_e4m3(v):
    a = v.abs().clamp(min=2.0 ** -6)
    return torch.exp2(torch.floor(torch.log2(a)) - 4)


# -------------------------------------------------------------------- norm

def _norm64(x, res, w, eps):
    t = x.double() + (0 if res is None else res.double())
    y = t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + eps) * w.double()
    n, H = y.shape
    G = -(-H // 128)
    yg = torch.nn.functional.pad(y, (0, G * 128 - H)).view(n, G, 128)
    s = (yg.abs().amax(dim=2) / 448).clamp(min=2.0 ** -126)
    return t, y, s, (yg / s[:, :, None]).view(n, -1)[:, :H]


def _check_norm(t, y, s, q, ref, dtype):
    t64, y64, s64, q64 = ref
    if t is not None:
        tol = U24 * t64.abs()
        assert ((t.double() - t64).abs() <= tol + _half_ulp(t64.abs() + tol, dtype)).all()
    if y is not None:
        tol = 32 * U24 * y64.abs() + 1e-37
        assert ((y.double() - y64).abs() <= tol + _half_ulp(y64.abs() + tol, dtype)).all()
    if q is not None:
        assert ((s.double() - s64).abs() <= 32 * U24 * s64).all()
        err = (q.double() - q64).abs()
        assert (err <= _half_ulp_e4m3(q64 * (1 + 2.0 ** -18)) + 2.0 ** -18 * q64.abs()).all()


NORM_CASES = [  # rows, H, pad, offset of the first element
    (1, 1, 0, 0), (1, 8, 0, 0), (3, 127, 0, 0), (2, 128, 0, 0), (5, 129, 7, 0), (16, 256, 0, 0), (7, 1000, 8, 0),
    (4, 1023, 1, 0), (33, 2048, 0, 0), (9, 2056, 0, 8), (1, 4096, 0, 0), (19, 4096, 16, 0), (6, 4099, 5, 3),
    (3, 8192, 0, 0), (2, 8200, 0, 0), (2, 12000, 3, 1), (2, 16384, 0, 0), (3, 16392, 0, 0), (2, 40000, 0, 0),
    (2, 40001, 2, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows, H, pad, off", NORM_CASES)
def test_norm(X, rows, H, pad, off, dtype):
    g = _gen(rows * 100003 + H)
    mk = lambda scale: _padded(rows, H, dtype, pad, off)[1].normal_(0, scale, generator=g)  # noqa: E731
    x, res = mk(1.0), mk(3.0)
    x[:, ::37] *= 20
    x[-1] = 0                                    # a row whose sum is the residual alone
    w = (1 + 0.3 * torch.randn(H, device="cuda", generator=g)).to(dtype)
    (ts, t), (ys, y) = _padded(rows, H, dtype, pad, off), _padded(rows, H, dtype, pad, off)
    qb = torch.full((rows, off + H + pad), 0x5a, dtype=torch.uint8, device="cuda")
    q = qb.view(torch.float8_e4m3fn)[:, off:off + H]
    s = torch.full((rows, -(-H // 128)), -1.0, device="cuda")
    for r in (res, None):
        X.rmsnorm(x, w, 1e-5, residual=r, sum_out=t, y_out=y, q_out=q, scale_out=s)
        _check_norm(t, y, s, q.float(), _norm64(x, r, w, 1e-5), dtype)
    # nothing outside the rows is written
    assert torch.isnan(ts[:, :off]).all() and torch.isnan(ts[:, off + H:]).all()
    assert torch.isnan(ys[:, :off]).all() and torch.isnan(ys[:, off + H:]).all()
    assert (qb[:, :off] == 0x5a).all() and (qb[:, off + H:] == 0x5a).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows, H, pad, off", [
    (1, 2, 0, 0), (3, 126, 4, 2), (5, 129, 5, 2), (700, 130, 0, 0), (200, 1001, 1, 4), (300, 2301, 3, 0), (400, 2302, 0, 0),
    (160, 3527, 0, 0), (161, 5202, 8, 2), (170, 4354, 0, 2), (2, 8190, 4, 2), (3, 12003, 3, 6), (3, 16386, 0, 0),
    (2, 40002, 0, 0), (155, 8193, 7, 0)])
def test_norm_odd_rows(X, rows, H, pad, off, dtype):
    """Rows that start on a pair but not on 16 bytes, numbers of segments that fill no block."""
    test_norm(X, rows, H, pad, off, dtype)


@pytest.mark.parametrize("H", [256, 1027, 33000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_single_outputs_and_in_place(X, H, dtype):
    g = _gen(H)
    x = torch.empty((5, H), dtype=dtype, device="cuda").normal_(generator=g)
    res = torch.empty_like(x).normal_(generator=g)
    w = torch.rand(H, device="cuda", generator=g).to(dtype)
    t, y, q, s = torch.empty_like(x), torch.empty_like(x), X.alloc_e4m3(5, H), torch.empty((5, -(-H // 128)), device="cuda")
    X.rmsnorm(x, w, 1e-6, residual=res, sum_out=t, y_out=y, q_out=q, scale_out=s)
    for kw in (dict(sum_out=torch.empty_like(x)), dict(y_out=torch.empty_like(x)),
               dict(q_out=X.alloc_e4m3(5, H), scale_out=torch.empty_like(s))):
        X.rmsnorm(x, w, 1e-6, residual=res, **kw)
        for k, v in kw.items():
            ref = dict(sum_out=t, y_out=y, q_out=q, scale_out=s)[k]
            assert torch.equal(v.float(), ref.float()), k
    # the sum over the residual, the norm over x: the usual in-place step
    x2, r2 = x.clone(), res.clone()
    X.rmsnorm(x2, w, 1e-6, residual=r2, sum_out=r2, y_out=x2, q_out=(q2 := X.alloc_e4m3(5, H)), scale_out=(s2 := torch.empty_like(s)))
    assert torch.equal(r2, t) and torch.equal(x2, y) and torch.equal(q2.float(), q.float()) and torch.equal(s2, s)


@pytest.mark.parametrize("H", [512, 515])
def test_norm_special_values(X, H):
    """Rows of zeros, tiny and huge values, NaN and infinity follow the formula."""
    x = torch.randn((7, H), device="cuda", generator=_gen(3))
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e15
    x[3, 5] = float("nan")
    x[4, 200] = float("inf")
    x[5, 128:256] = 0                            # a group of zeros in an ordinary row
    x[6] *= 1e-42                                # subnormal inputs
    w = torch.ones(H, device="cuda")
    for eps in (1e-6, 0.0):
        y, q, s = torch.empty_like(x), X.alloc_e4m3(7, H), torch.empty((7, -(-H // 128)), device="cuda")
        X.rmsnorm(x, w, eps, y_out=y, q_out=q, scale_out=s)
        qf = q.float()
        if eps:
            assert (y[0] == 0).all() and (qf[0] == 0).all() and (s[0] == 2.0 ** -126).all()
            _check_norm(None, y[1:3], s[1:3], qf[1:3], _norm64(x[1:3], None, w, eps), F32)
        assert torch.isnan(y[3]).all() and torch.isnan(qf[3]).all() and torch.isnan(s[3]).all()
        assert torch.isnan(y[4, 200]) and torch.isnan(qf[4, 200]) and torch.isnan(s[4, 1])
        others = [i for i in range(H) if i // 128 != 1]
        assert (y[4, others] == 0).all() and (qf[4, others] == 0).all()
        assert (qf[5, 128:256] == 0).all() and s[5, 1] == 2.0 ** -126
        _check_norm(None, y[5:6], s[5:6], qf[5:6], _norm64(x[5:6], None, w, eps), F32)


def test_norm_empty_batch_and_many_rows(X):
    w = torch.ones(64, dtype=BF16, device="cuda")
    assert X.rmsnorm(torch.empty((0, 64), dtype=BF16, device="cuda"), w, y_out=torch.empty((0, 64), dtype=BF16, device="cuda")) == 0
    rows = (1 << 25) + 77                        # rows * H past 2^31
    x = torch.empty((rows, 64), dtype=BF16, device="cuda").fill_(1.0)
    x[-1] = torch.arange(64, device="cuda").to(BF16)
    y, q, s = torch.empty_like(x), X.alloc_e4m3(rows, 64), torch.empty((rows, 1), device="cuda")
    X.rmsnorm(x, w, 1e-6, y_out=y, q_out=q, scale_out=s)
    _check_norm(None, y[-3:], s[-3:], q[-3:].float(), _norm64(x[-3:], None, w, 1e-6), BF16)
    assert bool((y[:-1] == 1).all())


# ----------------------------------------------------------------- weights

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows, cols, pad, off", [(1, 1, 0, 0), (128, 128, 0, 0), (127, 129, 0, 0), (300, 257, 3, 1),
                                                  (512, 256, 0, 0), (517, 280, 8, 0), (40, 1000, 0, 8), (2080, 96, 0, 0)])
def test_quantize_weight(X, rows, cols, pad, off, dtype):
    _, W = _padded(rows, cols, dtype, pad, off)
    W.normal_(0, 0.02, generator=_gen(rows + cols))
    W[rows // 2:, cols // 2:] *= 50
    if rows > 256:
        W[128:256] = 0                           # blocks of zeros
    qb = torch.full((rows, off + cols + pad), 0x5a, dtype=torch.uint8, device="cuda")
    q = qb.view(torch.float8_e4m3fn)[:, off:off + cols]
    _, s = X.quantize_weight(W, q)
    nr, nc = -(-rows // 128), -(-cols // 128)
    Wb = torch.nn.functional.pad(W.double(), (0, nc * 128 - cols, 0, nr * 128 - rows)).view(nr, 128, nc, 128)
    s64 = (Wb.abs().amax(dim=(1, 3)) / 448).clamp(min=2.0 ** -126)
    assert torch.equal(s, s64.float())           # the largest magnitude is exact, the quotient rounded once
    # by the stored scale: the quotient rounded to e4m3 (through fp32: 2^-24 beside its half spacing)
    t = (Wb / s.double()[:, None, :, None]).view(nr * 128, nc * 128)[:rows, :cols]
    err = (q.float().double() - t).abs()
    assert (err <= _half_ulp_e4m3(t) + 2.0 ** -23 * t.abs()).all()
    assert (qb[:, :off] == 0x5a).all() and (qb[:, off + cols:] == 0x5a).all()


def test_quantize_special_values(X):
    W = torch.randn((256, 256), device="cuda", generator=_gen(4))
    W[3, 4] = float("nan")
    W[200, 7] = float("inf")
    W[:128, 128:] = 1e-40
    q, s = X.quantize_weight(W)
    qf = q.float()
    assert torch.isnan(s[0, 0]) and torch.isnan(qf[:128, :128]).all()
    assert torch.isinf(s[1, 0]) and torch.isnan(qf[200, 7])
    rest = qf[128:, :128].clone()
    rest[200 - 128, 7] = 0
    assert (rest == 0).all()
    assert s[0, 1] == 2.0 ** -126 and torch.isfinite(qf[:128, 128:]).all() and torch.isfinite(qf[128:, 128:]).all()


# ----------------------------------------------------------------- product

def _operand(rows, K, seed, pad=0, off=0):
    """e4m3 [rows, K] (pitch a multiple of 16) in memory whose every other byte is NaN."""
    pitch = off + -(-(K + pad) // 16) * 16
    buf = torch.full((rows, pitch), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    t = buf[:, off:off + K]
    t.copy_((torch.randn((rows, K), device="cuda", generator=_gen(seed)) * 100).clamp(-448, 448).to(torch.float8_e4m3fn))
    return t


def _ref_mm(a, sa, w, sw):
    """The product and the sum of its terms' magnitudes, in 64 bits."""
    N, K = w.shape
    out = torch.zeros((a.shape[0], N), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(out)
    for j in range(0, K, 128):
        f = sa[:, j // 128, None].double() * sw[:, j // 128].double().repeat_interleave(128)[:N]
        A, B = a[:, j:j + 128].float().double(), w[:, j:j + 128].float().double()
        out += (A @ B.t()) * f
        mag += (A.abs() @ B.abs().t()) * f.abs()
    return out, mag


def _mm(X, M, N, K, dtype, pad=0, off=0, out_pad=0):
    a, w = _operand(M, K, 7 * M + K, pad, off), _operand(N, K, 11 * N + K, pad, off)
    kb = -(-K // 128)
    sa = torch.rand((M, kb + 1), device="cuda", generator=_gen(M))[:, :kb] * 0.02
    sw = torch.rand((-(-N // 128), kb + 3), device="cuda", generator=_gen(N))[:, :kb] * 1e-3
    buf = torch.full((M, N + out_pad), -7.0, dtype=dtype, device="cuda")
    out = buf[:, :N]
    assert X.matmul_fp8(a, sa, w, sw, out) == X.XPRESS_OK
    ref, mag = _ref_mm(a, sa, w, sw)
    err = (out.double() - ref).abs()
    gamma = (128 + kb + 2) * 2 * U24 * mag
    store = _half_ulp(ref.abs() + gamma, dtype) if dtype is BF16 else U24 * (ref.abs() + gamma)
    assert (err <= gamma + store).all(), float((err / (gamma + store)).max())
    assert (buf[:, N:] == -7.0).all()
    assert X.matmul_fp8_status() == X.XPRESS_OK
    return out


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300, 513])
def test_matmul_row_counts(X, M):
    _mm(X, M, 2088, 512, BF16)
    _mm(X, M, 200, 1000, F32, out_pad=3)


@pytest.mark.parametrize("N", [1, 2, 7, 8, 31, 127, 128, 129, 255, 256, 257, 385, 1000, 2080, 4097])
@pytest.mark.parametrize("M", [1, 24, 150, 300])
def test_matmul_column_counts(X, M, N):
    _mm(X, M, N, 384, BF16, out_pad=1)


@pytest.mark.parametrize("K", [1, 15, 16, 31, 32, 33, 127, 128, 129, 255, 257, 640, 1000, 1024, 2176, 4096, 8200])
@pytest.mark.parametrize("M", [1, 16, 40, 130, 260])
def test_matmul_inner_sizes(X, M, K):
    _mm(X, M, 300, K, F32, pad=16, off=16)


@pytest.mark.parametrize("M, N, K", [(1, 128, 65536), (33, 130, 65536), (140, 384, 30000), (1, 40000, 128),
                                     (70, 20000, 256), (1024, 1024, 256), (16, 19456, 512), (270, 5000, 4096)])
def test_matmul_shapes(X, M, N, K):
    _mm(X, M, N, K, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M, N, K", [(600, 3330, 1000), (1025, 3001, 1544), (640, 4096, 2048), (1000, 12001, 100),
                                     (130, 60000, 648), (4097, 4100, 16)])
def test_matmul_many_rows_ragged(X, M, N, K, dtype):
    """Shapes that the kernel for many rows takes, none a multiple of its tile."""
    _mm(X, M, N, K, dtype, pad=8, off=16, out_pad=5)
    _mm(X, M, N, K, dtype)


@pytest.mark.parametrize("M, N, K", [(1, 100, 8192), (9, 1000, 8192), (16, 130, 16384), (30, 260, 8192), (32, 100, 4096),
                                     (5, 4096, 1024), (17, 4100, 4104), (24, 4096, 4096)])
def test_matmul_split_k(X, M, N, K):
    """K split over clusters of 2, 4 and 8, rows of a that fill no share."""
    _mm(X, M, N, K, F32, out_pad=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_matmul_many_rows_by_16_bytes(X, dtype):
    """Rows of out on 16 bytes, but not on 32, in more tiles than SMs."""
    _mm(X, 2049, 4104 if dtype is BF16 else 4100, 200, dtype)
    _mm(X, 2049, 4096, 200, dtype, out_pad=8 if dtype is BF16 else 4)


@pytest.mark.parametrize("M, N, K", [(512, 4096, 4096), (300, 600, 8192), (566, 1550, 2048), (200, 4096, 4096),
                                     (129, 257, 16384), (1000, 2000, 8192), (640, 3001, 1544), (513, 100, 8200),
                                     (400, 5000, 3000)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_matmul_many_rows_split_k(X, M, N, K, dtype):
    """K split over clusters of the kernel for many rows, whole and partial tiles."""
    _mm(X, M, N, K, dtype, pad=8, off=16, out_pad=5)
    out = _mm(X, M, N, K, dtype)
    assert torch.equal(out, _mm(X, M, N, K, dtype))


def test_matmul_reproducible(X):
    for M, N, K in ((5, 512, 4096), (64, 4096, 2048), (300, 1000, 1000)):
        assert torch.equal(_mm(X, M, N, K, F32), _mm(X, M, N, K, F32))


def test_matmul_empty_and_nan_rows(X):
    q = lambda r, k: X.alloc_e4m3(r, k)  # noqa: E731
    assert X.matmul_fp8(q(0, 64), torch.empty((0, 1), device="cuda"), q(5, 64), torch.empty((1, 1), device="cuda"),
                        torch.empty((0, 5), device="cuda")) == X.XPRESS_OK
    for M, N in ((3, 260), (200, 260), (300, 260), (700, 5000)):
        a, w = _operand(M, 256, 1), _operand(N, 256, 2)
        a[1, 130] = float("nan")
        w[258, 3] = float("nan")
        out = torch.empty((M, N), device="cuda")
        X.matmul_fp8(a, torch.ones((M, 2), device="cuda"), w, torch.ones((-(-N // 128), 2), device="cuda"), out)
        nan = torch.isnan(out)
        assert nan[1].all() and nan[:, 258].all()
        nan[1] = False
        nan[:, 258] = False
        assert not nan.any()


def test_matmul_infinite_scale(X):
    for M, N in ((2, 130), (150, 130), (700, 5000)):
        a, w = _operand(M, 256, 1), _operand(N, 256, 2)
        sa, sw = torch.ones((M, 2), device="cuda"), torch.ones((-(-N // 128), 2), device="cuda")
        sa[0, 1] = float("inf")
        sw[1:, 0] = float("nan")
        out = torch.empty((M, N), device="cuda")
        X.matmul_fp8(a, sa, w, sw, out)
        assert not torch.isfinite(out[0]).any() and torch.isnan(out[:, 128:]).all() and torch.isfinite(out[1:, :128]).all()


def test_matmul_output_past_32_bits(X):
    M, N, K = 20000, 151936, 32                  # M * N = 3.04e9
    a, w = _operand(M, K, 5), _operand(N, K, 6)
    sa, sw = torch.rand((M, 1), device="cuda"), torch.rand((N // 128, 1), device="cuda")
    out = torch.zeros((M, N), dtype=BF16, device="cuda")
    X.matmul_fp8(a, sa, w, sw, out)
    at = torch.tensor([0, 1, 14133, 14134, 14135, 16383, M - 1], device="cuda")
    ref, mag = _ref_mm(a[at], sa[at], w, sw)
    gamma = 131 * 2 * U24 * mag
    assert ((out[at].double() - ref).abs() <= gamma + _half_ulp(ref.abs() + gamma, BF16)).all()


def test_norm_then_product_is_the_heads_error(X):
    """The 8-bit head against the 64-bit product of the unquantised operands:
    per element, e4m3 keeps 2^-4 relative or 2^-10 of a group's largest
    magnitude, for both operands."""
    rows, H, V = 16, 512, 2080
    g = _gen(12)
    x = torch.empty((rows, H), dtype=BF16, device="cuda").normal_(generator=g)
    w = torch.ones(H, dtype=BF16, device="cuda")
    W = torch.empty((V, H), dtype=BF16, device="cuda").normal_(0, 0.02, generator=g)
    q, s = X.alloc_e4m3(rows, H), torch.empty((rows, H // 128), device="cuda")
    X.rmsnorm(x, w, 1e-6, q_out=q, scale_out=s)
    wq, ws = X.quantize_weight(W)
    out = torch.empty((rows, V), dtype=F32, device="cuda")
    X.matmul_fp8(q, s, wq, ws, out)
    y = _norm64(x, None, w, 1e-6)[1]
    ea = torch.maximum(2.0 ** -4 * y.abs(), s.double().repeat_interleave(128, 1) * 2.0 ** -10)
    ew = torch.maximum(2.0 ** -4 * W.double().abs(), ws.double().repeat_interleave(128, 0)[:V].repeat_interleave(128, 1) * 2.0 ** -10)
    bound = ea @ W.double().abs().t() + y.abs() @ ew.t() + ea @ ew.t()
    assert ((out.double() - y @ W.double().t()).abs() <= bound * 1.001).all()
    # and far less than the bound on the whole: errors of both signs
    rel = (out.double() - y @ W.double().t()).norm() / (y @ W.double().t()).norm()
    assert rel < 2.0 ** -4


# ------------------------------------------------------- streams and graphs

def test_other_streams(X):
    """Operands made on one stream, the call on another that waits for it."""
    side = torch.cuda.Stream()
    M, N, K = 16, 4096, 2048
    a, w = _operand(M, K, 1), _operand(N, K, 2)
    sa, sw = torch.ones((M, K // 128), device="cuda"), torch.ones((N // 128, K // 128), device="cuda")
    want, out = torch.empty((M, N), device="cuda"), torch.empty((M, N), device="cuda")
    X.matmul_fp8(a, sa, w, sw, want)
    side.wait_stream(torch.cuda.current_stream())
    X.matmul_fp8(a, sa, w, sw, out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    with torch.cuda.stream(side):
        out2 = torch.empty_like(want)
        X.matmul_fp8(a, sa, w, sw, out2)
    side.synchronize()
    assert torch.equal(out2, want)


def test_graph_capture(X):
    """The head captured once and replayed on new inputs in the same memory."""
    rows, H, V = 16, 1024, 3000
    x = torch.randn((rows, H), device="cuda").to(BF16)
    w = torch.ones(H, dtype=BF16, device="cuda")
    W = (torch.randn((V, H), device="cuda") * 0.02).to(BF16)
    wq, ws = X.quantize_weight(W)
    q, s, out = X.alloc_e4m3(rows, H), torch.empty((rows, H // 128), device="cuda"), torch.empty((rows, V), device="cuda")

    def step():
        X.rmsnorm(x, w, 1e-6, q_out=q, scale_out=s)
        X.matmul_fp8(q, s, wq, ws, out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(torch.randn((rows, H), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    step()
    assert torch.equal(got, out)
