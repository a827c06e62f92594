"""xpress_rmsnorm on rows whose squares leave fp32's range, against the formula in
64 bits.

Tolerances: those of the ordinary rows (32 u |y|, half an ulp of the storage type;
the rescaled sum of squares takes the same roundings, and its power of two none), and
for outputs that are subnormal 2^-147 absolute: three products, each rounded to a
multiple of 2^-149."""
import pytest

import test_gpu_head as G

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16, F32, U24 = torch.bfloat16, torch.float32, 2.0 ** -24
X = G.X                                          # the module's fixture

SCALES = [1e-45, 1e-42, 1e-38, 1e-30, 3e-20, 1e-18, 1e-3, 1.0, 1e15, 1e18, 3e19, 1e30, 5e37]
SUBNORMAL = 2.0 ** -147


def _rows(H, dtype, copies, g):
    """A row of every scale (twice with its largest value alone at that scale), as fp32 or
    bf16 holds it."""
    z = torch.randn((len(SCALES), H), device="cuda", generator=g, dtype=torch.float64).clamp_(-4, 4)
    x = z * torch.tensor(SCALES, dtype=torch.float64, device="cuda")[:, None]
    one = z * 1e-3
    one[:, H // 3] = torch.tensor(SCALES, dtype=torch.float64, device="cuda") * 4
    return torch.cat([x, one, torch.zeros((1, H), dtype=torch.float64, device="cuda")]).to(dtype).repeat(copies, 1)


def _check(y, s, q, x, w, eps, dtype):
    _, y64, s64, q64 = G._norm64(x, None, w, torch.tensor(eps, dtype=F32).item())    # the eps that the call gets
    ok = torch.isfinite(y64).all(dim=1)          # eps = 0 and a row of zeros: 0 / 0
    assert int((~ok).sum()) == (0 if eps else int((x == 0).all(dim=1).sum()))
    assert torch.isnan(y[~ok]).all()
    y, s, q, y64, s64, q64 = (v[ok] for v in (y, s, q, y64, s64, q64))
    tol = 32 * U24 * y64.abs() + SUBNORMAL
    assert ((y.double() - y64).abs() <= tol + G._half_ulp(y64.abs() + tol, dtype)).all()
    assert ((s.double() - s64).abs() <= 32 * U24 * s64).all()
    err = (q.double() - q64).abs()
    # (2^-20: the subnormal y's error over the smallest scale, 2^-126)
    assert (err <= G._half_ulp_e4m3(q64 * (1 + 2.0 ** -18)) + 2.0 ** -18 * q64.abs() + 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("eps", [1e-6, 0.0, 1e-30, 1e-40])
@pytest.mark.parametrize("H, copies, pad", [(8, 1, 0), (512, 1, 0), (515, 1, 0), (1000, 6, 1), (2048, 6, 0), (4096, 1, 0),
                                            (4096, 6, 0), (5202, 6, 0), (9000, 1, 0), (16384, 6, 0), (20000, 1, 0),
                                            (20001, 6, 2)])
def test_norm_outside_the_squares_range(X, H, copies, pad, eps, dtype):
    g = G._gen(H)
    v = _rows(H, dtype, copies, g)
    x = G._padded(*v.shape, dtype, pad)[1]
    x.copy_(v)
    w = (1 + 0.2 * torch.rand(H, device="cuda", generator=g)).to(dtype)
    t, y, q = torch.empty_like(v), torch.empty_like(v), X.alloc_e4m3(*v.shape)
    s = torch.empty((v.shape[0], -(-H // 128)), device="cuda")
    X.rmsnorm(x, w, eps, sum_out=t, y_out=y, q_out=q, scale_out=s)
    assert torch.equal(t, v)                     # the sum is not the scaled one
    _check(y, s, q.float(), x, w, eps, dtype)
    # in place, with a residual of zeros: the same (rows that are not padded may be
    # read in other pieces, and their squares added in another order)
    res, y2 = torch.zeros_like(v), x.clone()
    X.rmsnorm(y2, w, eps, residual=res, sum_out=res, y_out=y2, q_out=q, scale_out=s)
    assert torch.equal(res, v)
    _check(y2, s, q.float(), x, w, eps, dtype)
    assert pad or torch.equal(y2.nan_to_num(7.0), y.nan_to_num(7.0))


@pytest.mark.parametrize("H", [512, 4099, 20000])
def test_norm_of_huge_rows_with_an_infinity_or_a_nan(X, H):
    x = torch.full((3, H), 1e30, device="cuda")
    x[0, 5], x[1, 6], x[2, 7], x[2, 8] = float("inf"), float("nan"), float("inf"), float("nan")
    y = torch.empty_like(x)
    X.rmsnorm(x, torch.ones(H, device="cuda"), 1e-6, y_out=y)
    assert torch.isnan(y[0, 5]) and int((y[0] == 0).sum()) == H - 1
    assert torch.isnan(y[1:]).all()
