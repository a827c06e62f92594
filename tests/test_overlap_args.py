"""Outputs of linear and sample in memory that the call also reads: refused where a written
place could be read afterwards, accepted where rows only lie between one another (without a
GPU: the tensors' places are looked at before their device)."""
import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _built():
    BLD.build()


def _buf(n, dt=torch.bfloat16):
    return torch.zeros(n, dtype=dt)


def _rows(buf, at, n, cols, pitch):
    return buf.as_strided((n, cols), (pitch, 1), at)


def _refused(call):
    with pytest.raises(ValueError, match="overlaps"):
        call()


def _passes(call):
    # the next check is the one of the device
    with pytest.raises(ValueError, match="CUDA device"):
        call()


@pytest.mark.parametrize("at", [-15, -1, 1, 8, 16, 17, 40])
def test_linear_out_over_its_residual(at):
    buf, x, w = _buf(400), _buf(6 * 8).view(6, 8), _buf(16 * 8).view(16, 8)
    _refused(lambda: X.linear(x, w, _rows(buf, 100 + at, 6, 16, 16), residual=_rows(buf, 100, 6, 16, 16)))
    same = _rows(buf, 100, 6, 16, 16)
    _passes(lambda: X.linear(x, w, same, residual=same))
    _passes(lambda: X.linear(x, w, _rows(buf, 100, 6, 16, 16), residual=same))


def test_linear_rows_between_rows():
    """Column ranges of one buffer, and what comes after the last row."""
    buf, x, w = _buf(400), _buf(6 * 8).view(6, 8), _buf(16 * 8).view(16, 8)
    wide = _rows(buf, 0, 6, 40, 40)
    _passes(lambda: X.linear(x, w, wide[:, 16:32], residual=wide[:, :16]))
    _passes(lambda: X.linear(x, w, wide[:, :16], residual=wide[:, 24:]))
    _refused(lambda: X.linear(x, w, wide[:, 15:31], residual=wide[:, :16]))
    _refused(lambda: X.linear(x, w, wide[:, :16], residual=wide[:, 15:31]))
    _passes(lambda: X.linear(x, w, _rows(buf, 96, 6, 16, 16), residual=_rows(buf, 0, 6, 16, 16)))
    # two pitches: rows of 16 at 20 and at 40 elements
    _passes(lambda: X.linear(x[:2], w, _rows(buf, 20, 2, 16, 80), residual=_rows(buf, 0, 2, 16, 40)))
    _refused(lambda: X.linear(x, w, _rows(buf, 16, 6, 16, 20), residual=_rows(buf, 0, 6, 16, 40)))


def test_linear_out_over_its_operands():
    buf = _buf(600)
    x, w, bias = _rows(buf, 0, 6, 16, 16), _rows(buf, 96, 16, 16, 16), buf[352:368]
    out = _rows(_buf(96), 0, 6, 16, 16)
    _passes(lambda: X.linear(x, w, out, bias=bias))
    for at in (0, 1, 40, 95, 96, 200, 340, 352, 367):
        _refused(lambda: X.linear(x, w, _rows(buf, at, 6, 16, 16), bias=bias))
    _passes(lambda: X.linear(x, w, _rows(buf, 368, 6, 16, 16), bias=bias))
    f = torch.zeros(500, dtype=torch.float32)
    xb = f.view(torch.bfloat16).as_strided((6, 16), (48, 1), 0)               # 32 bytes of every 96
    _passes(lambda: X.linear(xb, w, f.as_strided((6, 16), (24, 1), 8)))
    _refused(lambda: X.linear(xb, w, f.as_strided((6, 16), (24, 1), 7)))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_sample_out_over_its_logits(dt):
    buf, T = _buf(400, dt), torch.ones(4)
    logits = _rows(buf, 50, 4, 30, 32)
    _passes(lambda: X.sample(logits, T, out=logits))
    for at in (-29, -2, -1, 1, 2, 29, 32, 64, 125):
        _refused(lambda: X.sample(logits, T, out=_rows(buf, 50 + at, 4, 30, 32)))
    _passes(lambda: X.sample(logits, T, out=_rows(buf, 50 + 3 * 32 + 30, 4, 30, 32)))
    wide = _rows(buf, 0, 4, 90, 90)
    _passes(lambda: X.sample(wide[:, :30], T, out=wide[:, 30:60]))
    _refused(lambda: X.sample(wide[:, :30], T, out=wide[:, 29:59]))


def test_sample_outputs_over_the_parameters():
    f = torch.zeros(200)
    i = f.view(torch.int32)
    logits, T, u = torch.zeros((6, 8)), f[0:3], f[10:16]
    k, p, m = i[20:23], f[30:33], f[40:43]
    kw = dict(u=u, rows=2, top_k=k, top_p=p, min_p=m)
    _passes(lambda: X.sample(logits, T, tokens_out=i[50:56], out=f[60:108].view(6, 8), **kw))
    for at in (0, 2, 9, 11, 15, 18, 22, 27, 32, 38, 42):
        _refused(lambda: X.sample(logits, T, tokens_out=i[at:at + 6], **kw))
    for at in (0, 1, 8, 40):
        _refused(lambda: X.sample(logits, T, out=f[at:at + 48].view(6, 8), **kw))
    _refused(lambda: X.sample(logits, T, tokens_out=i[50:56], out=f[52:100].view(6, 8), **kw))
    _refused(lambda: X.sample(f[50:98].view(6, 8), T, tokens_out=i[60:66], **kw))
    # a row's own number, and with one row each its sequence's parameters, are read before its token is written
    _passes(lambda: X.sample(logits, T, tokens_out=i[10:16], **kw))
    _passes(lambda: X.sample(logits[:3], T, u=u[:3], tokens_out=k, top_k=k))
    _refused(lambda: X.sample(logits, f[100:106], u=u, tokens_out=i[101:107]))


def test_rows_longer_than_their_pitch():
    """Expanded rows go on to the entry point, which refuses them."""
    row = _buf(64).view(1, 64)
    T = torch.ones(5)
    _passes(lambda: X.sample(row.expand(5, 64), T, out=_buf(320).view(5, 64)))
    _passes(lambda: X.sample(_buf(320).view(5, 64), T, out=row.expand(5, 64)))
    _passes(lambda: X.sample(row[:, 1:].expand(5, 63), T, out=row[:, :63].expand(5, 63)))
    _passes(lambda: X.linear(row.expand(5, 64), row.expand(6, 64), row[:, :6].expand(5, 6)))
    _passes(lambda: X.linear(row.expand(5, 64), _buf(384).view(6, 64), _rows(_buf(100), 0, 5, 6, 3)))


def test_against_every_place():
    """Small placements of rows, counted out byte by byte."""
    import itertools
    buf, T = _buf(120), torch.ones(3)
    for at, n, cols, pitch in itertools.product((30, 31, 34, 39, 47), (1, 2, 3), (1, 3, 5), (5, 7, 14)):
        for n2, at2, pitch2 in itertools.product((n,), range(20, 64), (5, 6, 7, 14)):
            a, b = _rows(buf, at, n, cols, pitch), _rows(buf, at2, n2, cols, pitch2)
            places = [{t.storage_offset() + i * t.stride(0) + j for i in range(n) for j in range(cols)} for t in (a, b)]
            call = lambda: X.sample(a, T[:n], out=b)  # noqa: E731, B023
            if at != at2 and places[0] & places[1]:
                _refused(call)
            else:
                _passes(call)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [700, 40000, 1000003])
def test_tokens_over_what_their_row_has_read(V):
    """tokens_out in the numbers' memory, or with one row each in a sequence's parameters."""
    g = torch.Generator(device="cuda").manual_seed(7)
    logits = torch.randn((5, V), device="cuda", generator=g)
    T, u = torch.full((5,), 0.9, device="cuda"), torch.rand(5, device="cuda", generator=g)
    kw = dict(top_k=torch.full((5,), 40, dtype=torch.int32, device="cuda"), top_p=torch.full((5,), 0.9, device="cuda"),
              min_p=torch.full((5,), 1e-3, device="cuda"))
    want = torch.empty(5, dtype=torch.int32, device="cuda")
    X.sample(logits, T, u=u, tokens_out=want, **kw)
    for name in ("u", "T", "top_k", "top_p", "min_p"):
        args = dict(T=T.clone(), u=u.clone(), **{k: v.clone() for k, v in kw.items()})
        tokens = args[name].view(torch.int32)
        X.sample(logits, args.pop("T"), tokens_out=tokens, **args)
        assert torch.equal(tokens, want), name
