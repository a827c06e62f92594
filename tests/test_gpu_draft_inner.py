"""FeedForward with an inner width that is no multiple of 8, alone and in DraftHead: each
product against its definition in 64 bits."""
import pytest

import test_gpu_linear as LIN
from paper_2608_02438_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
b, B, H, V = 2, 4, 256, 1056


@pytest.fixture(scope="module")
def mods():
    from paper_2608_02438_gb300 import binding as X
    from paper_2608_02438_gb300 import build
    from paper_2608_02438_gb300 import draft_head as D
    build.build()
    return X, D


def _block(D, X, inner, g, offset=0):
    """Weights as a checkpoint has them: contiguous rows, from `offset` elements of their storage."""
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731

    def at(t):
        flat = torch.empty(t.numel() + offset, dtype=BF16, device="cuda")
        flat[offset:] = t.reshape(-1)
        return flat[offset:].view(t.shape)
    return D.FeedForward((1 + 0.1 * rnd(H)).to(BF16), at((0.06 * rnd(inner, H)).to(BF16)), at((0.05 * rnd(H, inner)).to(BF16)),
                         (0.2 * rnd(inner)).to(BF16), (0.2 * rnd(H)).to(BF16), X.XPRESS_ACT_SILU)


@pytest.mark.parametrize("inner", [1, 7, 250, 1001, 1004])
@pytest.mark.parametrize("rows", [1, 8])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("offset", [0, 3])
def test_any_inner_width(mods, inner, rows, residual, offset):
    X, D = mods
    g = torch.Generator(device="cuda").manual_seed(91)
    block = _block(D, X, inner, g, offset)
    W1, W2 = block.W1.clone(), block.W2.clone()
    x = torch.randn((rows, H), device="cuda", generator=g).to(BF16)
    r = torch.randn((rows, H), device="cuda", generator=g).to(BF16) if residual else None
    out = block(x, r, 1e-6)
    total = (x.float() + r.float()).to(BF16) if residual else x
    normed, mid = torch.empty_like(x), LIN.like(rows, inner, BF16, -inner % 8)
    X.rmsnorm(x, block.norm_weight, 1e-6, residual=r, y_out=normed)
    X.linear(normed, block.W1, mid, bias=block.b1, act=block.act)
    LIN.check(mid, normed, W1, block.b1, block.act)
    LIN.check(out, mid, W2, block.b2, X.XPRESS_ACT_NONE, total)


def test_in_a_head_on_the_refiners_stream(mods):
    X, D = mods
    g = torch.Generator(device="cuda").manual_seed(92)
    w = W.make_weights(H, V, 256, B, W.BF16, 93, "strong")
    side = torch.cuda.Stream()
    ref = X.Refiner({k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}, H, V, 256, B, X.XPRESS_BF16, stream=side)
    block = _block(D, X, 333, g)
    head = D.DraftHead(ref, torch.ones(H, dtype=BF16, device="cuda"), (0.1 * torch.randn((V, H), device="cuda", generator=g)).to(BF16),
                       block=block)
    x = torch.randn((b, B, H), device="cuda", generator=g).to(BF16)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        base = head.base_logits(x)
    side.synchronize()
    assert torch.equal(base["sum"].view(-1, H), block(x.view(-1, H), None, head.eps))
    assert X.matmul_fp8_status() == X.XPRESS_OK


def test_padded_rows_are_used_as_they_are(mods):
    X, D = mods
    padded = LIN.operand(H, 333, torch.Generator(device="cuda").manual_seed(94), 0.05)
    block = D.FeedForward(torch.ones(H, dtype=BF16, device="cuda"), torch.zeros((333, H), dtype=BF16, device="cuda"), padded)
    assert block.W2.data_ptr() == padded.data_ptr() and block.W2.stride() == padded.stride()
