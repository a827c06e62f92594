"""DraftHead.next_tokens under a grammar: a state that allows nothing, and temperatures at
which a forbidden token must not come out either."""
import pytest

from paper_2608_02438_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
b, B, H, V = 4, 8, 512, 2080


@pytest.fixture(scope="module")
def setup():
    from paper_2608_02438_gb300 import binding as X
    from paper_2608_02438_gb300 import build
    from paper_2608_02438_gb300 import draft_head as D
    build.build()
    w = W.make_weights(H, V, 256, B, W.BF16, 81, "strong")
    ref = X.Refiner({k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}, H, V, 256, B, X.XPRESS_BF16)
    g = torch.Generator(device="cuda").manual_seed(82)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    head = D.DraftHead(ref, torch.ones(H, dtype=BF16, device="cuda"), (0.1 * rnd(V, H)).to(BF16))
    mask = torch.zeros((3, V // 32), dtype=torch.int32, device="cuda")
    mask[1, 2] = 0x38                                              # ids 67, 68, 69
    mask[2, :] = -1
    return D, head, mask, (3 * rnd(b, V)).to(BF16)


@pytest.mark.parametrize("T", [0.0, 0.7, 1000.0, float("inf")])
@pytest.mark.parametrize("filters", [{}, dict(top_k=50, top_p=0.9), dict(min_p=0.05)])
def test_a_state_that_allows_nothing(setup, T, filters):
    D, head, mask, logits = setup
    col = lambda v: torch.full((b,), v, device="cuda", dtype=torch.int32 if isinstance(v, int) else torch.float32)  # noqa: E731
    f = D.Filters(**{k: col(v) for k, v in filters.items()})
    states = torch.tensor([0, 1, 2, -1], dtype=torch.int32, device="cuda")
    got = head.next_tokens(logits, col(T), col(0.6), D.Rules(mask=mask), f, states).tolist()
    assert got[0] == -1
    assert got[1] in (67, 68, 69)
    plain = head.next_tokens(logits, col(T), col(0.6), None, f).tolist()
    assert got[2:] == plain[2:]


@pytest.mark.parametrize("T", [100.0, 300.0, 1e4, 1e30, float("inf")])
def test_forbidden_tokens_are_not_drawn_at_high_temperatures(setup, T):
    D, head, mask, logits = setup
    states = torch.ones(b, dtype=torch.int32, device="cuda")
    for u in (0.0, 0.2, 0.5, 0.8, 0.9999):
        got = head.next_tokens(logits, torch.full((b,), T, device="cuda"), torch.full((b,), u, device="cuda"), D.Rules(mask=mask), None,
                               states).tolist()
        assert all(t in (67, 68, 69) for t in got), got
