"""A round with a feed-forward block in front of the head and with the requests' filters,
all together: the block against its definition in 64 bits, the truncated target rows
against the filters' definition, the refinement and the acceptance against the oracle
from the rows as stored; and the next token of a request."""
import numpy as np
import pytest

import oracle as O
import test_gpu_linear as LIN
import test_gpu_sample as SMP
from paper_2608_02438_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
b, B, H, V, I = 4, 8, 512, 2080, 1000


@pytest.fixture(scope="module")
def setup():
    from paper_2608_02438_gb300 import binding as X
    from paper_2608_02438_gb300 import build
    from paper_2608_02438_gb300 import draft_head as D
    build.build()
    w = W.make_weights(H, V, 256, B, W.BF16, 61, "strong")
    ref = X.Refiner({k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}, H, V, 256, B, X.XPRESS_BF16)
    g = torch.Generator(device="cuda").manual_seed(62)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    block = D.FeedForward((1 + 0.1 * rnd(H)).to(BF16), LIN.operand(I, H, g, 0.06), LIN.operand(H, I, g, 0.05), (0.2 * rnd(I)).to(BF16),
                          (0.2 * rnd(H)).to(BF16), X.XPRESS_ACT_GELU)
    d = dict(x=rnd(b, B, H).to(BF16), residual=(2 * rnd(b, B, H)).to(BF16), target=(3 * rnd(b, B + 1, V)).to(BF16),
             anchor=torch.randint(0, V, (b,), device="cuda", generator=g, dtype=torch.int32),
             temperature=torch.tensor([0.0, 1.0, 0.7, 1.3], device="cuda"), seed=torch.arange(b, device="cuda", dtype=torch.int64) + 7)
    head = D.DraftHead(ref, (1 + 0.1 * rnd(H)).to(BF16), (0.1 * rnd(V, H)).to(BF16), block=block)
    filters = D.Filters(top_k=torch.tensor([0, 20, 0, 5], dtype=torch.int32, device="cuda"),
                        top_p=torch.tensor([0.9, 1.0, 0.8, 0.95], device="cuda"), min_p=torch.tensor([0.0, 0.1, 0.0, 0.0], device="cuda"))
    return X, D, w, ref, block, d, head, filters


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("residual", [False, True])
def test_block(setup, residual):
    X, D, w, ref, block, d, head, filters = setup
    x, r = d["x"].reshape(-1, H), d["residual"].reshape(-1, H) if residual else None
    out = block(x, r, 1e-6)
    total = (x.float() + r.float()).to(BF16) if residual else x
    normed, inner = torch.empty_like(x), LIN.like(b * B, I, BF16, 8)
    X.rmsnorm(x, block.norm_weight, 1e-6, residual=r, y_out=normed)
    X.linear(normed, block.W1, inner, bias=block.b1, act=block.act)
    LIN.check(inner, normed, block.W1, block.b1, block.act)
    LIN.check(out, inner, block.W2, block.b2, X.XPRESS_ACT_NONE, total)


@pytest.mark.parametrize("with_rules", [False, True])
def test_round(setup, with_rules):
    X, D, w, ref, block, d, head, filters = setup
    rules = D.Rules(repetition=torch.full((b,), 1.2, device="cuda"), history=torch.arange(400, device="cuda", dtype=torch.int32),
                    history_offsets=torch.arange(b + 1, device="cuda", dtype=torch.int64) * 100) if with_rules else None
    out = head.round(d["x"], d["residual"], d["target"], d["anchor"], d["temperature"], d["seed"], 5, B, rules, filters)
    torch.cuda.synchronize()
    assert ref.device_status("refine", b) == X.XPRESS_OK and X.matmul_fp8_status() == X.XPRESS_OK
    assert torch.equal(out["sum"].reshape(-1, H), block(d["x"].reshape(-1, H), d["residual"].reshape(-1, H), head.eps))
    ruled = head.target_logits(d["target"], out["tokens"], rules)
    rows = out["target"].view(-1, V)
    SMP.check(ruled.view(-1, V), d["temperature"], None, None, rows, B + 1, filters.top_k, filters.top_p, filters.min_p, D.MASKED)
    m = O.Model(w, H, V, 256, B, O.BF16)
    h, s, tgt = _bits(out["h"]), _bits(out["s"]), _bits(out["target"])
    for i in range(b):
        T = float(d["temperature"][i])
        o = O.jacobi(m, h[i], s[i], int(d["anchor"][i]), out["draft"][i].cpu().numpy(), T, int(d["seed"][i]), 5, B)
        assert out["tokens"][i].tolist() == o["tokens"].tolist(), f"tokens of block {i}"
        n, ot, _ = O.accept(m, tgt[i], s[i], o["tokens"], o["lse"], o["sel"], o["z_final"], T, int(d["seed"][i]), 5)
        assert int(out["accept_len"][i]) == n and out["out_tokens"][i].tolist() == ot.tolist(), f"acceptance of block {i}"
        for j, t in enumerate(out["out_tokens"][i].tolist()):
            assert t < 0 or float(out["target"][i, j, t]) > D.MASKED      # what is emitted was kept


def test_next_tokens(setup):
    X, D, w, ref, block, d, head, filters = setup
    logits, u = d["target"][:, 0].contiguous(), torch.tensor([0.3, 0.999, 0.0, 0.61], device="cuda")
    tokens = head.next_tokens(logits, d["temperature"], u, None, filters)
    SMP.check(logits, d["temperature"], u, tokens, None, 1, filters.top_k, filters.top_p, filters.min_p)
    mask = torch.zeros((2, V // 32), dtype=torch.int32, device="cuda")
    mask[1, 3] = 6                                                     # ids 97 and 98
    states = torch.tensor([1, 1, 1, -1], dtype=torch.int32, device="cuda")
    again = head.next_tokens(logits, d["temperature"], u, D.Rules(mask=mask), filters, states)
    assert all(t in (97, 98) for t in again[:3].tolist()) and int(again[3]) == int(tokens[3])


def test_refusals(setup):
    X, D, w, ref, block, d, head, filters = setup
    with pytest.raises(ValueError, match="temperature"):
        head.target_logits(d["target"], torch.zeros((b, B), dtype=torch.int32, device="cuda"), None, filters)
    with pytest.raises(ValueError, match="mask_row"):
        head.next_tokens(d["target"][:, 0], d["temperature"], d["temperature"], D.Rules(mask=torch.zeros((1, V // 32), dtype=torch.int32)))
    with pytest.raises(ValueError, match="block"):
        D.DraftHead(ref, head.norm_weight, torch.zeros((V, H), dtype=BF16, device="cuda"),
                    block=D.FeedForward(block.norm_weight, block.W1[:, :-8], block.W2))
