"""DraftHead's wiring of the request's rules: the base and target rows that come out of it
against the definition of the rules (that of test_gpu_logits) on the rows that went in, with
one rule at a time and with all of them; and what an empty grammar state emits."""
import numpy as np
import pytest

import oracle as O
import test_gpu_logits as L
from paper_2608_02438_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
f4 = np.float32
b, B, H, V = 4, 8, 512, 2080
X = L.X                                          # the module's fixture


@pytest.fixture(scope="module")
def setup(X):
    from paper_2608_02438_gb300 import draft_head as D
    w = W.make_weights(H, V, 256, B, W.BF16, 41, "strong")
    ref = X.Refiner({k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}, H, V, 256, B, X.XPRESS_BF16)
    g = torch.Generator(device="cuda")
    g.manual_seed(42)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    W_lm = (rnd(V, H) * 0.1).to(BF16)
    norm = (1 + 0.1 * rnd(H)).to(BF16)
    d = dict(x=rnd(b, B, H).to(BF16), residual=(2 * rnd(b, B, H)).to(BF16), target=(3 * rnd(b, B + 1, V)).to(BF16),
             anchor=torch.randint(0, V, (b,), device="cuda", generator=g, dtype=torch.int32),
             temperature=torch.zeros(b, device="cuda"), seed=torch.arange(b, device="cuda", dtype=torch.int64) + 5)
    return D, w, ref, W_lm, norm, d, D.DraftHead(ref, norm, W_lm)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


ALL = ("repetition", "frequency", "presence", "bias", "grammar")


def _rules(D, on):
    """Rules with those of ALL that are in `on`, and the two definitions' cases (base, target)."""
    rng = np.random.Generator(np.random.PCG64(43))
    lens = [40, 0, 300, 7]
    hist = [rng.integers(0, V, n).astype(np.int32) for n in lens]
    plen = np.array([n // 2 for n in lens], np.int32)
    rep, freq, pres = (rng.uniform(lo, hi, b).astype(f4) for lo, hi in ((1.1, 1.6), (0.2, 0.9), (0.2, 0.9)))
    bias = [(rng.choice(V, 20, replace=False).astype(np.int32), rng.normal(0, 3, 20).astype(f4)) for _ in range(b)]
    bits = rng.random((4, V)) < np.array([0.5, 0.1, 0.02, 1.0])[:, None]
    mask = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
    base_row, target_row = (rng.integers(-1, 4, b * n).astype(np.int32) for n in (B, B + 1))
    kw = dict(history=_dev(np.concatenate(hist)), history_offsets=_dev(L._offsets(lens)), prompt_len=_dev(plen))
    if "repetition" in on: kw["repetition"] = _dev(rep)                                  # noqa: E701
    if "frequency" in on: kw["frequency"] = _dev(freq)                                   # noqa: E701
    if "presence" in on: kw["presence"] = _dev(pres)                                     # noqa: E701
    if "bias" in on:
        kw.update(bias_ids=_dev(np.concatenate([i for i, _ in bias])), bias_values=_dev(np.concatenate([v for _, v in bias])),
                  bias_offsets=_dev(L._offsets([20] * b)))
    if "grammar" in on:
        kw.update(mask=_dev(mask), base_mask_row=_dev(base_row), target_mask_row=_dev(target_row))
    c = dict(b=b, V=V, hist=hist, plen=plen, rep=rep if "repetition" in on else np.ones(b, f4),
             freq=freq if "frequency" in on else np.zeros(b, f4), pres=pres if "presence" in on else np.zeros(b, f4),
             bias=bias if "bias" in on else None, bits=bits, mask=mask if "grammar" in on else None)
    return D.Rules(**kw), dict(c, R=B, draft=None, mask_row=base_row), dict(c, R=B + 1, mask_row=target_row)


@pytest.mark.parametrize("on", [()] + [(k,) for k in ALL] + [ALL[:4], ALL])
def test_rows_are_those_of_the_definition(X, setup, on):
    D, w, ref, W_lm, norm, d, head = setup
    rules, base, target = _rules(D, on)
    out = head.round(d["x"], d["residual"], d["target"], d["anchor"], d["temperature"], d["seed"], 5, B, rules)
    # the base rows that went in: the head's product is reproducible
    q, sc = X.alloc_e4m3(b * B, H), torch.empty((b * B, H // 128), device="cuda")
    s = torch.empty((b * B, V), dtype=BF16, device="cuda")
    X.rmsnorm(d["x"].view(-1, H), norm, head.eps, residual=d["residual"].view(-1, H), q_out=q, scale_out=sc)
    X.matmul_fp8(q, sc, *X.quantize_weight(W_lm), s)
    torch.cuda.synchronize()
    L._check(base, s, out["s"].view(-1, V), out["draft"].view(-1), D.MASKED)
    # the target's rows count the refined block's tokens
    target["draft"] = out["tokens"].cpu().numpy()
    L._check(target, d["target"].view(-1, V), out["target"].view(-1, V), None, D.MASKED)
    # each rule does something here, so that one that was not passed on would show
    changed = (out["s"].view(-1, V) != s).any(dim=1), (out["target"] != d["target"]).any(dim=2)
    assert bool(changed[0].any()) == bool(on) and bool(changed[1].any()) == bool(on)


@pytest.mark.parametrize("on", ["repetition", "frequency", "presence"])
def test_target_rows_count_the_block_itself(X, setup, on):
    """No history: what changes in a target row are the block's own tokens before it."""
    D, w, ref, W_lm, norm, d, head = setup
    rules, _, _ = _rules(D, (on,))
    rules.history, rules.history_offsets, rules.prompt_len = None, None, None
    tokens = torch.randint(0, V, (b, B), device="cuda", dtype=torch.int32)
    out = head.target_logits(d["target"], tokens, rules)
    changed = out != d["target"]
    for i in range(b):
        for j in range(B + 1):
            seen = set(tokens[i, :j].tolist())
            assert set(torch.nonzero(changed[i, j]).view(-1).tolist()) <= seen
            assert j < 2 or bool(changed[i, j].any())


def test_a_target_state_that_allows_nothing(X, setup):
    """Its row is MASKED throughout, and the acceptance emits id 0 from it at temperature 0, as
    Rules says: the request has to be ended by its caller."""
    D, w, ref, W_lm, norm, d, head = setup
    mask = torch.full((2, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    mask[1] = 0
    rows = torch.zeros((b, B + 1), dtype=torch.int32, device="cuda")
    rows[:, 0] = 1
    rules = D.Rules(mask=mask, base_mask_row=torch.zeros(b * B, dtype=torch.int32, device="cuda"),
                    target_mask_row=rows.view(-1))
    tgt = d["target"].clone()
    out = head.round(d["x"], d["residual"], tgt, d["anchor"], d["temperature"], d["seed"], 5, B, rules)
    torch.cuda.synchronize()
    assert (out["target"][:, 0] == D.MASKED).all() and torch.equal(out["target"][:, 1:], tgt[:, 1:])
    assert (out["out_tokens"][:, 0] == 0).all()
    m = O.Model(w, H, V, 256, B, O.BF16)
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    for i in range(b):
        o = O.jacobi(m, bits(out["h"][i]), bits(out["s"][i]), int(d["anchor"][i]), out["draft"][i].cpu().numpy(), 0.0,
                     int(d["seed"][i]), 5, B)
        n, ot, _ = O.accept(m, bits(out["target"][i]), bits(out["s"][i]), o["tokens"], o["lse"], o["sel"], o["z_final"], 0.0,
                            int(d["seed"][i]), 5)
        assert int(out["accept_len"][i]) == n and out["out_tokens"][i].tolist() == ot.tolist()
