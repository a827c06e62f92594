"""The 8-bit head, the rules, the refinement and the acceptance run together
(draft_head.DraftHead) against the oracle on the same stored inputs: the
head's h, s and the target's rows under the rules are read back bit for bit, and
the oracle refines and accepts from them (integer outputs, compared exactly)."""
import numpy as np
import pytest

import oracle as O
from paper_2608_02438_gb300 import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02438_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.fixture(scope="module")
def setup(X):
    from paper_2608_02438_gb300 import draft_head as D
    cfg = W.tiny_config("head", b=4, B=8, H=512, V=2080, r=256, dtype=W.BF16, temps=(0.0, 1.0), seed=31)
    w = W.make_weights(cfg.H, cfg.V, cfg.r, cfg.B, cfg.dtype, 32, "strong")
    ref = X.Refiner({k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}, cfg.H, cfg.V, cfg.r, cfg.B, X.XPRESS_BF16)
    g = torch.Generator(device="cuda")
    g.manual_seed(33)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    W_lm = (rnd(cfg.V, cfg.H) * 0.1).to(BF16)
    norm = (1 + 0.1 * rnd(cfg.H)).to(BF16)
    d = dict(x=rnd(cfg.b, cfg.B, cfg.H).to(BF16), residual=(2 * rnd(cfg.b, cfg.B, cfg.H)).to(BF16),
             target=(3 * rnd(cfg.b, cfg.B + 1, cfg.V)).to(BF16),
             anchor=torch.randint(0, cfg.V, (cfg.b,), device="cuda", generator=g, dtype=torch.int32),
             temperature=torch.tensor([cfg.temps[i % 2] for i in range(cfg.b)], dtype=torch.float32, device="cuda"),
             seed=torch.arange(cfg.b, device="cuda", dtype=torch.int64) + 77)
    return D, cfg, w, ref, W_lm, norm, d, D.DraftHead(ref, norm, W_lm)


def _rules(D, cfg, grammar):
    rng = np.random.Generator(np.random.PCG64(34))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    lens = np.array([40, 0, 300, 7])
    kw = dict(repetition=dev(rng.uniform(1.0, 1.5, cfg.b).astype(np.float32)),
              presence=dev(rng.uniform(0.0, 1.0, cfg.b).astype(np.float32)),
              history=dev(rng.integers(0, cfg.V, lens.sum()).astype(np.int32)),
              history_offsets=dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)),
              prompt_len=dev((lens // 2).astype(np.int32)))
    bits = rng.random((5, cfg.V)) < np.array([0.5, 0.1, 0.02, 1.0, 0.0])[:, None]
    if grammar:
        # states 0 .. 3 on both kinds of rows; the empty state 4 on one base row
        base = rng.integers(0, 4, cfg.b * cfg.B).astype(np.int32)
        base[3] = 4
        kw.update(mask=dev(np.packbits(bits, axis=1, bitorder="little").view(np.int32)), base_mask_row=dev(base),
                  target_mask_row=dev(rng.integers(0, 4, cfg.b * (cfg.B + 1)).astype(np.int32)))
    return D.Rules(**kw), bits


@pytest.mark.parametrize("use_rules, grammar", [(False, False), (True, False), (True, True)])
def test_round_matches_the_oracle(X, setup, use_rules, grammar):
    D, cfg, w, ref, W_lm, norm, d, head = setup
    rules, bits = _rules(D, cfg, grammar) if use_rules else (None, None)
    out = head.round(d["x"], d["residual"], d["target"], d["anchor"], d["temperature"], d["seed"], 5, cfg.B, rules)
    torch.cuda.synchronize()
    assert ref.device_status("refine", cfg.b) == X.XPRESS_OK and X.matmul_fp8_status() == X.XPRESS_OK
    m = O.Model(w, cfg.H, cfg.V, cfg.r, cfg.B, O.BF16)
    h, s, tgt = _bits(out["h"]), _bits(out["s"]), _bits(out["target"])
    for i in range(cfg.b):
        T = float(d["temperature"][i])
        o = O.jacobi(m, h[i], s[i], int(d["anchor"][i]), out["draft"][i].cpu().numpy(), T, int(d["seed"][i]), 5, cfg.B)
        assert out["tokens"][i].tolist() == o["tokens"].tolist(), f"tokens of block {i}"
        n, ot, _ = O.accept(m, tgt[i], s[i], o["tokens"], o["lse"], o["sel"], o["z_final"], T, int(d["seed"][i]), 5)
        assert int(out["accept_len"][i]) == n and out["out_tokens"][i].tolist() == ot.tolist(), f"acceptance of block {i}"
        if grammar:
            # what is emitted is allowed by the state of its target row
            rows = rules.target_mask_row.view(cfg.b, -1)[i].tolist()
            for j, t in enumerate(out["out_tokens"][i].tolist()):
                assert t < 0 or bits[rows[j]][t]
    # Y^(0) is the first maximum of the stored rows (0 where nothing is allowed)
    s_f = out["s"].float()
    want = s_f.argmax(dim=2).to(torch.int32)
    if grammar:
        want.view(-1)[3] = 0
    assert torch.equal(out["draft"], want)


def test_base_logits_follow_the_unquantised_head(X, setup):
    """s against the bf16 head's product of the same normalised rows: the 8-bit
    operands keep 2^-4 of a value, errors of both signs over 512 terms."""
    D, cfg, w, ref, W_lm, norm, d, head = setup
    out = head.base_logits(d["x"], d["residual"])
    assert torch.equal(out["sum"], (d["x"].float() + d["residual"].float()).to(BF16))
    want = out["h"].reshape(-1, cfg.H).double() @ W_lm.double().t()
    got = out["s"].reshape(-1, cfg.V).double()
    assert (got - want).norm() / want.norm() < 2.0 ** -4


def test_draft_head_refusals(X, setup):
    D, cfg, w, ref, W_lm, norm, d, head = setup
    with pytest.raises(ValueError):
        D.DraftHead(ref, norm, W_lm[:, :-1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side), pytest.raises(ValueError):
        head.round(d["x"], d["residual"], d["target"], d["anchor"], d["temperature"], d["seed"], 5, cfg.B)
