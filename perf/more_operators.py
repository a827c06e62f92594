"""Cases of what stands around the drafter's head: the bf16 matrix product with
bias, activation and residual in its epilogue (the feed-forward block between the
drafter's last layer and the head), and the draw of tokens from logits with
temperature, top-k, top-p and min-p from given random numbers, with the truncated
rows that an acceptance reads.

Every case is a dict of plain values; ``prepare`` makes its inputs on the GPU
from a seed, ``run`` takes one pass through the operator (its plain form in
elementary torch operations, or the framework's entry point when ``own`` is
true), ``exact`` evaluates the definition in 64 bits.
"""
import math

import torch

own = False

VOCAB, HIDDEN, INNER = 151936, 4096, 16384   # the framework's Qwen3-8B shape; a feed-forward block of four times its width
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "silu", "gelu", "relu")
DROPPED = -8192.0                            # what removed logits become, as the acceptance takes masked ones


# ------------------------------------------------------------------- cases

def listed():
    return [
        # product: one token through a square residual block, the smallest call of a decode step
        dict(name="linear_token", op="linear", M=1, N=HIDDEN, K=HIDDEN, out="bf16", bias=True, act="silu", residual=True, pad=0),
        # product: one block of 16 into the feed-forward block, bound by the weights
        dict(name="linear_block16_in", op="linear", M=16, N=INNER, K=HIDDEN, out="bf16", bias=True, act="gelu", residual=False, pad=0),
        # product: sizes that fit no tile, padded rows, 32-bit residual stream
        dict(name="linear_ragged", op="linear", M=77, N=2083, K=1000, out="f32", bias=True, act="relu", residual=True, pad=5),
        # product: out of the feed-forward block for 32 blocks of 16
        dict(name="linear_serving_out", op="linear", M=512, N=HIDDEN, K=INNER, out="bf16", bias=True, act="none", residual=True, pad=0),
        # product: a long prompt's positions into the feed-forward block, bound by the tensor cores
        dict(name="linear_prompt_in", op="linear", M=16384, N=INNER, K=HIDDEN, out="bf16", bias=True, act="silu", residual=False, pad=0),
        # draw: the next token of one request with the usual filters
        dict(name="sample_token", op="sample", b=1, R=1, V=VOCAB, dtype="bf16", sigma=4.0, T=0.7, k=50, p=0.9, min_p=0.0, out=False, pad=0),
        # draw: the next tokens of a batch from the whole softmax
        dict(name="sample_batch_plain", op="sample", b=64, R=1, V=VOCAB, dtype="bf16", sigma=4.0, T=1.0, k=0, p=1.0, min_p=0.0, out=False, pad=0),
        # draw: a batch of flat rows (a small odd vocabulary in 32 bits, half of it forbidden) whose nucleus has thousands of tokens
        dict(name="sample_flat_f32", op="sample", b=48, R=1, V=32003, dtype="f32", sigma=1.5, T=1.2, k=0, p=0.95, min_p=0.0, out=False, pad=0),
        # truncation: the target's rows of one block and its bonus row
        dict(name="truncate_block", op="sample", b=1, R=17, V=VOCAB, dtype="bf16", sigma=4.0, T=1.0, k=20, p=0.95, min_p=0.0, out=True, pad=0),
        # truncation: the target's rows of a batch of 32, each request with filters of its own
        dict(name="truncate_serving", op="sample", b=32, R=17, V=VOCAB, dtype="bf16", sigma=4.0, T=0.9, k=-1, p=0.9, min_p=0.05, out=True, pad=0),
        # truncation: 32-bit rows that start anywhere, a large top-k
        dict(name="truncate_f32_odd", op="sample", b=8, R=17, V=50021, dtype="f32", sigma=3.0, T=1.0, k=1000, p=0.98, min_p=0.0, out=True, pad=3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _snap(rng, n):
    """Half of the sizes as real models have them (multiples of 64), half as they come."""
    return n if n < 64 or rng.random() < 0.5 else n // 64 * 64


def draw(rng):
    if rng.random() < 0.5:
        K = _snap(rng, _log_int(rng, 64, INNER))
        N = _snap(rng, _log_int(rng, 64, INNER))
        M = _log_int(rng, 1, 16384 if rng.random() < 0.5 else 512)
        M = max(1, min(M, 16384 * INNER * HIDDEN // (N * K)))
        return dict(op="linear", M=M, N=N, K=K, out=rng.choice(["bf16", "bf16", "f32"]) if M * N < 2 ** 26 else "bf16",
                    bias=rng.random() < 0.7, act=rng.choice(ACTS), residual=rng.random() < 0.6, pad=rng.choice([0, 0, 0, 8, 3]))
    V = _snap(rng, _log_int(rng, 64, VOCAB))
    R = rng.choice([1, 1, 1, 17, 5, 33])
    b = _log_int(rng, 1, max(1, 32 * 17 // R))
    k = rng.choice([0, 0, -1, 1, 20, 50, 1000, V // 2])
    return dict(op="sample", b=b, R=R, V=V, dtype=rng.choice(["bf16", "bf16", "f32"]) if b * R * V < 2 ** 25 else "bf16",
                sigma=rng.choice([1.5, 3.0, 4.0]), T=rng.choice([0.3, 0.7, 1.0, 1.5]), k=k, p=rng.choice([1.0, 1.0, 0.95, 0.8, 0.3]),
                min_p=rng.choice([0.0, 0.0, 0.05]), out=R > 1 or rng.random() < 0.2, pad=rng.choice([0, 0, 0, 8, 3]))


# ------------------------------------------------------------------ inputs

def _rows(rows, cols, dtype, pad):
    """An uninitialised [rows, cols] whose rows are `pad` elements apart."""
    return torch.empty((rows, cols + pad), dtype=dtype, device="cuda")[:, :cols]


def _operand(rows, cols, scale, g):
    """A bf16 operand [rows, cols] whose rows start on 16 bytes."""
    t = torch.empty((rows, -(-cols // 8) * 8), dtype=torch.bfloat16, device="cuda")
    t.normal_(0.0, scale, generator=g)
    return t[:, :cols]


def _prepare_linear(case, g):
    M, N, K = case["M"], case["N"], case["K"]
    dt = DTYPES[case["out"]]
    st = dict(x=_operand(M, K, 1.0, g), w=_operand(N, K, 1.5 / math.sqrt(K), g), bias=None, act=case["act"], residual=None,
              out=_rows(M, N, dt, case["pad"]))
    if case["bias"]:
        st["bias"] = (0.3 * torch.randn(N, device="cuda", generator=g)).to(torch.bfloat16)
    if case["residual"]:
        st["residual"] = _rows(M, N, dt, case["pad"])
        st["residual"].normal_(0.0, 2.0, generator=g)
    return st


def _prepare_sample(case, g):
    b, R, V = case["b"], case["R"], case["V"]
    n = b * R
    rnd = lambda *s: torch.rand(s, device="cuda", generator=g)  # noqa: E731
    logits = _rows(n, V, DTYPES[case["dtype"]], case["pad"])
    logits.normal_(0.0, case["sigma"], generator=g)
    # every third row is sure of one token or two
    sure = torch.arange(0, n, 3, device="cuda")
    for lift in (10.0, 8.0):
        at = (V * rnd(len(sure))).long().clamp_(max=V - 1)
        logits[sure, at] += lift * case["sigma"] / 4.0
    if case["dtype"] == "f32":
        logits[:, 1::2] = float("-inf")                            # a grammar that forbids every other token
        if n > 2:
            logits[2] = float("-inf")                              # ... or all of them
    T = case["T"] * (0.8 + 0.4 * rnd(b))
    k = None
    if case["k"] > 0:
        k = torch.full((b,), case["k"], dtype=torch.int32, device="cuda")
    elif case["k"] < 0:                                            # requests of all kinds: no top-k, 1, 20, 50, 300
        kinds = torch.tensor([0, 20, 50, 300, 1], dtype=torch.int32, device="cuda")
        k = kinds[torch.arange(b, device="cuda") % 5]
        T[b // 2::7] = 0.0                                         # and greedy ones
    p = None
    if case["p"] < 1.0:
        p = (case["p"] + (1.0 - case["p"]) * 0.5 * rnd(b)).clamp_(max=0.999)
        p[3::8] = 1.0                                              # requests without
    min_p = None
    if case["min_p"] > 0.0:
        min_p = case["min_p"] * rnd(b)
        min_p[1::2] = 0.0
    return dict(logits=logits, rows=R, temperature=T, top_k=k, top_p=p, min_p=min_p, u=rnd(n),
                tokens=torch.empty(n, dtype=torch.int32, device="cuda"),
                out=_rows(n, V, logits.dtype, case["pad"]) if case["out"] else None)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    st = dict(linear=_prepare_linear, sample=_prepare_sample)[case["op"]](case, g)
    st["op"] = case["op"]
    return st


# -------------------------------------------------------------- plain forms

def _plain_linear(st):
    y = st["x"].float() @ st["w"].float().t()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    if st["act"] == "silu":
        y = y * torch.sigmoid(y)
    elif st["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif st["act"] == "relu":
        y = y.clamp(min=0.0)
    if st["residual"] is not None:
        y = st["residual"].float() + y
    return dict(out=y.to(st["out"].dtype))


def _plain_sample_rows(l, T, k, p, min_p, u):
    """Tokens and kept places of the rows l (fp32): masses in 64 bits, since what
    decides is next to a border."""
    n, V = l.shape
    l = torch.where(l.isnan(), torch.full_like(l, float("-inf")), l) + 0.0
    order = torch.sort(l, dim=1, descending=True, stable=True)
    top = order.values[:, :1]
    greedy = T <= 0.0
    z = (order.values.double() - top.double()) / torch.where(greedy, torch.ones_like(T), T).double()[:, None]
    w = torch.where(order.values > float("-inf"), torch.exp(z), torch.zeros_like(z))
    rank = torch.arange(V, device=l.device)[None, :]
    keep = order.values > float("-inf")
    if min_p is not None:
        keep &= w >= min_p.double()[:, None]
    if k is not None:
        keep &= (rank < k[:, None]) | (k <= 0)[:, None]
    keep &= (rank == 0) | ~greedy[:, None]
    w = w * keep
    if p is not None:
        mass = w.cumsum(dim=1)
        before = torch.nn.functional.pad(mass[:, :-1], (1, 0))
        keep &= (before < p.double()[:, None] * mass[:, -1:]) | (p >= 1.0)[:, None] | (rank == 0)
        w = w * keep
    # back to the order of the ids
    kept = torch.zeros_like(keep).scatter_(1, order.indices, keep)
    mass = torch.zeros_like(w).scatter_(1, order.indices, w).cumsum(dim=1)
    token = (mass <= u.double()[:, None] * mass[:, -1:]).sum(dim=1).clamp(max=V - 1)
    return torch.where(top[:, 0] > float("-inf"), token, torch.full_like(token, -1)).to(torch.int32), kept


def _plain_sample(st):
    logits, R = st["logits"], st["rows"]
    n, V = logits.shape
    spread = lambda t: None if t is None else t.repeat_interleave(R)  # noqa: E731
    T, k, p, min_p = (spread(st[name]) for name in ("temperature", "top_k", "top_p", "min_p"))
    cut = lambda t, at: None if t is None else t[at]  # noqa: E731
    tokens, outs = [], []
    step = max(1, (1 << 26) // V)                                  # the 64-bit arrays of some rows at a time
    for i in range(0, n, step):
        at = slice(i, min(n, i + step))
        tok, kept = _plain_sample_rows(logits[at].float(), T[at], cut(k, at), cut(p, at), cut(min_p, at), st["u"][at])
        tokens.append(tok)
        if st["out"] is not None:
            outs.append(torch.where(kept, logits[at], torch.full_like(logits[at], DROPPED)))
    out = dict(tokens=torch.cat(tokens))
    if st["out"] is not None:
        out["out"] = torch.cat(outs)
    return out


# --------------------------------------------------------------------- run

def run(state):
    op = state["op"]
    if not own:
        return dict(linear=_plain_linear, sample=_plain_sample)[op](state)
    from paper_2608_02438_gb300 import binding as X
    if op == "linear":
        act = dict(none=X.XPRESS_ACT_NONE, silu=X.XPRESS_ACT_SILU, gelu=X.XPRESS_ACT_GELU, relu=X.XPRESS_ACT_RELU)[state["act"]]
        X.linear(state["x"], state["w"], state["out"], bias=state["bias"], act=act, residual=state["residual"])
        return dict(out=state["out"])
    X.sample(state["logits"], state["temperature"], u=state["u"], tokens_out=state["tokens"], out=state["out"],
             rows=state["rows"], top_k=state["top_k"], top_p=state["top_p"], min_p=state["min_p"], mask_value=DROPPED)
    out = dict(tokens=state["tokens"])
    if state["out"] is not None:
        out["out"] = state["out"]
    return out


# -------------------------------------------------------------------- work

def work(case):
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        es = {"bf16": 2, "f32": 4}[case["out"]]
        return dict(bytes=2 * (M + N) * K + (2 * N if case["bias"] else 0) + M * N * es * (2 if case["residual"] else 1),
                    flops=2 * M * N * K)
    n, es = case["b"] * case["R"], {"bf16": 2, "f32": 4}[case["dtype"]]
    return dict(bytes=n * case["V"] * es * (2 if case["out"] else 1) + 8 * n + 16 * case["b"], flops=4 * n * case["V"])


# ------------------------------------------------------------------- exact

def _exact_linear(st):
    y = torch.mm(st["x"].double(), st["w"].double().t())
    if st["bias"] is not None:
        y += st["bias"].double()
    if st["act"] == "silu":
        y /= 1.0 + torch.exp(-y)
    elif st["act"] == "gelu":
        y *= 0.5 * torch.erfc(-y / math.sqrt(2.0))
    elif st["act"] == "relu":
        y = torch.maximum(y, torch.zeros_like(y))
    if st["residual"] is not None:
        y += st["residual"].double()
    return dict(out=y)


def _exact_sample(st):
    logits, R = st["logits"], st["rows"]
    n, V = logits.shape
    get = lambda name, off: [off] * (n // R) if st[name] is None else st[name].tolist()  # noqa: E731
    temps, ks, ps, mins, us = get("temperature", 0.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0), st["u"].tolist()
    tokens = torch.full((n,), -1, dtype=torch.int32, device=logits.device)
    out = None if st["out"] is None else torch.full((n, V), DROPPED, dtype=torch.float64, device=logits.device)
    for i in range(n):
        q = i // R
        l = logits[i].double()
        ids = torch.nonzero(l > float("-inf"))[:, 0]               # ascending
        if len(ids) == 0:
            continue
        l = l[ids]
        l, at = torch.sort(l, descending=True, stable=True)        # ties: the lowest id first
        ids = ids[at]
        if temps[q] <= 0.0:
            ids, l, w = ids[:1], l[:1], torch.ones_like(l[:1])
        else:
            if 0 < ks[q] < len(l):
                l, ids = l[:ks[q]], ids[:ks[q]]
            if mins[q] > 0.0:
                m = max(1, int((l >= l[0] + temps[q] * math.log(mins[q])).sum()))
                l, ids = l[:m], ids[:m]
            w = torch.exp((l - l[0]) / temps[q])
            if ps[q] < 1.0:
                mass = w.cumsum(0)
                m = int((mass < ps[q] * mass[-1]).sum()) + 1       # the first token that reaches it is the last one kept
                l, ids, w = l[:m], ids[:m], w[:m]
        ids, at = torch.sort(ids)
        mass = w[at].cumsum(0)
        j = min(int((mass <= us[i] * mass[-1]).sum()), len(ids) - 1)
        tokens[i] = ids[j].to(torch.int32)
        if out is not None:
            out[i, ids] = l[at]
    res = dict(tokens=tokens)
    if out is not None:
        res["out"] = out
    return res


def exact(case, seed):
    st = prepare(case, seed)
    return dict(linear=_exact_linear, sample=_exact_sample)[case["op"]](st)
