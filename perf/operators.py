"""Cases of the 8-bit drafter head: the final norm with its 8-bit output, the
weights' quantisation, the block-scaled 8-bit matrix product and the request's
rules on the logits.

Every case is a dict of plain values; ``prepare`` makes its inputs on the GPU
from a seed, ``run`` takes one pass through the operator (its plain form in
elementary torch operations, or the framework's entry point when ``own`` is
true), ``exact`` evaluates the definition in 64 bits.
"""
import math

import torch

own = False

BLOCK = 128                  # elements that share a scale along K, and rows of a weight block
FP8_MAX = 448.0              # largest e4m3 value
MIN_SCALE = 2.0 ** -126      # scale of an all-zero group
EPS = 1e-6

VOCAB, HIDDEN, RANK = 151936, 4096, 256      # the framework's Qwen3-8B shape
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------- cases

def listed():
    return [
        # norm: one token of a single request, where latency counts
        dict(name="norm_token", op="norm", rows=1, H=HIDDEN, dtype="bf16", residual=True, q=True, pad=0),
        # norm: a batch of 32 blocks of 16 in 32 bits, an odd hidden size and padded rows (no vector fits)
        dict(name="norm_f32_odd", op="norm", rows=512, H=4099, dtype="f32", residual=False, q=True, pad=5),
        # norm: the positions of a long prompt
        dict(name="norm_prompt", op="norm", rows=16384, H=HIDDEN, dtype="bf16", residual=True, q=True, pad=0),
        # weights: one of the refiner-sized matrices (2r x r), ragged against the 128-blocks
        dict(name="quant_small", op="quant", rows=2 * RANK + 5, cols=RANK + 24, dtype="f32"),
        # weights: the LM head of the Qwen3-8B shape, once per load
        dict(name="quant_lm_head", op="quant", rows=VOCAB, cols=HIDDEN, dtype="bf16"),
        # product: one token against a square projection, the smallest call of a decode step
        dict(name="mm_token_square", op="mm", M=1, N=HIDDEN, K=HIDDEN, dtype="bf16"),
        # product: base logits of one block of 16 (the benchmark's request), bound by the weights
        dict(name="mm_block16_lm_head", op="mm", M=16, N=VOCAB, K=HIDDEN, dtype="bf16"),
        # product: sizes that fit no tile, 32-bit output
        dict(name="mm_ragged", op="mm", M=77, N=2088, K=1000, dtype="f32"),
        # product: base logits of 64 blocks of 32, bound by the tensor cores
        dict(name="mm_long_lm_head", op="mm", M=2048, N=VOCAB, K=HIDDEN, dtype="bf16"),
        # rules: the next token of one request with a short history
        dict(name="rules_token", op="rules", b=1, R=1, V=VOCAB, dtype="bf16", hist=700, n_bias=20, masked=1.0, draft=False),
        # rules: target rows (block and bonus) of a batch of 32 under a grammar
        dict(name="rules_serving", op="rules", b=32, R=17, V=VOCAB, dtype="bf16", hist=6000, n_bias=300, masked=0.5, draft=True),
        # rules: 32-bit logits of a small odd vocabulary, long histories
        dict(name="rules_f32_odd", op="rules", b=6, R=5, V=32003, dtype="f32", hist=40000, n_bias=0, masked=0.3, draft=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _snap(rng, n):
    """Half of the sizes as real models have them (multiples of 64), half as they come."""
    return n if n < 64 or rng.random() < 0.5 else n // 64 * 64


def draw(rng):
    op = rng.choice(["norm", "quant", "mm", "rules"])
    if op == "norm":
        H = _snap(rng, _log_int(rng, 64, 8192))
        rows = _log_int(rng, 1, min(16384, 16384 * HIDDEN // H))
        return dict(op=op, rows=rows, H=H, dtype=rng.choice(["bf16", "bf16", "f32"]) if rows * H < 2 ** 25 else "bf16",
                    residual=rng.random() < 0.6, q=rng.random() < 0.8, pad=rng.choice([0, 0, 0, 8, 3]))
    if op == "quant":
        cols = _snap(rng, _log_int(rng, 64, 8192))
        rows = _log_int(rng, 1, min(VOCAB, VOCAB * HIDDEN // cols))
        return dict(op=op, rows=rows, cols=cols, dtype="f32" if rows * cols < 2 ** 28 and rng.random() < 0.3 else "bf16")
    if op == "mm":
        K = _snap(rng, _log_int(rng, 64, 8192))
        N = _snap(rng, _log_int(rng, 64, min(VOCAB, VOCAB * HIDDEN // K)))
        return dict(op=op, M=_log_int(rng, 1, 2048), N=N, K=K, dtype=rng.choice(["bf16", "bf16", "f32"]))
    V = _snap(rng, _log_int(rng, 1000, VOCAB))
    R = rng.choice([1, 1, 16, 17, 5, 33])
    b = _log_int(rng, 1, max(1, 32 * 17 // R))
    return dict(op=op, b=b, R=R, V=V, dtype=rng.choice(["bf16", "bf16", "f32"]) if b * R * V < 2 ** 25 else "bf16",
                hist=_log_int(rng, 1, 40000 if b <= 8 else 8000), n_bias=rng.choice([0, 1, 30, 300]),
                masked=rng.choice([0.0, 0.3, 1.0]), draft=R > 1 and rng.random() < 0.7)


# ------------------------------------------------------------------ inputs

def _pitched(rows, cols, dtype, device, align):
    """[rows, cols] whose rows start `align` elements apart (rounded up)."""
    return torch.empty((rows, -(-cols // align) * align), dtype=dtype, device=device)[:, :cols]


def _prepare_norm(case, g):
    dt, H, rows, pad = DTYPES[case["dtype"]], case["H"], case["rows"], case["pad"]

    def rows_of(scale):
        t = torch.empty((rows, H + pad), dtype=dt, device="cuda")
        t.normal_(0.0, scale, generator=g)
        return t[:, :H]

    x, res = rows_of(1.0), rows_of(2.0) if case["residual"] else None
    x[:, :: 257] *= 12.0                                           # the few large channels that hidden states have
    w = (1.0 + 0.2 * torch.randn(H, device="cuda", generator=g)).to(dt)
    new = lambda: torch.empty((rows, H + pad), dtype=dt, device="cuda")[:, :H]  # noqa: E731
    return dict(x=x, residual=res, weight=w, sum_out=new() if res is not None else None, y_out=new(),
                q_out=_pitched(rows, H, torch.float8_e4m3fn, "cuda", 16) if case["q"] else None,
                scale_out=torch.empty((rows, -(-H // BLOCK)), device="cuda") if case["q"] else None)


def _prepare_quant(case, g):
    rows, cols = case["rows"], case["cols"]
    W = torch.empty((rows, cols), dtype=DTYPES[case["dtype"]], device="cuda")
    W.normal_(0.0, 0.02, generator=g)
    return dict(W=W, q_out=_pitched(rows, cols, torch.float8_e4m3fn, "cuda", 16),
                scale_out=torch.empty((-(-rows // BLOCK), -(-cols // BLOCK)), device="cuda"))


def _prepare_mm(case, g):
    M, N, K = case["M"], case["N"], case["K"]
    KB = -(-K // BLOCK)

    def values(rows):
        # e4m3 values as a quantiser leaves them: each group's largest near 448
        t = _pitched(rows, K, torch.float8_e4m3fn, "cuda", 16)
        step = max(1, (1 << 27) // max(K, 1))
        for r in range(0, rows, step):
            n = min(step, rows - r)
            t[r:r + n] = (torch.randn((n, K), device="cuda", generator=g) * 130.0).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
        return t

    scales = lambda r, mean: mean * (0.5 + torch.rand((r, KB), device="cuda", generator=g))  # noqa: E731
    return dict(a=values(M), a_scale=scales(M, 0.01), w=values(N), w_scale=scales(-(-N // BLOCK), 2e-4),
                out=torch.empty((M, N), dtype=DTYPES[case["dtype"]], device="cuda"))


def _prepare_rules(case, g):
    b, R, V = case["b"], case["R"], case["V"]
    rnd = lambda *s: torch.rand(s, device="cuda", generator=g)  # noqa: E731
    logits = torch.empty((b * R, V), dtype=DTYPES[case["dtype"]], device="cuda")
    logits.normal_(0.0, 4.0, generator=g)
    # histories of uneven length (one of them empty in a batch), frequent tokens first
    share = rnd(b).cpu()
    lens = [max(1, int(case["hist"] * (0.5 + 0.5 * float(u)))) for u in share]
    if b > 2:
        lens[1] = 0
    offsets = torch.tensor([0] + lens, dtype=torch.int64).cumsum(0)
    history = (V * rnd(int(offsets[-1])) ** 3).to(torch.int32).clamp_(max=V - 1)
    prompt_len = torch.tensor([n // 3 for n in lens], dtype=torch.int32)
    repetition = 1.0 + 0.5 * rnd(b)
    repetition[: b // 4] = 1.0                                     # requests without a repetition penalty
    st = dict(logits=logits, rows=R, out=torch.empty_like(logits),
              argmax_out=torch.empty(b * R, dtype=torch.int32, device="cuda"), repetition=repetition, frequency=rnd(b),
              presence=rnd(b), history=history, history_offsets=offsets.cuda(), prompt_len=prompt_len.cuda(),
              draft=None, bias_ids=None, bias_values=None, bias_offsets=None, mask=None, mask_row=None)
    if case["draft"]:
        draft = (V * rnd(b, R - 1) ** 3).to(torch.int32).clamp_(max=V - 1)
        draft[:, (R - 1) // 2] = draft[:, 0]                       # a token that the block repeats
        st["draft"] = draft
    if case["n_bias"]:
        n = min(case["n_bias"], V)
        st["bias_ids"] = torch.cat([torch.randperm(V, device="cuda", generator=g)[:n] for _ in range(b)]).to(torch.int32)
        st["bias_values"] = 6.0 * rnd(b * n) - 3.0
        st["bias_offsets"] = torch.arange(b + 1, device="cuda", dtype=torch.int64) * n
    if case["masked"] > 0:
        # grammar states: most allow nearly everything or a few tokens, and one allows nothing
        states = max(2, int(b * R * case["masked"]))
        words = -(-V // 32)
        allow = torch.tensor([0.9, 0.002, 0.3], device="cuda")[torch.arange(states, device="cuda") % 3]
        allow[1] = 0.0
        mask = torch.zeros((states, words), dtype=torch.int32, device="cuda")
        for j in range(32):
            bit = (rnd(states, words) < allow[:, None]).to(torch.int32)
            mask |= bit << j
        st["mask"] = mask
        at = torch.arange(b * R, device="cuda", dtype=torch.int32)
        st["mask_row"] = torch.where(at < states, at, torch.full_like(at, -1))
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    st = dict(norm=_prepare_norm, quant=_prepare_quant, mm=_prepare_mm, rules=_prepare_rules)[case["op"]](case, g)
    st["op"] = case["op"]
    return st


# -------------------------------------------------------------- plain forms

def _groups(t):
    """[rows, H] as [rows, groups, 128], the last group filled with zeros."""
    rows, H = t.shape
    n = -(-H // BLOCK)
    return torch.nn.functional.pad(t, (0, n * BLOCK - H)).view(rows, n, BLOCK)


def _plain_norm(st):
    x, res = st["x"], st["residual"]
    t = x.float() if res is None else x.float() + res.float()
    y = t * torch.rsqrt((t * t).mean(dim=1, keepdim=True) + EPS) * st["weight"].float()
    out = dict(y=y.to(x.dtype))
    if res is not None:
        out["sum"] = t.to(x.dtype)
    if st["q_out"] is not None:
        yg = _groups(y)
        scale = (yg.abs().amax(dim=2) / FP8_MAX).clamp(min=MIN_SCALE)
        out["q"] = (yg / scale[:, :, None]).view(y.shape[0], -1)[:, :y.shape[1]].to(torch.float8_e4m3fn)
        out["scale"] = scale
    return out


def _plain_quant(st):
    W = st["W"].float()
    rows, cols = W.shape
    nr, nc = -(-rows // BLOCK), -(-cols // BLOCK)
    Wb = torch.nn.functional.pad(W, (0, nc * BLOCK - cols, 0, nr * BLOCK - rows)).view(nr, BLOCK, nc, BLOCK)
    scale = (Wb.abs().amax(dim=(1, 3)) / FP8_MAX).clamp(min=MIN_SCALE)
    q = (Wb / scale[:, None, :, None]).view(nr * BLOCK, nc * BLOCK)[:rows, :cols]
    return dict(q=q.to(torch.float8_e4m3fn), scale=scale)


def _plain_mm(st):
    a, w, K = st["a"], st["w"], st["a"].shape[1]
    A = a.float() * st["a_scale"].repeat_interleave(BLOCK, dim=1)[:, :K]
    sw = st["w_scale"].repeat_interleave(BLOCK, dim=1)[:, :K].repeat_interleave(BLOCK, dim=0)[:w.shape[0]]
    return dict(out=(A @ (w.float() * sw).t()).to(st["out"].dtype))


def _plain_rules(st):
    logits, R = st["logits"], st["rows"]
    n, V = logits.shape
    b, dev = n // R, logits.device
    x = logits.float().view(b, R, V)
    # how often each id was answered, and whether it stands in the prompt
    lens = st["history_offsets"][1:] - st["history_offsets"][:-1]
    seq = torch.repeat_interleave(torch.arange(b, device=dev), lens, output_size=st["history"].numel())
    pos = torch.arange(st["history"].numel(), device=dev) - st["history_offsets"][:-1][seq]
    at = seq * V + st["history"].long()
    answered = (pos >= st["prompt_len"][seq]).to(torch.int32)
    counts = torch.zeros(b * V, dtype=torch.int32, device=dev).scatter_add_(0, at, answered).view(b, 1, V)
    prompt = torch.zeros(b * V, dtype=torch.int32, device=dev).scatter_add_(0, at, 1 - answered).view(b, 1, V)
    if st["draft"] is not None:
        # row j also counts the block's tokens 0 .. j-1
        e = torch.zeros((b, R, V), dtype=torch.int32, device=dev)
        d = st["draft"].long()
        e[:, 1:].scatter_add_(2, d[:, :, None], torch.ones_like(d, dtype=torch.int32)[:, :, None])
        counts = counts + e.cumsum(dim=1, dtype=torch.int32)
    col = lambda v: v.view(b, 1, 1)  # noqa: E731
    rep = col(st["repetition"])
    y = torch.where((counts > 0) | (prompt > 0), torch.where(x > 0, x / rep, x * rep), x)
    y = y - col(st["frequency"]) * counts - col(st["presence"]) * (counts > 0)
    if st["bias_ids"] is not None:
        nb = st["bias_offsets"][1:] - st["bias_offsets"][:-1]
        seq = torch.repeat_interleave(torch.arange(b, device=dev), nb, output_size=st["bias_ids"].numel())
        bias = torch.zeros(b * V, device=dev)
        bias[seq * V + st["bias_ids"].long()] = st["bias_values"]
        y = y + bias.view(b, 1, V)
    y = y.reshape(n, V)
    allowed = None
    if st["mask"] is not None:
        rows = st["mask_row"].long()
        words = st["mask"][rows.clamp(min=0)]
        bits = (words[:, :, None] >> torch.arange(32, device=dev, dtype=torch.int32)) & 1
        allowed = (bits.reshape(n, -1)[:, :V] != 0) | (rows < 0)[:, None]
        y = torch.where(allowed, y, torch.full_like(y, float("-inf")))
    out = y.to(logits.dtype)
    best = out.float().argmax(dim=1).to(torch.int32)
    if allowed is not None:
        best = torch.where(allowed.any(dim=1), best, torch.full_like(best, -1))
    return dict(out=out, argmax=best)


# --------------------------------------------------------------------- run

def run(state):
    op = state["op"]
    if not own:
        return dict(norm=_plain_norm, quant=_plain_quant, mm=_plain_mm, rules=_plain_rules)[op](state)
    from paper_2608_02438_gb300 import binding as X
    if op == "norm":
        X.rmsnorm(state["x"], state["weight"], EPS, residual=state["residual"], sum_out=state["sum_out"],
                  y_out=state["y_out"], q_out=state["q_out"], scale_out=state["scale_out"])
        out = dict(y=state["y_out"])
        if state["residual"] is not None:
            out["sum"] = state["sum_out"]
        if state["q_out"] is not None:
            out["q"], out["scale"] = state["q_out"], state["scale_out"]
        return out
    if op == "quant":
        X.quantize_weight(state["W"], state["q_out"], state["scale_out"])
        return dict(q=state["q_out"], scale=state["scale_out"])
    if op == "mm":
        X.matmul_fp8(state["a"], state["a_scale"], state["w"], state["w_scale"], state["out"])
        return dict(out=state["out"])
    X.process_logits(state["logits"], state["out"], state["argmax_out"], rows=state["rows"],
                     repetition=state["repetition"], frequency=state["frequency"], presence=state["presence"],
                     history=state["history"], history_offsets=state["history_offsets"],
                     prompt_len=state["prompt_len"], draft=state["draft"], bias_ids=state["bias_ids"],
                     bias_values=state["bias_values"], bias_offsets=state["bias_offsets"], mask=state["mask"],
                     mask_row=state["mask_row"], mask_value=float("-inf"))
    return dict(out=state["out"], argmax=state["argmax_out"])


# -------------------------------------------------------------------- work

def work(case):
    es = {"bf16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "norm":
        n = case["rows"] * case["H"]
        arrays = 2 + (2 if case["residual"] else 0)
        scales = 4 * case["rows"] * -(-case["H"] // BLOCK)
        return dict(bytes=n * es * arrays + case["H"] * es + ((n + scales) if case["q"] else 0), flops=8 * n)
    if case["op"] == "quant":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * (es + 1) + 4 * -(-case["rows"] // BLOCK) * -(-case["cols"] // BLOCK), flops=2 * n)
    if case["op"] == "mm":
        M, N, K = case["M"], case["N"], case["K"]
        KB = -(-K // BLOCK)
        return dict(bytes=(M + N) * K + 4 * KB * (M + -(-N // BLOCK)) + M * N * es, flops=2 * M * N * K)
    n = case["b"] * case["R"]
    states = max(2, int(n * case["masked"])) if case["masked"] > 0 else 0
    side = 3 * case["b"] * case["hist"] + 8 * case["b"] * case["n_bias"] + 4 * states * -(-case["V"] // 32)
    return dict(bytes=2 * n * case["V"] * es + side + 4 * n, flops=4 * n * case["V"])


# ------------------------------------------------------------------- exact

def _amax_scales(m):
    """Scales of groups with the largest magnitudes m (64 bits)."""
    return torch.maximum(m / FP8_MAX, torch.full_like(m, MIN_SCALE))


def _exact_norm(st):
    t = st["x"].double()
    if st["residual"] is not None:
        t = t + st["residual"].double()
    rms = torch.sqrt(t.square().sum(dim=1) / t.shape[1] + EPS)
    y = t * st["weight"].double() / rms[:, None]
    out = dict(y=y)
    if st["residual"] is not None:
        out["sum"] = t
    if st["q_out"] is not None:
        q, scales = torch.empty_like(y), []
        for k in range(0, y.shape[1], BLOCK):
            s = _amax_scales(y[:, k:k + BLOCK].abs().max(dim=1).values)
            q[:, k:k + BLOCK] = y[:, k:k + BLOCK] / s[:, None]       # before its rounding to 8 bits
            scales.append(s)
        out["q"], out["scale"] = q, torch.stack(scales, dim=1)
    return out


def _exact_quant(st):
    W = st["W"]
    rows, cols = W.shape
    q = torch.empty((rows, cols), dtype=torch.float64, device=W.device)
    scale = torch.empty((-(-rows // BLOCK), -(-cols // BLOCK)), dtype=torch.float64, device=W.device)
    for j, k in enumerate(range(0, cols, BLOCK)):
        strip = W[:, k:k + BLOCK].double()
        m = strip.abs().max(dim=1).values
        m = torch.cat([m, m.new_zeros(-rows % BLOCK)]).view(-1, BLOCK).max(dim=1).values
        scale[:, j] = _amax_scales(m)
        q[:, k:k + BLOCK] = strip / scale[:, j].repeat_interleave(BLOCK)[:rows, None]
    return dict(q=q, scale=scale)


def _exact_mm(st):
    a, w, sa, sw = st["a"], st["w"], st["a_scale"].double(), st["w_scale"].double()
    out = torch.zeros((a.shape[0], w.shape[0]), dtype=torch.float64, device=a.device)
    for j, k in enumerate(range(0, a.shape[1], BLOCK)):
        part = a[:, k:k + BLOCK].double() @ w[:, k:k + BLOCK].double().t()
        part *= sa[:, j, None]
        part *= sw[:, j].repeat_interleave(BLOCK)[:w.shape[0]]
        out += part
    return dict(out=out)


def _exact_rules(st):
    logits, R = st["logits"], st["rows"]
    n, V = logits.shape
    out = torch.empty((n, V), dtype=torch.float64, device=logits.device)
    offs, plen = st["history_offsets"].tolist(), st["prompt_len"].tolist()
    boffs = None if st["bias_offsets"] is None else st["bias_offsets"].tolist()
    mrow = None if st["mask_row"] is None else st["mask_row"].tolist()
    bit = torch.arange(V, device=logits.device)
    rep, fre, pre = (st[k].tolist() for k in ("repetition", "frequency", "presence"))
    for i in range(n // R):
        hist = st["history"][offs[i]:offs[i + 1]].long()
        in_prompt = torch.bincount(hist[:plen[i]], minlength=V) > 0
        base = torch.bincount(hist[plen[i]:], minlength=V)
        for j in range(R):
            c = base
            if st["draft"] is not None and j:
                c = base + torch.bincount(st["draft"][i, :j].long(), minlength=V)
            l = logits[i * R + j].double()
            penal = torch.minimum(l / rep[i], l * rep[i])          # the smaller of the two: repetition >= 1
            l = torch.where(in_prompt | (c > 0), penal, l)
            l = l - (fre[i] * c + pre[i] * (c > 0))
            if boffs is not None:
                l.index_add_(0, st["bias_ids"][boffs[i]:boffs[i + 1]].long(),
                             st["bias_values"][boffs[i]:boffs[i + 1]].double())
            if mrow is not None and mrow[i * R + j] >= 0:
                word = st["mask"][mrow[i * R + j]]
                l[(word[bit // 32] >> (bit % 32).to(torch.int32)) & 1 == 0] = float("-inf")
            out[i * R + j] = l
    return dict(out=out, argmax=None)                              # the argmax is one of rounded values


def exact(case, seed):
    st = prepare(case, seed)
    return dict(norm=_exact_norm, quant=_exact_quant, mm=_exact_mm, rules=_exact_rules)[case["op"]](st)
