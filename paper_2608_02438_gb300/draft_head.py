"""The drafter's head in 8 bits around a refiner: one speculative round.

What a serving loop runs between the drafter's last layer and the emitted
tokens (Sec. 3.1, Fig. 2a of the paper around the refinement of Sec. 4.2):

    x      = x + W2 act(W1 norm(x) + b1) + b2   xpress_linear, twice (a head with a feed-forward block)
    h, q   = norm(x + residual)              xpress_rmsnorm (bf16 for the refiner, e4m3 for the head)
    s      = q W_lm^T                        xpress_matmul_fp8 (weights quantised once)
    s, Y0  = the request's rules on s        xpress_process_logits
    Y      = the refined block               xpress_refine_block
    target = the rules on the target's rows  xpress_process_logits (row j counts Y_1 .. Y_j)
    target = what top-k, top-p, min-p keep   xpress_sample (requests with filters)
    tokens = accepted prefix + correction    xpress_accept

Example (``refiner`` a :class:`binding.Refiner`, tensors on its device)::

    head = DraftHead(refiner, norm_weight, W_lm)
    rules = Rules(repetition=rep, history=tokens, history_offsets=offsets, prompt_len=plen)
    out = head.round(x, residual, target, anchor, temperature, seed, offset, K_max, rules)
    out["out_tokens"], out["accept_len"]

The token before the first round comes from ``head.next_tokens``, with the same rules
and filters.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as X

# A masked logit for the refinement and the acceptance: finite, so that a row
# whose mask allows nothing still has a softmax; far below every logit; and not
# so large that the rounding of l / T, which their exponentials carry, grows past
# 1 (at -1e30 a group of masked ids would win every draw).  Exact in bf16.
MASKED = -8192.0


@dataclass
class Rules:
    """The sampling rules of b requests (tensors as binding.process_logits takes
    them; None: the rule is off).  mask holds the grammar states' bit rows;
    base_mask_row [b * B] and target_mask_row [b * (B + 1)] name a row's state,
    -1 for a row that is not masked.  A mask needs the table of the rows that it is
    to be used on (ValueError without: nothing else tells a row's state).

    What a round emits is allowed by its target row's state, unless that state allows
    nothing: such a row is MASKED throughout and some forbidden token comes out of it
    (id 0 at temperature 0).  End the request instead of asking for that row."""
    repetition: torch.Tensor | None = None
    frequency: torch.Tensor | None = None
    presence: torch.Tensor | None = None
    history: torch.Tensor | None = None
    history_offsets: torch.Tensor | None = None
    prompt_len: torch.Tensor | None = None
    bias_ids: torch.Tensor | None = None
    bias_values: torch.Tensor | None = None
    bias_offsets: torch.Tensor | None = None
    mask: torch.Tensor | None = None
    base_mask_row: torch.Tensor | None = None
    target_mask_row: torch.Tensor | None = None

    def common(self) -> dict:
        return {k: v for k, v in vars(self).items() if not k.endswith("mask_row")}

    def rows(self, table: str) -> torch.Tensor | None:
        """The state table `table` of a grammar; None without a grammar."""
        rows = getattr(self, table)
        if (self.mask is None) != (rows is None):
            raise ValueError(f"Rules: mask and {table} go together (-1 in {table} leaves a row unmasked)")
        return rows


@dataclass
class Filters:
    """The sampling filters of b requests, each a tensor [b] as binding.sample takes it
    (None: off).  The target's distribution that the acceptance keeps is then the
    truncated one, renormalised, at the request's temperature; the drafts' is as
    before, so that only the accepted lengths depend on it.  Removed logits are MASKED,
    which has no mass at temperatures below 80 (e^-100)."""
    top_k: torch.Tensor | None = None
    top_p: torch.Tensor | None = None
    min_p: torch.Tensor | None = None

    def any(self) -> bool:
        return any(v is not None for v in vars(self).values())


def _padded(rows: int, cols: int, device) -> torch.Tensor:
    """An uninitialised bf16 [rows, cols] whose rows start on 16 bytes."""
    return torch.empty((rows, (cols + 7) // 8 * 8), dtype=torch.bfloat16, device=device)[:, :cols]


def _rows_on_16_bytes(w: torch.Tensor) -> torch.Tensor:
    """w, or where a row of it starts elsewhere, a copy with padded rows."""
    if w.dtype != torch.bfloat16 or w.dim() != 2:
        return w
    rows, cols = w.shape
    if w.data_ptr() % 16 == 0 and w.stride(0) % 8 == 0 and w.stride(0) >= cols and w.stride(1) == 1:
        return w
    return _padded(rows, cols, w.device).copy_(w.detach())


@dataclass
class FeedForward:
    """A block in front of the head, x + W2 act(W1 norm(x) + b1) + b2: norm_weight [H],
    W1 [I, H], W2 [H, I], b1 [I] and b2 [H] (None: no bias), bf16; act an XPRESS_ACT_*.
    Any I: weights whose rows do not all start on 16 bytes, as binding.linear wants
    them, are copied once, here, on torch's current stream."""
    norm_weight: torch.Tensor
    W1: torch.Tensor
    W2: torch.Tensor
    b1: torch.Tensor | None = None
    b2: torch.Tensor | None = None
    act: int = X.XPRESS_ACT_SILU

    def __post_init__(self):
        self.W1, self.W2 = _rows_on_16_bytes(self.W1), _rows_on_16_bytes(self.W2)

    def __call__(self, x, residual, eps: float):
        """x, residual [n, H] (residual may be None) -> the block's output [n, H]."""
        n, dev = x.shape[0], x.device
        total = torch.empty_like(x, memory_format=torch.contiguous_format) if residual is not None else x
        normed = torch.empty((n, x.shape[1]), dtype=torch.bfloat16, device=dev)
        inner = _padded(n, self.W1.shape[0], dev)
        out = torch.empty_like(normed)
        X.rmsnorm(x, self.norm_weight, eps, residual=residual, sum_out=total if residual is not None else None, y_out=normed)
        X.linear(normed, self.W1, inner, bias=self.b1, act=self.act)
        X.linear(inner, self.W2, out, bias=self.b2, residual=total)
        return out


class DraftHead:
    """A bf16 refiner's drafter head: the final norm's weight [H] and the LM head
    W_lm [V, H], quantised here once (W_lm is not kept).  The weights are quantised on
    the refiner's stream, after what torch's current stream has done so far, and both
    streams' next calls find them ready."""

    def __init__(self, refiner: X.Refiner, norm_weight: torch.Tensor, W_lm: torch.Tensor, eps: float = 1e-6,
                 block: FeedForward | None = None):
        if refiner.dtype != X.XPRESS_BF16:
            raise ValueError("the 8-bit head serves bf16 refiners")
        if tuple(W_lm.shape) != (refiner.V, refiner.H):
            raise ValueError(f"W_lm: expected [{refiner.V}, {refiner.H}], got {list(W_lm.shape)}")
        if block is not None and (tuple(block.W1.shape) != (block.W2.shape[1], refiner.H) or block.W2.shape[0] != refiner.H):
            raise ValueError(f"block: expected W1 [I, {refiner.H}] and W2 [{refiner.H}, I], got {list(block.W1.shape)} and "
                             f"{list(block.W2.shape)}")
        self.refiner, self.norm_weight, self.eps, self.block = refiner, norm_weight, eps, block
        here = torch.cuda.current_stream(W_lm.device)
        refiner.stream.wait_stream(here)
        self.w, self.w_scale = X.quantize_weight(W_lm, stream=refiner.stream)
        here.wait_stream(refiner.stream)
        if block is not None:
            for t in (block.W1, block.W2):               # (copies may be this stream's memory)
                t.record_stream(refiner.stream)

    def base_logits(self, x, residual=None, rules: Rules | None = None) -> dict:
        """x [b, B, H] (the drafter's last layer, before its final norm) -> h
        [b, B, H], s [b, B, V] under the rules, their first maxima draft [b, B]
        (0 where a mask allows nothing), and the residual stream sum (with a block,
        what comes out of it)."""
        R, rules = self.refiner, rules or Rules()
        mask_row = rules.rows("base_mask_row")
        b = x.shape[0]
        n, dev = b * R.B, x.device
        h = torch.empty((n, R.H), dtype=torch.bfloat16, device=dev)
        x, residual = x.reshape(n, R.H), None if residual is None else residual.reshape(n, R.H)
        total = torch.empty_like(h) if residual is not None else None
        if self.block is not None:
            x = after = self.block(x, residual, self.eps)
            total = residual = None
        q = X.alloc_e4m3(n, R.H, dev)
        scale = torch.empty((n, (R.H + 127) // 128), dtype=torch.float32, device=dev)
        s = torch.empty((n, R.V), dtype=torch.bfloat16, device=dev)
        draft = torch.empty(n, dtype=torch.int32, device=dev)
        X.rmsnorm(x, self.norm_weight, self.eps, residual=residual, sum_out=total, y_out=h, q_out=q, scale_out=scale)
        X.matmul_fp8(q, scale, self.w, self.w_scale, s)
        X.process_logits(s, s, draft, rows=R.B, mask_row=mask_row, mask_value=MASKED, **rules.common())
        if self.block is not None:
            total = after
        return dict(h=h.view(b, R.B, R.H), s=s.view(b, R.B, R.V), draft=draft.clamp_(min=0).view(b, R.B),
                    sum=None if total is None else total.view(b, R.B, R.H))

    def target_logits(self, target, tokens, rules: Rules | None = None, filters: Filters | None = None, temperature=None):
        """The rules on the target's rows [b, B + 1, V] of the blocks `tokens`
        [b, B]: row j counts the block's tokens before it as answered.  With filters
        (and the requests' temperature [b]) the rows are truncated by them."""
        R, rules = self.refiner, rules or Rules()
        mask_row = rules.rows("target_mask_row")
        if filters is not None and filters.any() and temperature is None:
            raise ValueError("filters need the requests' temperature")
        out = torch.empty_like(target)
        n = target.shape[0] * (R.B + 1)
        X.process_logits(target.view(n, R.V), out.view(n, R.V), rows=R.B + 1, draft=tokens,
                         mask_row=mask_row, mask_value=MASKED, **rules.common())
        if filters is not None and filters.any():
            rows = out.view(n, R.V)
            X.sample(rows, temperature, out=rows, rows=R.B + 1, mask_value=MASKED, **vars(filters))
        return out

    def next_tokens(self, logits, temperature, u, rules: Rules | None = None, filters: Filters | None = None, mask_row=None):
        """The next token of each of b requests from the target's logits [b, V] (the
        prompt's last position, say) under the rules and filters, drawn with the
        numbers u [b] in [0, 1): int32 [b].  A grammar (rules.mask) needs the rows'
        states mask_row [b]; a state that allows nothing gives -1."""
        rules = rules or Rules()
        if (rules.mask is None) != (mask_row is None):
            raise ValueError("Rules.mask and mask_row go together (-1 in mask_row leaves a row unmasked)")
        out = torch.empty_like(logits)
        tokens = torch.empty(logits.shape[0], dtype=torch.int32, device=logits.device)
        X.process_logits(logits, out, mask_row=mask_row, **rules.common())            # -inf: never drawn, at any temperature
        X.sample(out, temperature, u=u, tokens_out=tokens, **vars(filters or Filters()))
        return tokens

    def round(self, x, residual, target, anchor, temperature, seed, offset: int, K_max: int,
              rules: Rules | None = None, filters: Filters | None = None) -> dict:
        """One round on torch's current stream, which has to be the refiner's:
        base logits, refinement and acceptance against target [b, B + 1, V]."""
        R, rules = self.refiner, rules or Rules()
        for table in ("base_mask_row", "target_mask_row"):         # before anything is launched
            rules.rows(table)
        if torch.cuda.current_stream(x.device).cuda_stream != R.stream.cuda_stream:
            raise ValueError("call round() on the refiner's stream")
        base = self.base_logits(x, residual, rules)
        out = R.refine_block(base["h"], base["s"], base["draft"], anchor, temperature, seed, offset, K_max)
        tgt = self.target_logits(target, out["tokens"], rules, filters, temperature)
        acc = R.accept(tgt, base["s"], out["tokens"], out["lse"], out["logit_sel"], out["z_final"], temperature, seed,
                       offset)
        return {**base, **out, **acc, "target": tgt}
