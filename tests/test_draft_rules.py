"""The grammar tables of draft_head.Rules, without a GPU: a mask and the table of
the rows that it is used on go together, and what does not fit is refused before
anything is allocated or launched."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")
from paper_2608_02438_gb300 import draft_head as D  # noqa: E402

MASK, ROWS = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)


class _Head(D.DraftHead):
    """Without a refiner's device: nothing past the checks can be reached."""

    def __init__(self):
        self.refiner = SimpleNamespace(B=2, H=8, V=64)


BASE = [dict(mask=MASK), dict(mask=MASK, target_mask_row=ROWS), dict(base_mask_row=ROWS)]
TARGET = [dict(mask=MASK), dict(mask=MASK, base_mask_row=ROWS), dict(target_mask_row=ROWS)]


@pytest.mark.parametrize("kw", BASE)
def test_base_rows_without_their_states(kw):
    with pytest.raises(ValueError, match="base_mask_row"):
        _Head().base_logits(torch.zeros((2, 2, 8), dtype=torch.bfloat16), None, D.Rules(**kw))


@pytest.mark.parametrize("kw", TARGET)
def test_target_rows_without_their_states(kw):
    with pytest.raises(ValueError, match="target_mask_row"):
        _Head().target_logits(torch.zeros((2, 3, 64), dtype=torch.bfloat16), ROWS.view(2, 2), D.Rules(**kw))


@pytest.mark.parametrize("kw", BASE + TARGET[1:])
def test_round_without_either(kw):
    with pytest.raises(ValueError, match="mask_row"):
        _Head().round(torch.zeros((2, 2, 8), dtype=torch.bfloat16), None, None, None, None, None, 0, 1, D.Rules(**kw))


def test_tables_that_fit():
    assert D.Rules().rows("base_mask_row") is None and D.Rules().rows("target_mask_row") is None
    r = D.Rules(mask=MASK, base_mask_row=ROWS, target_mask_row=ROWS)
    assert r.rows("base_mask_row") is ROWS and r.rows("target_mask_row") is ROWS
    # one side is enough for the calls of that side
    assert D.Rules(mask=MASK, base_mask_row=ROWS).rows("base_mask_row") is ROWS
