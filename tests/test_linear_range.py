"""linear's activation as a Python integer that is no C int (no GPU: the check comes first)."""
import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("act", [-(1 << 32), -(1 << 32) + 1, -(1 << 31) - 1, 1 << 31, 1 << 32])
def test_activation_outside_an_int(act):
    BLD.build()
    x, w, out = (torch.zeros(s, dtype=torch.bfloat16) for s in ((2, 16), (5, 16), (2, 5)))
    with pytest.raises(ValueError, match="act"):
        X.linear(x, w, out, act=act)
