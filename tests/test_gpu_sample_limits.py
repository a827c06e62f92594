"""xpress_sample where its definition is at a limit: rows with infinities under every filter,
and min_p above 1.

The definition is followed as the entry point states it, in 64 bits.  Masses: by its
documentation they are compared to about 2^-30 of the row's, taken as 2^-28 here; a kept
prefix or a token may lie that far from its border and no farther."""
import math

import pytest
import torch

from paper_2608_02438_gb300 import binding as X

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")
NEAR = 2.0 ** -28


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2608_02438_gb300 import build as BLD
    BLD.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def draw(logits, T, u, k=None, p=None, min_p=None, out=True):
    """Tokens and truncated rows (mask -inf) of logits [n, V], one value of each parameter for all rows."""
    n = logits.shape[0]
    col = lambda v, dt: None if v is None else torch.full((n,), v, dtype=dt, device="cuda")  # noqa: E731
    tokens = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    rows = torch.empty_like(logits) if out else None
    X.sample(logits, col(T, F32), u=u, tokens_out=tokens, out=rows, top_k=col(k, torch.int32), top_p=col(p, F32), min_p=col(min_p, F32))
    return tokens, rows


def verify(l, T, u, token, row=None, k=None, p=None, min_p=None):
    """One row's result against the definition, masses to NEAR of the row's.  Without the
    truncated row only where k, p and min_p leave no choice."""
    l = l.double()
    l = torch.where(l.isnan(), torch.full_like(l, -INF), l)
    v, order = torch.sort(l, descending=True, stable=True)
    order, v = order[v > -INF], v[v > -INF]
    if v[0] == INF:
        w = (v == INF).double()
    else:
        w = torch.exp((v - v[0]) / T)
    m = int((w > 0).sum()) if v[0] == INF else len(w)
    if min_p is not None and min_p > 0.0:
        m = min(m, max(1, int((w >= min_p).sum())))
    if k is not None and k > 0:
        m = min(m, k)
    w = w[:m]
    kept = m
    if row is not None:
        ids = torch.nonzero(row > -INF)[:, 0]
        kept = len(ids)
        assert 1 <= kept <= m and torch.equal(torch.sort(order[:kept]).values, ids), f"{kept} kept, not the first of the order"
        assert torch.equal(row[ids].double(), l[ids])
        if p is not None and p < 1.0:
            mass = w.cumsum(0)
            goal = float(torch.tensor(p, dtype=F32)) * mass[-1]
            assert kept == 1 or mass[kept - 2] < goal + NEAR * mass[-1], f"{kept} kept: too many"
            assert kept == m or mass[kept - 1] >= goal - NEAR * mass[-1], f"{kept} kept: too few"
        else:
            assert kept == m
    else:
        assert p is None or p >= 1.0
    ids, at = torch.sort(order[:kept])
    mass = w[:kept][at].cumsum(0)
    j = int(torch.searchsorted(ids, torch.tensor(token, device=ids.device)))
    assert j < kept and int(ids[j]) == token, f"token {token} is not kept"
    goal = float(torch.tensor(u, dtype=F32)) * mass[-1]
    assert mass[j] > goal - NEAR * mass[-1], f"token {token} is before its place"
    assert j == 0 or mass[j - 1] <= goal + NEAR * mass[-1], f"token {token} is behind its place"


def verify_all(logits, T, us, k=None, p=None, min_p=None):
    u = torch.tensor(us, dtype=F32, device="cuda")
    tokens, rows = draw(logits, T, u, k, p, min_p)
    for i in range(len(us)):
        verify(logits[i], T, us[i], int(tokens[i]), rows[i], k, p, min_p)
    only, _ = draw(logits, T, u, k, p, min_p, out=False)
    assert torch.equal(only, tokens)
    return tokens, rows


# ------------------------------------------------------------- infinities

@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("infs", [1, 2, 5, 128, 1024, 1500])
@pytest.mark.parametrize("f", [dict(), dict(k=1), dict(k=2), dict(k=1100), dict(p=0.5), dict(p=0.3), dict(p=1e-9), dict(p=0.999),
                               dict(k=4, p=0.7), dict(k=2000, p=0.4, min_p=0.5), dict(min_p=0.9), dict(k=3, min_p=2.0)])
def test_infinities_share_under_the_filters(dt, infs, f):
    """+inf logits have equal masses, all of it: the first top_k of them, and of these what top-p keeps."""
    g = _gen(31)
    V, n = 20011, 4
    logits = torch.empty((n, V), dtype=dt, device="cuda").normal_(0.0, 3.0, generator=g)
    for i in range(n):
        at = torch.randperm(V, device="cuda", generator=g)[:infs]
        logits[i, at] = INF
        logits[i, (at[0] + 1) % V] = float("nan") if i == 2 else logits[i, (at[0] + 1) % V]
    tokens, rows = verify_all(logits, 0.8, [0.0, 0.4, 0.75, 0.9999], **f)
    for i in range(n):                                            # whole numbers: no mass is next to a border
        m = int((logits[i] == INF).sum())
        m = min(m, f.get("k", m))
        if f.get("min_p", 0.0) > 1.0:
            m = 1
        if "p" in f:
            m = max(1, math.ceil(float(torch.tensor(f["p"], dtype=F32)) * m))
        assert int((rows[i] > -INF).sum()) == m


@pytest.mark.parametrize("dt, V", [(BF16, 1000003), (F32, 500009)])
def test_infinities_in_rows_past_shared_memory(dt, V):
    logits = torch.zeros((2, V), dtype=dt, device="cuda")
    logits[:, 7::1000] = INF
    for f in (dict(k=3), dict(p=0.5), dict(k=300, p=0.25)):
        verify_all(logits, 1.0, [0.1, 0.9], **f)


# ------------------------------------------------------------- min_p above 1

@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("ties", [1, 2, 300, 3000])
@pytest.mark.parametrize("min_p", [1.0, 1.0000001, 3.0, INF])
def test_min_p_above_one_keeps_the_first(dt, ties, min_p):
    """No weight reaches it; the first of the order is always kept.  At 1 all maxima are."""
    logits = torch.full((2, 20000), -1.0, dtype=dt, device="cuda")
    logits[:, 4:4 + 3 * ties:3] = 2.5
    for f in (dict(), dict(k=2), dict(p=0.9)):
        tokens, rows = draw(logits, 0.7, torch.tensor([0.0, 0.99], device="cuda"), min_p=min_p, **f)
        m = ties if min_p == 1.0 else 1
        m = min(m, f.get("k", m))
        if "p" in f:
            m = math.ceil(float(torch.tensor(f["p"], dtype=F32)) * m)
        for i, u in enumerate((0.0, 0.99)):
            assert torch.nonzero(rows[i] > -INF)[:, 0].tolist() == list(range(4, 4 + 3 * m, 3))
            assert int(tokens[i]) == 4 + 3 * math.floor(float(torch.tensor(u, dtype=F32)) * m)
