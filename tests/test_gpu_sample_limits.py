"""xpress_sample where its definition is at a limit: rows with infinities under every filter,
min_p above 1, and rows of which a large flat tail holds little of the mass.

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


# ------------------------------------------------------------- flat tails

def tail(V, dt, value, at, spread=0.0, top=0.0, n=4, seed=32):
    """Rows of one likely token and a tail around `value` below it."""
    logits = torch.full((n, V), top + value, device="cuda")
    if spread:
        logits += spread * torch.randn((n, V), device="cuda", generator=_gen(seed))
    logits[:, at] = top
    return logits.to(dt)


# weights below and around half of 2^-(61 - ceil(log2 V)), which all V may sum to
TAILS = [(1 << 24, BF16, -27.0), (1 << 24, BF16, -25.0), (1 << 23, F32, -27.3), (1000003, BF16, -29.25), (700001, BF16, -28.5), (300007, F32, -29.0)]


@pytest.mark.parametrize("V, dt, value", TAILS)
@pytest.mark.parametrize("spread", [0.0, 0.5])
def test_tokens_of_a_flat_tail(V, dt, value, spread):
    """The likely token last: small numbers draw from the tail, at its masses."""
    logits = tail(V, dt, value, V - 1, spread)
    share = float(torch.exp(logits[0, :-1].double()).sum())
    verify_all(logits, 1.0, [share * 0.1, share * 0.5, share * 0.9, 0.5])


@pytest.mark.parametrize("V, dt, value", TAILS[:4])
@pytest.mark.parametrize("spread", [0.0, 0.5])
def test_top_p_inside_a_flat_tail(V, dt, value, spread):
    logits = tail(V, dt, value, 11, spread)
    share = float(torch.exp(logits[0].double()).sum()) - 1.0
    p = 1.0 - share * 0.4                                         # in steps of 2^-24
    verify_all(logits, 1.0, [0.0, 0.5, 0.9999, 1.0 - 2.0 ** -24], p=p)


@pytest.mark.parametrize("f", [dict(min_p=1e-13), dict(k=1 << 23), dict(k=1 << 23, p=0.99999), dict(min_p=1e-13, p=0.99999)])
@pytest.mark.parametrize("spread", [0.0, 0.25])
def test_filters_that_leave_a_flat_tail(f, spread):
    V = 1 << 24
    logits = tail(V, BF16, -27.0, V - 1, spread)
    share = float(torch.exp(logits[0, :-1].double()).sum())
    verify_all(logits, 1.0, [share * 0.01, share * 0.1, share * 0.3, 0.5], **f)


@pytest.mark.parametrize("top, T, value", [(1e6, 1.0, -27.0), (0.0, 1e29, -27e29), (-1e6, 0.5, -13.5)])
@pytest.mark.parametrize("f", [dict(), dict(p=0.99999), dict(k=5_000_000)])
def test_flat_tails_of_large_and_far_logits(top, T, value, f):
    """Logits far from 0, where the exponent's parts take more than a float's bits, and a huge temperature."""
    V = 1 << 23
    logits = tail(V, F32, value, V - 1, 0.0, top)
    share = (V - 1) * math.exp(-27.0)
    verify_all(logits, T, [share * 0.1, share * 0.5, 0.5, 0.99], **f)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("many", [2, 1000, 70000])
def test_several_likely_tokens_and_a_tail(dt, many):
    V = 1 << 22
    logits = tail(V, dt, -26.0, V - 1, 0.3)
    logits[:, V - many:] = 0.0
    share = float(torch.exp(logits[0, :V - many].double()).sum()) / many
    for f in (dict(), dict(p=0.9), dict(p=1.0 - 2.0 ** -20), dict(k=V // 2)):
        verify_all(logits, 1.0, [share * 0.2, share * 0.8, 0.3, 0.95], **f)
