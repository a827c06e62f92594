"""xpress_sample on the GPU against its definition in 64 bits.

Kept places and tokens are whole numbers: they have to be equal, unless the definition's
own decision is closer to its border than the masses are compared (2^-30 of the row's, by
the entry point's documentation; taken as 2^-28 here).  Such a row may give either side."""
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


def define(l, T, k=0, p=1.0, min_p=0.0, u=0.0):
    """(kept ids, token, near) of one row, from the definition; near: a decision next to its border."""
    l = l.double()
    l = torch.where(l.isnan(), torch.full_like(l, -INF), l)
    ids = torch.nonzero(l > -INF)[:, 0]
    if len(ids) == 0:
        return ids, -1, False
    if float(l.max()) == INF:
        ids = ids[l[ids] == INF]
        l = torch.zeros_like(l)
    v, at = torch.sort(l[ids], descending=True, stable=True)
    ids, near = ids[at], False
    if not T > 0.0:
        return ids[:1], int(ids[0]), False
    w = torch.exp((v - v[0]) / T)
    m = len(ids)
    if k > 0:
        m = min(m, k)
    if min_p > 0.0:
        edge = math.log(min(min_p, 1.0)) * T
        m = min(m, max(1, int((v - v[0] >= edge).sum())))
        near |= bool(((v - v[0] - edge).abs()[v < v[0]] < 1e-12 * (1.0 + v[0].abs() + abs(edge))).any())
    w = w[:m]
    if p < 1.0:
        mass = w.cumsum(0)
        goal = p * mass[-1]
        near |= bool(((mass - goal).abs() < NEAR * mass[-1]).any())
        m = int((mass < goal).sum()) + 1
        m = max(1, min(m, len(w)))
    ids = torch.sort(ids[:m]).values
    w = torch.exp((l[ids] - v[0]) / T)
    mass = w.cumsum(0)
    goal = min(max(u, 0.0), 1.0) * mass[-1]
    j = min(int((mass <= goal).sum()), m - 1)
    near |= bool(((mass[:-1] - goal).abs() < NEAR * mass[-1]).any())
    return ids, int(ids[j]), near


def check(logits, T, u, tokens, out=None, rows=1, k=None, p=None, min_p=None, mask=-INF, most_near=0.02, source=None):
    n, V = logits.shape
    vals = lambda t, off: [off] * (n // rows) if t is None else t.tolist()  # noqa: E731
    Ts, ks, ps, ms = vals(T, 0.0), vals(k, 0), vals(p, 1.0), vals(min_p, 0.0)
    ks = [0 if x <= 0 else x for x in ks]
    us = [0.0] * n if u is None else u.tolist()
    toks = None if tokens is None else tokens.tolist()
    nears = 0
    for i in range(n):
        q = i // rows
        ids, token, near = define(logits[i], Ts[q], ks[q], ps[q], ms[q], us[i])
        nears += near
        if near:
            continue
        if toks is not None:
            assert toks[i] == token, f"row {i}: token {toks[i]}, should be {token}"
        if out is not None:
            want = torch.full((V,), mask, dtype=logits.dtype, device=logits.device)
            want[ids] = logits[i][ids]
            bad = out[i] != want
            assert not bool(bad.any()), f"row {i}: {int(bad.sum())} places of {V} differ, first {int(bad.nonzero()[0])}, kept {len(ids)}"
    assert nears <= max(1, most_near * n)


def run(logits, T, u=None, rows=1, k=None, p=None, min_p=None, want_out=True, mask=-INF, pad=0, most_near=0.02):
    n, V = logits.shape
    dev = logits.device
    col = lambda v, dt: None if v is None else torch.as_tensor(v, dtype=dt, device=dev).expand(n // rows).contiguous()  # noqa: E731
    T, k, p, min_p = col(T, F32), col(k, torch.int32), col(p, F32), col(min_p, F32)
    tokens = None if u is None else torch.full((n,), -7, dtype=torch.int32, device=dev)
    out = torch.full((n, V + pad), 3.0, dtype=logits.dtype, device=dev)[:, :V] if want_out else None
    assert X.sample(logits, T, u=u, tokens_out=tokens, out=out, rows=rows, top_k=k, top_p=p, min_p=min_p, mask_value=mask) == X.XPRESS_OK
    check(logits, T, u, tokens, out, rows, k, p, min_p, mask, most_near)
    if pad and n > 1 and want_out:
        assert bool((out.as_strided((n - 1, pad), (out.stride(0), 1), V) == 3.0).all())
    return tokens, out


def rows_of(n, V, dt, g, sigma=3.0, pad=0, offset=0):
    buf = torch.empty(n * (V + pad) + offset, dtype=dt, device="cuda")
    t = buf[offset:].view(n, V + pad)[:, :V]
    t.normal_(0.0, sigma, generator=g)
    return t


FILTERS = [dict(), dict(k=1), dict(k=7), dict(k=50), dict(k=1000), dict(p=0.9), dict(p=0.3), dict(p=0.999), dict(min_p=0.05),
           dict(k=40, p=0.8), dict(k=2000, p=0.95), dict(k=30, p=0.9, min_p=0.1), dict(p=0.7, min_p=0.02), dict(k=3, min_p=1e-6)]


@pytest.mark.parametrize("f", FILTERS)
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 31, 500, 4097, 32003])
def test_filters(f, dt, V):
    g = _gen(1)
    logits = rows_of(12, V, dt, g)
    run(logits, 0.8, u=torch.rand(12, device="cuda", generator=g), **f)


@pytest.mark.parametrize("f", [dict(), dict(k=50, p=0.9), dict(p=0.9), dict(k=0, p=0.99, min_p=0.01), dict(k=5000, p=0.9)])
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("n, T", [(1, 0.7), (5, 1.0), (40, 1.5)])
def test_large_vocabulary(f, dt, n, T):
    g = _gen(2)
    logits = rows_of(n, 151936, dt, g, 4.0)
    run(logits, T, u=torch.rand(n, device="cuda", generator=g), **f)


@pytest.mark.parametrize("f", [dict(), dict(k=20, p=0.9), dict(p=0.9)])
def test_many_rows(f):
    g = _gen(3)
    logits = rows_of(700, 3001, BF16, g, 2.0)
    run(logits, 1.0, u=torch.rand(700, device="cuda", generator=g), **f)


@pytest.mark.parametrize("dt, V", [(BF16, 1000003), (F32, 500009)])
@pytest.mark.parametrize("f", [dict(), dict(k=50, p=0.9), dict(p=0.95)])
def test_rows_past_shared_memory(dt, V, f):
    g = _gen(4)
    logits = rows_of(2, V, dt, g, 4.0, pad=5)
    tokens, out = run(logits, 0.9, u=torch.rand(2, device="cuda", generator=g), pad=1, **f)
    again = logits.clone()                                       # in place
    col = lambda v, dt: None if v is None else torch.full((2,), v, dtype=dt, device="cuda")  # noqa: E731
    X.sample(again, col(0.9, F32), out=again, top_k=col(f.get("k"), torch.int32), top_p=col(f.get("p"), F32))
    assert torch.equal(again, out)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("pad, offset, opad", [(0, 1, 0), (1, 0, 1), (3, 2, 0), (8, 8, 4), (5, 3, 7)])
def test_rows_that_start_anywhere(dt, pad, offset, opad):
    g = _gen(5)
    for V in (7, 1024, 5003):
        logits = rows_of(9, V, dt, g, 3.0, pad, offset)
        run(logits, 0.9, u=torch.rand(9, device="cuda", generator=g), k=17, p=0.95, pad=opad)
        run(logits, 0.9, u=torch.rand(9, device="cuda", generator=g), pad=opad)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_parameters_per_sequence(dt):
    g = _gen(6)
    b, R, V = 14, 5, 9001
    logits = rows_of(b * R, V, dt, g, 3.0)
    T = 0.3 + torch.rand(b, device="cuda", generator=g) * 1.5
    T[3], T[9] = 0.0, -1.0
    k = torch.randint(-1, 60, (b,), device="cuda", generator=g).to(torch.int32)
    k[5], k[6] = V, V + 10
    p = torch.rand(b, device="cuda", generator=g)
    p[2], p[4], p[7] = 1.0, 2.0, 0.0
    m = torch.rand(b, device="cuda", generator=g) * 0.1
    m[::3] = 0.0
    m[8], m[10] = 1.0, 3.0
    run(logits, T, u=torch.rand(b * R, device="cuda", generator=g), rows=R, k=k, p=p, min_p=m, mask=-8192.0)


def test_off_values():
    """NaN parameters switch a filter off, a NaN temperature is greedy."""
    g = _gen(7)
    nan = float("nan")
    logits = rows_of(4, 3000, F32, g)
    u = torch.rand(4, device="cuda", generator=g)
    T = torch.tensor([1.0, 1.0, 1.0, nan], device="cuda")
    p = torch.tensor([nan, 1.0, 0.5, 0.5], device="cuda")
    m = torch.tensor([nan, nan, nan, 0.1], device="cuda")
    tokens, out = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty_like(logits)
    X.sample(logits, T, u=u, tokens_out=tokens, out=out, top_p=p, min_p=m)
    want = [define(logits[i], *a) for i, a in enumerate([(1.0, 0, 1.0, 0.0, float(u[0])), (1.0, 0, 1.0, 0.0, float(u[1])),
                                                         (1.0, 0, 0.5, 0.0, float(u[2])), (0.0,)])]
    assert tokens.tolist() == [w[1] for w in want]
    assert [int((out[i] > -INF).sum()) for i in range(4)] == [len(w[0]) for w in want]


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("f", [dict(), dict(k=5), dict(p=0.5), dict(k=700, p=0.25), dict(min_p=0.5), dict(k=1000, p=0.001)])
@pytest.mark.parametrize("V", [8, 1024, 20000])
def test_ties(dt, f, V):
    """Equal logits: the first ids are kept; weights of 1 make every mass exact, so that no decision is near."""
    for value in (0.0, -3.5):
        logits = torch.full((4, V), value, dtype=dt, device="cuda")
        logits[1, V // 2:] = -INF
        u = torch.tensor([0.0, 0.5, 0.25, 0.9999999], device="cuda")
        n, tokens = 4, torch.empty(4, dtype=torch.int32, device="cuda")
        out = torch.empty_like(logits)
        col = lambda v, t: None if v is None else torch.full((n,), v, dtype=t, device="cuda")  # noqa: E731
        X.sample(logits, col(0.7, F32), u=u, tokens_out=tokens, out=out, top_k=col(f.get("k"), torch.int32), top_p=col(f.get("p"), F32),
                 min_p=col(f.get("min_p"), F32))
        for i in range(n):
            m = V // 2 if i == 1 else V
            if "k" in f:
                m = min(m, f["k"])
            if "p" in f:
                m = max(1, math.ceil(float(torch.tensor(f["p"], dtype=F32)) * m))
            assert bool((out[i, :m] == value).all()) and bool((out[i, m:] == -INF).all())
            assert int(tokens[i]) == min(m - 1, math.floor(float(u[i]) * m))


def test_signed_zeros_tie():
    for dt in (BF16, F32):
        logits = torch.full((1, 600), -1.0, dtype=dt, device="cuda")
        logits[0, 100:300] = 0.0
        logits[0, 100:300:2] = -0.0
        one = lambda v, t: torch.tensor([v], dtype=t, device="cuda")  # noqa: E731
        out = torch.empty_like(logits)
        X.sample(logits, one(1.0, F32), out=out, top_k=one(31, torch.int32))
        assert (out[0] > -INF).nonzero()[:, 0].tolist() == list(range(100, 131))
        assert torch.equal(out[0, 100:131].view(torch.int16 if dt == BF16 else torch.int32),
                           logits[0, 100:131].view(torch.int16 if dt == BF16 else torch.int32))


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("f", [dict(), dict(k=3), dict(p=0.9), dict(k=20, p=0.9, min_p=0.01)])
def test_masked_rows(dt, f):
    """Rows of which little or nothing is left: -inf, NaN, +inf, the lowest finite value, -8192."""
    g = _gen(9)
    V = 3333
    logits = rows_of(12, V, dt, g)
    low = torch.finfo(dt).min
    logits[0] = -INF                                             # nothing
    logits[1] = float("nan")
    logits[2], logits[2, 77] = -INF, 1.5                         # one place
    logits[3, 5:] = -INF                                         # the first few
    logits[4, ::2] = float("nan")
    logits[5, 40], logits[5, 90], logits[5, 91] = INF, INF, float("nan")
    logits[6] = low
    logits[7], logits[7, 2000:2005] = low, torch.tensor([1.0, 2.0, 3.0, 2.0, 1.0], device="cuda").to(dt)
    logits[8] = -8192.0
    logits[9, 8:] = -8192.0
    logits[10] = -INF
    logits[10, 3330:] = low
    logits[11, 1:] = torch.finfo(dt).max
    run(logits, 0.9, u=torch.rand(12, device="cuda", generator=g), mask=-8192.0, **f)


@pytest.mark.parametrize("T", [1e-30, 1e-3, 50.0, 1e30, INF])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_temperatures(T, dt):
    g = _gen(10)
    logits = rows_of(6, 5000, dt, g)
    u = torch.rand(6, device="cuda", generator=g)
    t = T if T < 1e29 else 1e30                                  # there every weight is 1
    for f in (dict(), dict(k=100), dict(p=0.5), dict(min_p=0.9)):
        n, tokens, out = 6, torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty_like(logits)
        col = lambda v, d: None if v is None else torch.full((n,), v, dtype=d, device="cuda")  # noqa: E731
        X.sample(logits, col(T, F32), u=u, tokens_out=tokens, out=out, top_k=col(f.get("k"), torch.int32), top_p=col(f.get("p"), F32),
                 min_p=col(f.get("min_p"), F32))
        check(logits, col(t, F32), u, tokens, out, 1, col(f.get("k"), torch.int32), col(f.get("p"), F32), col(f.get("min_p"), F32),
              most_near=1.0 if T > 1e29 else 0.02)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_wide_ranges(dt):
    """Values of all magnitudes and both signs: every level of the histogram."""
    g = _gen(11)
    V = 40000
    x = torch.randn((8, V), device="cuda", generator=g)
    mag = torch.exp(40.0 * torch.rand((8, V), device="cuda", generator=g) - 38.0)
    logits = (x.sign() * mag).to(dt)
    for f in (dict(k=25000), dict(k=3, p=0.99), dict(k=20000, p=0.5), dict(p=0.6), dict(p=0.05)):
        run(logits, 2.0, u=torch.rand(8, device="cuda", generator=g), **f)


def test_only_tokens_or_only_rows():
    g = _gen(12)
    logits = rows_of(20, 7001, BF16, g)
    u = torch.rand(20, device="cuda", generator=g)
    a, out = run(logits, 1.0, u=u, k=40, p=0.9)
    b, _ = run(logits, 1.0, u=u, k=40, p=0.9, want_out=False)
    _, c = run(logits, 1.0, k=40, p=0.9)
    assert torch.equal(a, b) and torch.equal(out, c)
    d = logits.clone()
    X.sample(d, torch.ones(20, device="cuda"), out=d, top_k=torch.full((20,), 40, dtype=torch.int32, device="cuda"),
             top_p=torch.full((20,), 0.9, device="cuda"))
    assert torch.equal(out, d)                                   # in place


def test_numbers_outside_the_unit_interval():
    g = _gen(13)
    logits = rows_of(5, 500, F32, g)
    u = torch.tensor([-1.0, 1.0, 7.0, float("nan"), 0.0], device="cuda")
    tokens = torch.empty(5, dtype=torch.int32, device="cuda")
    X.sample(logits, torch.ones(5, device="cuda"), u=u, tokens_out=tokens)
    assert [int(tokens[i]) for i in (0, 3, 4)] == [0, 0, 0] and [int(tokens[i]) for i in (1, 2)] == [499, 499]


def test_draws_follow_the_distribution():
    """One row, 200000 equally spaced numbers: every id is drawn in proportion to its mass, to one draw at each end."""
    g = _gen(14)
    n = 200000
    row = rows_of(1, 40, F32, g, 1.0)
    logits = row.expand(n, 40).contiguous()
    u = ((torch.arange(n, device="cuda") + 0.5) / n).float()
    tokens = torch.empty(n, dtype=torch.int32, device="cuda")
    X.sample(logits, torch.ones(n, device="cuda"), u=u, tokens_out=tokens)
    want = torch.softmax(row[0].double(), 0) * n
    assert bool(((torch.bincount(tokens.long(), minlength=40).double() - want).abs() <= 2.0).all())


def test_calls_repeat_and_run_on_other_streams_and_in_graphs():
    g = _gen(15)
    logits = rows_of(30, 30011, F32, g, 2.0)
    T, p = torch.full((30,), 1.3, device="cuda"), torch.full((30,), 0.9, device="cuda")
    u = torch.rand(30, device="cuda", generator=g)
    first, out = run(logits, T, u=u, p=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tokens, again = torch.empty_like(first), torch.empty_like(out)
    for _ in range(4):
        X.sample(logits, T, u=u, tokens_out=tokens, out=again, top_p=p, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(tokens, first) and torch.equal(again, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X.sample(logits, T, u=u, tokens_out=tokens, out=again, top_p=p)
    logits.normal_(0.0, 2.0, generator=g)
    u.uniform_(0.0, 1.0, generator=g)
    graph.replay()
    torch.cuda.synchronize()
    check(logits, T, u, tokens, again, p=p)


def test_rules_then_draw():
    """The request's rules in front: process_logits' masked rows are what the draw reads."""
    g = _gen(16)
    V, n = 5000, 6
    logits = rows_of(n, V, BF16, g)
    hist = torch.randint(0, V, (300,), device="cuda", generator=g).to(torch.int32)
    off = (torch.arange(n + 1, device="cuda") * 50).to(torch.int64)
    ruled = torch.empty_like(logits)
    X.process_logits(logits, ruled, repetition=torch.full((n,), 1.3, device="cuda"), history=hist, history_offsets=off)
    run(ruled, 0.8, u=torch.rand(n, device="cuda", generator=g), k=50, p=0.9, mask=-8192.0)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("f", [dict(), dict(p=0.9), dict(k=9000, p=0.7), dict(k=100), dict(min_p=0.98), dict(k=1025), dict(k=1024, p=0.5)])
@pytest.mark.parametrize("V", [20000, 151936])
def test_flat_rows(dt, f, V):
    """Logits next to one another: thousands are kept, in bf16 most of them equal."""
    g = _gen(17)
    logits = rows_of(3, V, dt, g, 0.02)
    run(logits, 1.1, u=torch.rand(3, device="cuda", generator=g), **f)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("p", [1e-30, 1e-7, 0.5, 0.9999, 1.0 - 2.0 ** -24])
@pytest.mark.parametrize("k", [None, 300, 2500])
def test_extreme_top_p(dt, p, k):
    g = _gen(18)
    logits = rows_of(4, 5000, dt, g)
    # at the last p the tail's masses are below what is told apart: such rows are near
    run(logits, 1.0, u=torch.rand(4, device="cuda", generator=g), p=p, k=k, most_near=1.0 if p > 0.99 else 0.02)


@pytest.mark.parametrize("sizes", [(1, 1), (1024, 1024), (1025, 700), (3000, 1), (3000, 2999)])
def test_ties_at_the_limit_of_the_few(sizes):
    """As many equal maxima as are settled at once, one more, and many; k of them are kept."""
    ties, k = sizes
    for dt in (BF16, F32):
        logits = torch.full((2, 20000), -2.0, dtype=dt, device="cuda")
        logits[:, 3:3 + 5 * ties:5] = 4.0
        tokens, out = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty_like(logits)
        one = lambda v, t: torch.full((2,), v, dtype=t, device="cuda")  # noqa: E731
        X.sample(logits, one(0.01, F32), u=torch.tensor([0.0, 0.999], device="cuda"), tokens_out=tokens, out=out, top_k=one(k, torch.int32))
        kept = list(range(3, 3 + 5 * k, 5))
        assert all((out[i] > -INF).nonzero()[:, 0].tolist() == kept for i in range(2))
        assert tokens.tolist() == [kept[0], kept[int(0.999 * k)]]
        X.sample(logits, one(0.0, F32), u=one(0.7, F32), tokens_out=tokens, out=out)          # greedy: the first of them
        assert tokens.tolist() == [3, 3] and all((out[i] > -INF).nonzero()[:, 0].tolist() == [3] for i in range(2))


def test_two_calls_at_once():
    g = _gen(19)
    a, b = rows_of(300, 20011, BF16, g), rows_of(200, 9001, F32, g)
    ua, ub = torch.rand(300, device="cuda", generator=g), torch.rand(200, device="cuda", generator=g)
    Ta, Tb = torch.full((300,), 0.9, device="cuda"), torch.full((200,), 1.2, device="cuda")
    pa, kb = torch.full((300,), 0.9, device="cuda"), torch.full((200,), 30, dtype=torch.int32, device="cuda")
    ta, tb = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (300, 200))
    oa, ob = torch.empty_like(a), torch.empty_like(b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        X.sample(a, Ta, u=ua, tokens_out=ta, out=oa, top_p=pa, stream=s1)
        X.sample(b, Tb, u=ub, tokens_out=tb, out=ob, top_k=kb, stream=s2)
    torch.cuda.synchronize()
    check(a, Ta, ua, ta, oa, p=pa)
    check(b, Tb, ub, tb, ob, k=kb)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("order", ["mixed", "falling", "rising", "one of 64"])
@pytest.mark.parametrize("k", [2, 16, 127, 128, 129, 400, 511, 513])
def test_few_elements_wherever_they_are(dt, order, k):
    """The largest spread over the row, all in its first or last part, or a few to each part."""
    g = _gen(20)
    V = 40003
    logits = rows_of(4, V, torch.float32, g)
    if order != "mixed":
        logits = torch.sort(logits, dim=1, descending=order != "rising").values
    if order == "one of 64":
        V = 40000
        logits = logits[:, :V].reshape(4, V // 64, 64).transpose(1, 2).reshape(4, V)
    logits = logits.to(dt).contiguous()
    u = torch.rand(4, device="cuda", generator=g)
    run(logits, 0.9, u=u, k=k)
    run(logits, 0.9, u=u, k=k, p=0.8)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("f", [dict(), dict(p=0.9), dict(k=300), dict(k=3000, p=0.99)])
@pytest.mark.parametrize("kept", [1, 2, 127, 128, 129, 1023, 1024, 1025, 9000])
def test_min_p_keeps_so_many(dt, f, kept):
    """min-p alone, or before the other filters, leaves a given number."""
    g = _gen(21)
    V, n = 30011, 4
    logits = torch.full((n, V), -20.0, device="cuda")
    for i in range(n):
        at = torch.randperm(V, device="cuda", generator=g)[:kept]
        logits[i, at] = torch.rand(kept, device="cuda", generator=g) * 2.0
    logits = logits.to(dt)
    u = torch.rand(n, device="cuda", generator=g)
    run(logits, 1.0, u=u, min_p=0.1, **f)
    run(logits, 1.0, u=u, min_p=0.1, want_out=False, **f)
