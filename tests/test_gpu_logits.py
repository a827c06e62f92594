"""GPU tests of xpress_process_logits against its definition, written out row
by row on the CPU.

The rules are at most six operations, each rounded on its own in fp32: against
64 bits |l - l64| <= 6 2^-24 (|l| max(rep, 1 / rep) + freq c + pres + |bias|),
plus half an ulp of the storage type; against the same operations in numpy's
fp32 the stored values are equal.  The argmax is the first maximum of the
stored row over the allowed ids, exactly.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
f4 = np.float32


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02438_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def _case(b, R, V, hist, n_bias, seed, draft=True, masked=0.5):
    """Host-side rules of b sequences (numpy); hist: history lengths."""
    rng = np.random.Generator(np.random.PCG64(seed))
    c = dict(b=b, R=R, V=V, rep=rng.uniform(0.7, 1.6, b).astype(f4), freq=rng.uniform(-0.5, 1, b).astype(f4),
             pres=rng.uniform(-0.5, 1, b).astype(f4))
    ids = lambda n: np.minimum((V * rng.random(n) ** 3).astype(np.int32), V - 1)  # noqa: E731
    c["hist"] = [ids(n) for n in hist]
    c["plen"] = np.array([rng.integers(0, n + 1) for n in hist], np.int32)
    c["draft"] = ids((b, R + 1)) if draft else None
    c["bias"] = [(rng.choice(V, min(n_bias, V), replace=False).astype(np.int32),
                  rng.normal(0, 3, min(n_bias, V)).astype(f4)) for _ in range(b)] if n_bias else None
    c["mask"] = c["mask_row"] = None
    if masked:
        n = max(3, int(b * R * masked))
        bits = rng.random((n, V)) < np.array([0.9, 0.0, 0.02])[np.arange(n) % 3][:, None]
        pad = -V % 32
        c["bits"] = bits
        c["mask"] = np.packbits(np.pad(bits, ((0, 0), (0, pad)), constant_values=True), axis=1,
                                bitorder="little").view(np.int32)      # bits past V are set: never read as ids
        c["mask_row"] = rng.integers(-1, n + 1, b * R).astype(np.int32)   # -1 and n: not masked
    return c


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def _call(X, c, logits, out, argmax, mask_value=float("-inf"), **over):
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    kw = dict(repetition=dev(c["rep"]), frequency=dev(c["freq"]), presence=dev(c["pres"]),
              history=dev(np.concatenate(c["hist"]).astype(np.int32)), history_offsets=dev(_offsets([len(h) for h in c["hist"]])),
              prompt_len=dev(c["plen"]), draft=dev(c["draft"]), mask=dev(c["mask"]), mask_row=dev(c["mask_row"]),
              mask_value=mask_value)
    if c["bias"] is not None:
        kw.update(bias_ids=dev(np.concatenate([i for i, _ in c["bias"]])),
                  bias_values=dev(np.concatenate([v for _, v in c["bias"]])),
                  bias_offsets=dev(_offsets([len(i) for i, _ in c["bias"]])))
    kw.update(over)
    assert X.process_logits(logits, out, argmax, rows=c["R"], **kw) == X.XPRESS_OK
    torch.cuda.synchronize()


def _reference(c, x, mask_value):
    """(fp32 values, 64-bit values, magnitude for the bound, allowed) per row."""
    b, R, V = c["b"], c["R"], c["V"]
    o32, o64 = np.empty((b * R, V), f4), np.empty((b * R, V))
    mag, ok = np.empty((b * R, V)), np.ones((b * R, V), bool)
    inside = lambda t: t[(t >= 0) & (t < V)]  # noqa: E731
    for q in range(b):
        prompt = np.zeros(V, bool)
        prompt[inside(c["hist"][q][:c["plen"][q]])] = True
        base = np.bincount(inside(c["hist"][q][c["plen"][q]:]), minlength=V)
        bias = np.zeros(V, f4)
        if c["bias"] is not None:
            for i, v in zip(*c["bias"][q]):                        # a later entry replaces an earlier one
                if 0 <= i < V:
                    bias[i] = v
        for j in range(R):
            n = base if c["draft"] is None else base + np.bincount(inside(c["draft"][q, :j]), minlength=V)
            seen = prompt | (n > 0)
            r = q * R + j
            for T, o in ((f4, o32), (np.float64, o64)):
                l = x[r].astype(T)
                rep, freq, pres = T(c["rep"][q]), T(c["freq"][q]), T(c["pres"][q])
                l = np.where(seen, np.where(l > 0, l / rep, l * rep), l)
                l = np.where(n > 0, (l - freq * n.astype(T)) - pres, l)
                o[r] = l + bias.astype(T)
            mag[r] = np.abs(x[r].astype(np.float64)) * max(c["rep"][q], 1 / c["rep"][q]) + \
                np.abs(c["freq"][q]) * n + abs(c["pres"][q]) + np.abs(bias)
            if c["mask"] is not None:
                m = r if c["mask_row"] is None else c["mask_row"][r]
                if 0 <= m < len(c["bits"]):
                    ok[r] = c["bits"][m]
    for o in (o32, o64):
        o[~ok] = mask_value
    return o32, o64, mag, ok


def _bf16_bits(a32):
    return torch.from_numpy(a32).to(BF16)


def _check(c, logits, out, argmax, mask_value=float("-inf")):
    x = logits.float().cpu().numpy()
    o32, o64, mag, ok = _reference(c, x, mask_value)
    if out is not None:
        want = _bf16_bits(o32) if logits.dtype is BF16 else torch.from_numpy(o32)
        got = out.cpu()
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        assert same.all(), f"{int((~same).sum())} of {same.numel()} values differ"
        g = got.double().numpy()
        fin = np.isfinite(o64) & ok
        bound = 6 * 2.0 ** -24 * mag + 1e-37
        if logits.dtype is BF16:                                    # half the spacing of the stored value
            bound = bound + 2.0 ** (np.floor(np.log2(np.where(fin, np.abs(o64), 0.0) + bound)) - 8)
        assert (np.abs(g[fin] - o64[fin]) <= bound[fin]).all()
    if argmax is not None:
        stored = (_bf16_bits(o32).float().numpy() if logits.dtype is BF16 else o32).copy()
        use = ok & ~np.isnan(stored)
        key = np.where(use, stored, -np.inf)
        top = key.max(axis=1, keepdims=True)
        first = np.argmax(use & (key == top), axis=1)
        want = np.where(use.any(axis=1), first, -1)
        np.testing.assert_array_equal(argmax.cpu().numpy(), want)


def _logits(c, dtype, seed, pad=0, off=0):
    n = c["b"] * c["R"]
    t = torch.full((n, off + c["V"] + pad), float("nan"), dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    v = t[:, off:off + c["V"]]
    v.normal_(0, 4, generator=g)
    return v


SHAPES = [  # b, R, V, history lengths, bias entries
    (1, 1, 1, [1], 1), (1, 1, 31, [0], 0), (1, 1, 32, [5], 3), (2, 1, 33, [7, 0], 40), (1, 4, 1000, [100], 10),
    (3, 2, 2047, [3, 1025, 1], 5), (2, 3, 2048, [4096, 33], 0), (2, 17, 2049, [0, 9000], 300),
    (5, 5, 4099, [50, 51, 52, 53, 54], 1), (1, 33, 8192, [30000], 100), (2, 1, 151936, [700, 5], 20),
    (40, 3, 20000, list(range(0, 400, 10)), 7), (1, 1, 9000, [20000], 5), (2, 3, 5001, [9000, 9001], 0),
    (1, 18, 30000, [50], 3), (70, 1, 60000, [3] * 70, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b, R, V, hist, n_bias", SHAPES)
def test_rules(X, b, R, V, hist, n_bias, dtype):
    c = _case(b, R, V, hist, n_bias, seed=b * 7 + V)
    for pad, off in ((0, 0), (3, 1), (8, 8)):
        x = _logits(c, dtype, V, pad, off)
        buf = torch.full((b * R, V + 5), 77.0, dtype=dtype, device="cuda")
        out, am = buf[:, :V], torch.full((b * R,), -9, dtype=torch.int32, device="cuda")
        _call(X, c, x, out, am)
        _check(c, x, out, am)
        assert (buf[:, V:] == 77.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [2080, 3001])
def test_rules_one_at_a_time_and_in_place(X, V, dtype):
    c = _case(3, 4, V, [60, 0, 500], 30, seed=5)
    none = dict(rep=np.ones(3, f4), freq=np.zeros(3, f4), pres=np.zeros(3, f4), bias=None, draft=None, mask=None,
                mask_row=None)
    x = _logits(c, dtype, 9)
    for keep in (["rep"], ["freq"], ["pres"], ["bias"], ["mask"], ["mask", "mask_row"], ["freq", "draft"],
                 ["rep", "draft"], list(none)):
        d = dict(c, **{k: v for k, v in none.items() if k not in keep})
        if keep == ["mask"]:                                        # row n by mask row n; the rest is not masked
            d["mask_row"] = None
        out, am = torch.empty_like(x), torch.empty(12, dtype=torch.int32, device="cuda")
        _call(X, d, x, out, am)
        _check(d, x, out, am)
        y, am2 = x.clone(), torch.empty_like(am)
        _call(X, d, y, y, am2)                                      # in place
        assert torch.equal(y.nan_to_num(1e9), out.nan_to_num(1e9)) and torch.equal(am, am2)
        am3 = torch.empty_like(am)
        _call(X, d, x, None, am3)                                   # argmax only
        assert torch.equal(am, am3)
        o2 = torch.empty_like(x)
        _call(X, d, x, o2, None)                                    # values only
        assert torch.equal(o2.nan_to_num(1e9), out.nan_to_num(1e9))
    # no rules at all: a copy and its first maximum
    out = torch.empty_like(x)
    assert X.process_logits(x, out, am) == X.XPRESS_OK
    assert torch.equal(out, x) and torch.equal(am.long(), x.float().argmax(dim=1))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rules_ids_outside_the_vocabulary_and_repeated_bias(X, dtype):
    V = 2500
    c = _case(2, 3, V, [40, 40], 6, seed=3)
    for q in range(2):
        c["hist"][q][::3] = np.array([-1, V, V + 5, 2 ** 31 - 1, -2 ** 31], np.int32)[np.arange(14) % 5]
        ids, vals = c["bias"][q]
        ids[1], ids[2], ids[4] = ids[0], -1, ids[0]                # three entries of one id, one outside
    c["draft"][:, 0] = -1
    c["draft"][1, 1] = V
    x = _logits(c, dtype, 4)
    out, am = torch.empty_like(x), torch.empty(6, dtype=torch.int32, device="cuda")
    _call(X, c, x, out, am)
    _check(c, x, out, am)


def test_rules_offsets_are_cut_to_their_arrays(X):
    V = 300
    c = _case(2, 1, V, [10, 10], 4, seed=8, draft=False, masked=0)
    x = _logits(c, F32, 4)
    out = torch.empty_like(x)
    bad = torch.tensor([-5, 10, 1 << 40], dtype=torch.int64, device="cuda")
    _call(X, c, x, out, None, history_offsets=bad, bias_offsets=torch.tensor([-3, 4, 1 << 50], dtype=torch.int64, device="cuda"))
    _check(c, x, out, None)
    _call(X, c, x, out, None, history_offsets=torch.tensor([15, 3, 1], dtype=torch.int64, device="cuda"))   # descending: empty
    d = dict(c, hist=[c["hist"][0][:0]] * 2, plen=np.zeros(2, np.int32))
    _check(d, x, out, None)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("mask_value", [float("-inf"), -1e30, "lowest"])
def test_rules_infinities_nans_and_empty_rows(X, dtype, mask_value):
    V = 2100
    mv = float(torch.finfo(dtype).min) if mask_value == "lowest" else mask_value
    c = _case(2, 4, V, [300, 300], 20, seed=6, masked=1.0)
    c["mask_row"] = np.array([0, 1, 2, -1, 1, 3, -1, 0], np.int32)    # rows 1 and 4: nothing allowed
    x = _logits(c, dtype, 4)
    x[0, 10], x[0, 11], x[3, 5], x[3, 6] = float("inf"), float("-inf"), float("nan"), float("inf")
    x[6] = float("-inf")                                             # a row of nothing but -inf: id 0 is its first maximum
    x[7] = float("nan")                                              # no value at all: -1
    x[2, 100:200] = float("nan")
    out, am = torch.empty_like(x), torch.empty(8, dtype=torch.int32, device="cuda")
    _call(X, c, x, out, am, mask_value=mv)
    stored = torch.tensor(mv, dtype=dtype).item()
    _check(c, x, out, am, stored)
    assert am[1] == -1 and am[4] == -1 and am[7] == -1
    assert (out[1] == stored).all() and (out[4] == stored).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b, R, V, hist", [(40, 17, 4200, 300), (90, 17, 4000, 5), (3, 17, 30000, 10000), (4, 16, 9001, 6000),
                                           (65, 9, 4096, 700), (30, 5, 44000, 20)])
def test_rules_groups_of_rows(X, b, R, V, hist, dtype):
    """Batches that leave a CTA several rows, whole groups and parts of one, with
    infinities, NaNs, rows that allow nothing, and in place."""
    c = _case(b, R, V, [hist + q for q in range(b)], 25, seed=V)
    x = _logits(c, dtype, V, pad=8 - V % 8)
    for j in range(R):                                               # each place of a group
        x[(b - 1) * R + j, 3 * j], x[j, 7 * j], x[R + j, 5 * j + 1] = float("inf"), float("-inf"), float("nan")
    x[2 * R] = float("nan")
    x[2 * R + 1] = float("-inf")
    c["mask_row"][2 * R:2 * R + 2] = -1
    c["mask_row"][1::7] = 1                                          # a grammar state without a token
    out, am = torch.empty_like(x), torch.full((b * R,), -9, dtype=torch.int32, device="cuda")
    _call(X, c, x, out, am)
    _check(c, x, out, am)
    y, am2 = x.clone(), torch.empty_like(am)
    _call(X, c, y, y, am2)
    assert torch.equal(am2, am) and ((y == out) | (y.isnan() & out.isnan())).all()


def test_rules_ties_go_to_the_lowest_id(X):
    for V, at in ((151936, (5, 70000, 151935)), (2500, (2047, 2048, 2499))):
        x = torch.zeros((3, V), dtype=BF16, device="cuda")
        x[0, list(at)] = 2.0
        x[1] = -0.0
        x[1, at[1]] = 0.0                                            # -0 and 0 are the same value
        x[2] = -1.0
        x[2, list(at[1:])] = -0.5
        am = torch.empty(3, dtype=torch.int32, device="cuda")
        X.process_logits(x, None, am)
        assert am.tolist() == [at[0], 0, at[1]]


def test_rules_rows_past_32_bits(X):
    n, V = 14500, 151936                                             # n * V = 2.2e9
    x = torch.zeros((n, V), dtype=BF16, device="cuda")
    x[-1, 7], x[-1, V - 1], x[-2, 99] = 3.0, 5.0, 4.0
    ids = torch.tensor([V - 1], dtype=torch.int32, device="cuda")
    off = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    off[-1] = 1                                                      # the last row's history alone
    am = torch.empty(n, dtype=torch.int32, device="cuda")
    X.process_logits(x, x, am, frequency=torch.full((n,), 3.0, device="cuda"), history=ids, history_offsets=off)
    assert am[-1] == 7 and am[-2] == 99 and x[-1, V - 1] == 2.0 and int(am[:-2].abs().sum()) == 0


def test_rules_calls_back_to_back_on_two_streams(X):
    """Calls that follow one another without a wait, two streams at a time, take
    only their own keys from the streams' workspaces."""
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    xs = [torch.randn((n, V), device="cuda", generator=g).to(BF16) for n, V in ((1, 151936), (5, 3000), (300, 700), (5000, 257))]
    want = [x.float().argmax(dim=1).to(torch.int32) for x in xs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for st in streams:
            with torch.cuda.stream(st):
                for i, x in enumerate(xs):
                    am = torch.empty(x.shape[0], dtype=torch.int32, device="cuda")
                    X.process_logits(x, None, am)
                    got.append((i, am))
    torch.cuda.synchronize()
    assert all(torch.equal(am, want[i]) for i, am in got)


def test_rules_empty_batch(X):
    e = torch.empty((0, 500), dtype=BF16, device="cuda")
    assert X.process_logits(e, e, torch.empty(0, dtype=torch.int32, device="cuda")) == X.XPRESS_OK


def test_rules_other_stream_and_graph(X):
    c = _case(4, 5, 5000, [10, 2000, 0, 77], 9, seed=2)
    x = _logits(c, BF16, 1)
    out, am = torch.empty_like(x), torch.empty(20, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _call(X, c, x, out, am, stream=side)
    _check(c, x, out, am)
    kw = dict(repetition=torch.full((20,), 1.3, device="cuda"), history=torch.arange(40, dtype=torch.int32, device="cuda"),
              history_offsets=torch.arange(21, dtype=torch.int64, device="cuda") * 2)
    want, wam = torch.empty_like(x), torch.empty_like(am)
    X.process_logits(x, want, wam, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X.process_logits(x, out, am, **kw)
    out.zero_()
    am.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(am, wam)
