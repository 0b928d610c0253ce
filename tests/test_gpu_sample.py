"""oscar_sample against the rule in 64 bits: tokens exactly, probabilities to their rounding."""
import numpy as np
import pytest

from q8_numbers import ints, torch_type

pytestmark = pytest.mark.gpu


def rule(x, temp, k, p, m, u):
    """Tokens and probabilities of rows x, one after the other."""
    B, V = x.shape
    tokens, probs = np.zeros(B, int), np.zeros((B, V))
    for b, row in enumerate(x):
        row = np.where(np.isnan(row), -np.inf, np.minimum(row, 3.4028234663852886e38))
        order = np.argsort(-row, kind="stable")
        order = order[row[order] > -np.inf]
        if len(order) == 0:
            continue
        if not temp[b] > 0:
            order, t = order[:1], 1.0
        else:
            t = temp[b]
        if k[b] > 0:
            order = order[:k[b]]
        w = np.exp((row[order] - row[order[0]]) / t)
        if p[b] < 1:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            order = order[:max(1, int((before < p[b] * w.sum()).sum()))]
            w = w[:len(order)]
        if m[b] > 0:
            order = order[:max(1, int((w >= m[b]).sum()))]
        few = np.sort(order)
        w = np.exp((row[few] - row.max()) / t)
        cum = np.cumsum(w)
        tokens[b] = few[min(int((cum <= u[b] * cum[-1]).sum()), len(few) - 1)]
        probs[b, few] = w / cum[-1]
    return tokens, probs


def check(x, io="f32", temp=None, k=None, p=None, m=None, u=None, seed=0, stride=0):
    """x: numbers that the type holds.  Runs with and without probabilities."""
    import torch
    from paper_2605_19660_amd import binding as ob
    B, V = x.shape
    rng = np.random.default_rng(seed)
    u = rng.random(B).astype(np.float32) if u is None else np.asarray(u, np.float32)
    f = lambda a, none: (np.full(B, none, np.float32) if a is None else np.broadcast_to(np.asarray(a, np.float32), (B,)).copy())
    temp_, p_, m_ = f(temp, 1.0), f(p, 1.0), f(m, 0.0)
    k_ = np.zeros(B, np.int32) if k is None else np.broadcast_to(np.asarray(k, np.int32), (B,)).copy()
    logits = torch.from_numpy(x).to(torch_type(io)).cuda()
    if stride:
        wide = torch.full((B, V + stride), float("inf"), dtype=logits.dtype, device="cuda")
        wide[:, :V] = logits
        logits = wide[:, :V]
    d = lambda given, a: None if given is None else torch.from_numpy(a).cuda()
    kw = dict(temperature=d(temp, temp_), top_k=None if k is None else ints(k_), top_p=d(p, p_), min_p=d(m, m_))
    ud = torch.from_numpy(u).cuda()
    want, probs = rule(x.astype(np.float64), temp_.astype(np.float64), k_, p_.astype(np.float64), m_.astype(np.float64), u.astype(np.float64))
    token, none = ob.sample(logits, ud, **kw)
    assert none is None and np.array_equal(token.cpu().numpy(), want), (token.tolist()[:8], want[:8])
    token, got = ob.sample(logits, ud, probs=True, **kw)
    assert np.array_equal(token.cpu().numpy(), want)
    got = got.double().cpu().numpy()
    # one rounding to fp32 (a subnormal one at worst), of weights and sums good to 1e-12
    assert (np.abs(got - probs) <= probs * (2.0 ** -24 + 1e-11) + 2.0 ** -149).all(), float(np.abs(got - probs).max())
    assert np.array_equal(got > 0, probs.astype(np.float32) > 0)
    return want, probs


def logits(rng, B, V, io="f32", tail=1.2):
    import torch
    rank = np.argsort(rng.random((B, V)), -1)
    x = 1.5 * rng.standard_normal((B, V)) - tail * np.log1p(rank)
    return torch.from_numpy(x).to(torch_type(io)).double().numpy()


@pytest.mark.parametrize("io", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 1024, 1025, 4097, 32000, 50001])
def test_against_the_rule(V, io):
    rng = np.random.default_rng(V)
    x = logits(rng, 6, V, io)
    check(x, io)
    check(x, io, temp=[0.7, 1.0, 0.0, 1.5, 30.0, 0.05])
    check(x, io, k=[1, 2, 50, 1000, 0, 2000])
    check(x, io, p=[0.1, 0.5, 0.9, 0.99, 1.0, 0.0])
    check(x, io, m=[0.0, 0.01, 0.1, 0.5, 1.0, 1.5])
    check(x, io, temp=[0.7, 1.0, 1.3, 1.5, 1.0, 0.9], k=[0, 20, 0, 3000, 5, 100], p=[0.9, 0.95, 0.3, 0.8, 1.0, 0.99],
          m=[0.0, 0.02, 0.1, 0.0, 0.3, 0.001], stride=V % 7)


def test_a_large_vocabulary_and_many_rows():
    rng = np.random.default_rng(1)
    x = logits(rng, 12, 128003)
    check(x, k=[50, 0, 0, 1024, 1025, 100000] * 2, p=[0.95, 0.9, 1.0, 0.9, 0.7, 0.999] * 2, temp=[0.8, 1.2] * 6, m=[0.0] * 6 + [0.02] * 6)


@pytest.mark.parametrize("B, V", [(1, 4096), (128, 4096), (129, 4096), (256, 4000), (257, 4097), (4, 128003), (6, 128003), (2, 524288), (1, 1 << 22)])
def test_every_way_a_row_is_cut(B, V):
    """Few and many rows of one and of many pieces; a piece that is masked whole, a row that is, one of equal numbers."""
    rng = np.random.default_rng(B + V)
    io = ("f32", "bf16", "f16")[B % 3]
    x = logits(rng, B, V, io)
    x[0, V // 4:V // 4 + V // 2] = -np.inf
    if B > 3:
        x[1] = -np.inf
        x[2] = 0.25
    among = lambda *a: np.array(a)[rng.integers(0, len(a), size=B)]
    check(x, io, p=0.9)
    check(x, io, temp=among(0.0, 0.7, 1.0, 1.3), k=among(0, 0, 1, 50, 1024), p=among(1.0, 0.5, 0.95), m=among(0.0, 0.0, 0.02))


@pytest.mark.parametrize("V", [5, 1000, 6000, 40000])
def test_equal_logits(V):
    """Ties go to the lowest index, in any number: rows of one value, of two, and of a few that repeat."""
    rng = np.random.default_rng(V)
    x = np.zeros((6, V))
    x[1, V // 3:] = -1.0
    x[2] = rng.integers(0, 3, size=V)
    x[3] = rng.integers(0, 3, size=V) * 1e-6 - 5.0
    x[4] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    x[5, ::2] = 3.0
    x = x.astype(np.float32).astype(np.float64)
    check(x)
    for k in (1, 3, V // 2, V - 1, V, V + 5):
        check(x, k=k)
        check(x, k=k, p=0.5)
    for p in (0.25, 0.5, 0.75, 0.9):
        check(x, p=p)
        check(x, p=p, u=[0.0, 0.999999, 0.5, 0.25, 0.75, 0.1])
    check(x, m=0.5)


@pytest.mark.parametrize("V", [7, 3000, 20000])
def test_masked_infinite_and_missing_logits(V):
    rng = np.random.default_rng(V)
    x = logits(rng, 10, V)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, rng.random(V) < 0.9] = -np.inf
    x[3, rng.random(V) < 0.5] = np.nan
    x[4, V // 2] = np.inf
    x[5, [0, V - 1]] = np.inf
    x[6] = -3.4028234663852886e38
    x[7] = np.where(rng.random(V) < 0.5, 3.4028234663852886e38, -3.4028234663852886e38)
    x[8] = -np.inf
    x[8, V - 1] = -1e30
    x[9, :V - 2] = -np.inf
    x = x.astype(np.float32).astype(np.float64)
    for kw in (dict(), dict(k=2), dict(p=0.6), dict(m=0.1), dict(k=V // 2 + 1, p=0.9), dict(temp=0.0), dict(temp=1e-30),
               dict(temp=np.inf), dict(temp=np.nan), dict(p=np.nan, m=np.nan), dict(p=-1.0), dict(k=-3)):
        check(x, **kw)


def test_numbers_at_the_ends():
    rng = np.random.default_rng(3)
    x = logits(rng, 8, 5000)
    last = np.nextafter(np.float32(1), np.float32(0))
    for kw in (dict(), dict(k=30), dict(p=0.9)):
        check(x, u=[0.0, last, 0.5, 1e-30, 0.0, last, 2.0 ** -24, 0.25], **kw)


def test_narrow_and_wide_spreads():
    """Logits that differ in their last bits only, or by thousands."""
    rng = np.random.default_rng(4)
    V = 9000
    base = np.float32(17.0)
    x = np.stack([base + rng.integers(0, 50, size=V) * np.spacing(base), rng.standard_normal(V) * 3000, rng.standard_normal(V) * 1e-30,
                  np.where(rng.random(V) < 0.001, 20.0, -80.0), -np.arange(V) * 0.01, np.arange(V) * 1e-3]).astype(np.float32).astype(np.float64)
    for kw in (dict(), dict(k=40), dict(k=5000), dict(p=0.3), dict(p=0.999), dict(k=6000, p=0.9, m=1e-4), dict(temp=0.01, p=0.9), dict(temp=1000.0, p=0.9)):
        check(x, **kw)


def test_draws_follow_the_probabilities():
    """Random numbers spread evenly over [0, 1) give every token its share."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(5)
    x = torch.from_numpy(logits(rng, 1, 200)).float().cuda()
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token, probs = ob.sample(x.expand(n, -1).contiguous(), u, top_p=torch.full((n,), 0.9, device="cuda"), probs=True)
    share = torch.bincount(token.long(), minlength=200).double() / n
    # an interval of the running sum holds as many of the n points as its length says, one more or less
    assert float((share - probs[0].double()).abs().max()) <= 1.0 / n + 1e-6


def test_replays_and_other_streams():
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(6)
    B, V = 4, 30000
    x, u = torch.zeros(B, V, device="cuda"), torch.zeros(B, device="cuda")
    k, p = ints([0, 40, 0, 2000]), torch.tensor([0.9, 1.0, 1.0, 0.8], device="cuda")
    tokens, probs = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, V, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.sample(x, u, top_k=k, top_p=p, tokens=tokens, probs=probs)
    s = torch.cuda.Stream()
    for i in range(4):
        x.copy_(torch.from_numpy(logits(rng, B, V)))
        u.copy_(torch.from_numpy(rng.random(B)))
        graph.replay()
        torch.cuda.synchronize()
        t, q = ob.sample(x, u, top_k=k, top_p=p, probs=True, stream=s)
        s.synchronize()
        assert torch.equal(t, tokens) and torch.equal(q, probs)
        want, _ = rule(x.double().cpu().numpy(), np.ones(B), k.cpu().numpy(), p.double().cpu().numpy(), np.zeros(B), u.double().cpu().numpy())
        assert np.array_equal(tokens.cpu().numpy(), want)


def test_long_lists_of_every_kind():
    """Lists of hundreds to thousands of tokens that are sorted: spread, crowded on one side of zero or about it, beside one
    far above, in a few values with many ties."""
    rng = np.random.default_rng(7)
    V = 20000
    x = np.stack([rng.standard_normal(V), rng.random(V) * 1e-3, (rng.random(V) - 0.5) * 1e-35, rng.random(V) * 1e-4 - 30.0,
                  rng.integers(0, 200, size=V) * 0.25, rng.integers(0, 3, size=V) - 1.0, -np.arange(V) * 1e-4, rng.standard_normal(V) ** 3])
    x[3, 17] = 40.0
    x = x.astype(np.float32).astype(np.float64)
    for k in (255, 256, 257, 512, 513, 1000, 1024):
        check(x, k=k)
        check(x, k=k, p=0.8, temp=0.5)
    check(x, k=1025)
    check(x, k=5000, p=0.9)
    check(x, p=0.02)
    check(x, m=0.97, temp=2.0)


@pytest.mark.parametrize("levels", [1, 1000, 3000])
def test_many_small_weights_beside_a_large_one(levels):
    """2^22 tokens of which all but one weigh 2.5e-13: a top_p that needs hundreds of thousands of them.  They are too many
    for a list, and their sum is 1e-6 of the one that is large."""
    import torch
    from paper_2605_19660_amd import binding as ob
    V = 1 << 22
    x = (-29.0 - (np.arange(V) * 7919 % levels) * np.spacing(np.float32(29))).astype(np.float32)
    x[V - 1] = 0.0
    p, u = np.float32(0.999999), np.float32(2e-8)
    # sums of up to 2^22 numbers in 64 bits of mantissa: 2^-41 of the sum, 2 of the small ones
    w = np.exp(x.astype(np.longdouble))
    order = np.argsort(-x, kind="stable")
    before = np.concatenate([[0], np.cumsum(w[order])[:-1]])
    n = int((before < np.longdouble(p) * w.sum()).sum())
    assert 100_000 < n < 400_000
    token, probs = ob.sample(torch.from_numpy(x)[None].cuda(), torch.tensor([u]).cuda(), top_p=torch.tensor([p]).cuda(), probs=True)
    stays = probs[0].cpu().numpy() > 0
    assert abs(int(stays.sum()) - n) <= 4, (int(stays.sum()), n)
    # the largest n, equal ones by index, whatever n came out as
    mine = np.sort(order[:int(stays.sum())])
    assert np.array_equal(np.nonzero(stays)[0], mine)
    cum = np.cumsum(w[mine])
    assert abs(int(np.searchsorted(mine, int(token))) - int((cum <= np.longdouble(u) * cum[-1]).sum())) <= 4
    want = (w[mine] / cum[-1]).astype(np.float64)
    got = probs[0].double().cpu().numpy()[mine]
    assert (np.abs(got - want) <= want * (2.0 ** -24 + 1e-11)).all()


def test_a_number_of_1_and_more_draws_the_last_that_stays():
    """Every way a row is drawn: no filter, a list by tokens and by weights, rows that one workgroup searches."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(31)
    for B, V in ((1, 50), (4, 9001), (3, 128003)):
        x = logits(rng, B, V)
        x[0, V - 3:] = -np.inf
        for kw in (dict(), dict(k=40), dict(p=0.9), dict(m=0.02), dict(p=0.95, m=1e-3), dict(k=2000, p=0.9), dict(temp=1e-9, p=0.9)):
            f = {n: np.broadcast_to(np.asarray(a, np.int32 if n == "k" else np.float32), (B,)) for n, a in kw.items()}
            g = lambda n, none: f.get(n, np.full(B, none)).astype(np.float64)
            _, probs = rule(x.astype(np.float32).astype(np.float64), g("temp", 1.0), f.get("k", np.zeros(B, int)), g("p", 1.0), g("m", 0.0), np.zeros(B))
            want = [int(np.nonzero(r)[0][-1]) for r in probs]
            names = dict(temp="temperature", k="top_k", p="top_p", m="min_p")
            args = {names[n]: torch.from_numpy(a.copy()).cuda() for n, a in f.items()}
            for u in (1.0, 2.5, np.inf):
                token, _ = ob.sample(torch.from_numpy(x).float().cuda(), torch.full((B,), u, device="cuda"), **args)
                assert token.tolist() == want, (B, V, kw, u)


@pytest.mark.parametrize("V", [5000, 70000])
def test_tokens_of_hardly_any_weight(V):
    """min_p lets tokens of e^-60 of the largest stay, which no sum of the row shows: a random number of 0 draws the first of them, a tiny one
    the token it says."""
    x = np.zeros((6, V))
    x[:, :4096] = -np.inf
    x[:, 10:110] = -60.0
    x[4:, 10:110] = -69.0
    x[5, 7] = -70.0                                             # (does not stay)
    last = np.nextafter(np.float32(1), np.float32(0))
    few = 8.756510762696521e-27 / (V - 4096)                    # e^-60 of the sum, nearly
    check(x, m=1e-30, u=[0.0, 20.5 * few, 99.5 * few, 1e-20, 0.0, last])


def test_lists_that_span_all_numbers():
    """Hundreds of tokens about the largest fp32 numbers of both signs: the list's span is itself no number."""
    rng = np.random.default_rng(41)
    V = 3000
    x = np.stack([rng.choice([-1.0, 1.0], size=V) * rng.uniform(1e38, 3.4e38, size=V), rng.uniform(-3.4e38, 3.4e38, size=V),
                  np.where(rng.random(V) < 0.9, -3.4028234663852886e38, 3.4028234663852886e38)]).astype(np.float32).astype(np.float64)
    x[0, 7], x[1, 9] = np.inf, -np.inf
    for kw in (dict(k=1000), dict(k=300, p=0.5), dict(k=1024, temp=1e38), dict(k=700, temp=1e37, p=0.9), dict(k=2000, temp=np.inf), dict(temp=1e38, p=0.9)):
        check(x, **kw)


def test_a_count_past_the_bins_of_a_low_temperature():
    """top_k whose last token lies further below the largest than the bins of a low temperature reach, over many tokens."""
    rng = np.random.default_rng(42)
    x = logits(rng, 4, 128003)
    x[2:, 500] = x[2:].max() + 20.0
    for kw in (dict(k=50, temp=0.05), dict(k=1000, temp=0.1), dict(k=50, temp=[0.1, 0.3, 0.1, 0.4], p=0.9), dict(k=[1000, 1024, 50, 1025], temp=0.2, p=0.999)):
        check(x, **kw)
