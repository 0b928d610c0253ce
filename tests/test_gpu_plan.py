"""oscar_plan_step against the rule written out sequence by sequence: pages given back, pages handed out, who waits, and
the rows of the step."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def rule(lens, keep, want, table, free, n_free, n_rows, ps):
    """The header's words, one sequence after the other."""
    table, free = table.copy(), free.copy()
    B, P = table.shape
    N = len(free)
    up = lambda x: -(-x // ps)
    lens = [min(max(int(x), 0), P * ps) for x in lens]
    k = [min(max(int(x), 0), n) for x, n in zip(lens if keep is None else keep, lens)]
    count = n_free
    for b in range(B):
        for p in range(up(k[b]), up(lens[b])):
            free[count] = table[b, p]
            count += 1
    top, asked, rows, given = count, 0, 0, 0
    out = {"lens": [], "new_lens": [], "row_starts": [], "positions": [], "row_seq": [], "slots": []}
    wants_rows = 0
    for b in range(B):
        w = max(int(want[b]), 0)
        fits = w > 0 and k[b] + w <= ps * P
        need = up(k[b] + w) - up(k[b]) if fits else 0
        asked += need
        paged = fits and (need == 0 or asked <= top)
        wants_rows += w if paged else 0
        n = w if paged and wants_rows <= n_rows else 0
        if n:
            for i in range(need):
                table[b, up(k[b]) + i] = free[count - 1]
                count -= 1
        out["lens"].append(k[b] + n)
        out["new_lens"].append(n)
        out["row_starts"].append(rows)
        for t in range(n):
            pos = k[b] + t
            out["positions"].append(pos)
            out["row_seq"].append(b)
            out["slots"].append(table[b, pos // ps] * ps + pos % ps)
        rows += n
    out["row_starts"].append(rows)
    for name in ("positions", "row_seq", "slots"):
        out[name] += [-1] * (n_rows - rows)
    out["n_free"] = [count]
    return {n: np.array(x, np.int64) for n, x in out.items()}, table, free


def world(B, P, ps, seed, spare, long=False):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, P * ps + 1, size=B) if long else rng.integers(0, min(P * ps, 3 * ps) + 1, size=B)
    held = -(-lens // ps)
    total = int(held.sum()) + spare
    perm = rng.permutation(total)
    table = np.full((B, P), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.zeros(max(total, 1), np.int32)
    free[:spare] = perm[at:]
    return rng, lens, table, free


def call(lens, keep, want, table, free, n_free, n_rows, ps, in_place=False, maps=True, fill=-7):
    import torch
    from paper_2605_19660_amd import binding as ob
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
    lens, keep, want, table, free, n_free = (dev(x) for x in (lens, keep, want, table, free, [n_free]))
    kw = dict(lens_out=lens, new_lens=want, n_free_out=n_free) if in_place else {}
    p = ob.plan_step(lens, want, table, free, n_free, n_rows, keep=keep, page_size=ps, **kw)
    got = {n: getattr(p, n).cpu().numpy().astype(np.int64) for n in p._fields}
    return got, table.cpu().numpy(), free.cpu().numpy()


def same(got, ref):
    for n, x in ref[0].items():
        assert np.array_equal(got[0][n], x), n
    assert np.array_equal(got[1], ref[1])
    assert np.array_equal(got[2], ref[2])


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,P,ps", [(1, 1, 128), (8, 9, 128), (63, 5, 128), (64, 5, 16), (200, 40, 128), (1023, 4, 128),
                                    (1024, 4, 128), (1025, 3, 128), (3000, 6, 64), (5, 3, 1), (17, 4, 100)])
def test_against_the_rule(B, P, ps, in_place):
    for seed in range(3):
        rng, lens, table, free = world(B, P, ps, seed, spare=int(B * (0.3 + seed)), long=seed == 2)
        want = np.where(rng.random(B) < 0.7, 1, rng.integers(-2, 2 * ps + 2, size=B))
        keep = None
        if seed:
            r = rng.random(B)
            keep = np.where(r < 0.2, 0, np.where(r < 0.5, lens - rng.integers(0, ps + 2, size=B), lens + rng.integers(0, 2, size=B)))
        n_free = int(B * (0.3 + seed))
        n_rows = int(np.maximum(want, 0).sum()) + 3 if seed != 1 else int(np.maximum(want, 0).sum() * 0.7)
        same(call(lens, keep, want, table, free, n_free, n_rows, ps, in_place),
             rule(lens, keep, want, table, free, n_free, n_rows, ps))


@pytest.mark.parametrize("n_rows", [0, 1, 8191, 8192, 8193, 40000])
def test_a_long_prompt_among_single_tokens(n_rows):
    """Rows within one launch and in a launch of their own."""
    lens = np.array([5, 0, 127, 128, 0], np.int64)
    want = np.array([1, 30001, 1, 1, 9000], np.int64)
    table = np.full((5, 300), -1, np.int32)
    table[0, 0], table[2, 0], table[3, 0] = 3, 1, 2
    free = np.concatenate([np.arange(4, 504), np.zeros(4, int)]).astype(np.int32)
    same(call(lens, None, want, table, free, 400, n_rows, 128), rule(lens, None, want, table, free, 400, n_rows, 128))


def test_pages_come_back_and_are_handed_out_in_the_same_step():
    """A sequence ends and another takes its place; its pages are the first to go out."""
    lens, keep, want = np.array([300, 128, 10]), np.array([0, 128, 10]), np.array([200, 1, 200])
    table = np.array([[7, 5, 3, -1], [1, -1, -1, -1], [0, -1, -1, -1]], np.int32)
    free = np.array([2, 0, 0, 0, 0, 0, 0, 0], np.int32)
    got = call(lens, keep, want, table, free, 1, 1000, 128, in_place=True)
    same(got, rule(lens, keep, want, table, free, 1, 1000, 128))
    assert got[1][0, :2].tolist() == [3, 5] and got[1][1, 1] == 7 and got[1][2, 1] == 2
    assert got[0]["new_lens"].tolist() == [200, 1, 200] and got[0]["n_free"].tolist() == [0]


def test_who_waits_for_pages_is_not_overtaken_but_keeps_nobody_from_its_own_page():
    lens, want = np.array([0, 5, 0, 7]), np.array([500, 1, 100, 1])
    table = np.full((4, 4), -1, np.int32)
    table[1, 0], table[3, 0] = 0, 1
    free = np.array([2, 3, 4, 0, 0], np.int32)
    got = call(lens, None, want, table, free, 3, 700, 128)
    same(got, rule(lens, None, want, table, free, 3, 700, 128))
    assert got[0]["new_lens"].tolist() == [0, 1, 0, 1] and got[0]["n_free"].tolist() == [3]


def test_numbers_that_make_no_sense_stay_inside_their_tensors():
    """Lengths, stacks and page numbers out of range: what comes out is not defined, what lies around it is untouched."""
    import torch
    from paper_2605_19660_amd import binding as ob
    big = 2 ** 31 - 1
    e = lambda *s: torch.full(s, -9, dtype=torch.int32, device="cuda")
    for lens, keep, want, count in (([big, -5, 900], [big, 3, -7], [big, big, 1], big), ([-1, big, big], [0, 0, 0], [1, 1, 1], -4)):
        table, free = e(5, 4), e(8 + 6)
        table[1:4] = torch.tensor([[99, -3, big, 5]] * 3)
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        p = ob.plan_step(dev(lens), dev(want), table[1:4], free[3:11], dev([count]), 6, keep=dev(keep))
        assert (table[0] == -9).all() and (table[4] == -9).all() and (free[:3] == -9).all() and (free[11:] == -9).all()
        assert int(p.row_starts[-1]) <= 6


def test_an_empty_batch():
    import torch
    from paper_2605_19660_amd import binding as ob
    e = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    p = ob.plan_step(e(0), e(0), e(0, 3), e(4), torch.tensor([2], dtype=torch.int32, device="cuda"), 5)
    assert p.n_free.tolist() == [2] and p.row_starts.tolist() == [0] and p.slots.tolist() == [-1] * 5


def test_replayed_steps_keep_the_books():
    """A captured plan in place, replayed: every page is in the stack or in one row of the table, once, at any time."""
    import torch
    from paper_2605_19660_amd import binding as ob
    B, P, N, rows = 6, 8, 30, 300
    e = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    lens, keep, want, table, free, n_free = e(B), e(B), e(B), e(B, P), e(N), e(1)
    free.copy_(torch.arange(N))
    n_free.fill_(N)
    out = dict(new_lens=e(B), row_starts=e(B + 1), positions=e(rows), row_seq=e(rows), slots=e(rows))
    step = lambda: ob.plan_step(lens, want, table, free, n_free, rows, keep=keep, lens_out=lens, n_free_out=n_free, **out)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
    torch.cuda.synchronize()
    lens.zero_(), table.zero_(), free.copy_(torch.arange(N)), n_free.fill_(N)
    rng = np.random.default_rng(0)
    book = (np.zeros(B, int), np.zeros((B, P), np.int32), np.arange(N, dtype=np.int32), N)
    for i in range(40):
        w = np.where(rng.random(B) < 0.6, 1, rng.integers(0, 400, size=B))
        k = np.where(rng.random(B) < 0.15, 0, book[0] - (rng.random(B) < 0.3))
        want.copy_(torch.from_numpy(w)), keep.copy_(torch.from_numpy(k))
        graph.replay()
        ref, tab, fr = rule(book[0], k, w, book[1], book[2], book[3], rows, 128)
        same(({**{n: out[n].cpu().numpy() for n in out}, "lens": lens.cpu().numpy(), "n_free": n_free.cpu().numpy()},
              table.cpu().numpy(), free.cpu().numpy()), (ref, tab, fr))
        book = (ref["lens"], tab, fr, int(ref["n_free"][0]))
        held = np.concatenate([tab[b, :-(-int(n) // 128)] for b, n in enumerate(book[0])] + [fr[:book[3]]])
        assert sorted(held.tolist()) == list(range(N))
