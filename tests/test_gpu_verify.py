"""oscar_verify_drafts against the rule in exact and 64-bit arithmetic: types, vocabularies of every alignment,
ragged drafts, equal rows, empty rows, numbers that are no probabilities, and what it is distributed as."""
from fractions import Fraction

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _mods():
    import torch
    from paper_2605_19660_amd import binding as ob
    return torch, ob


def clean(x):
    x = np.where(x > 0, x.astype(np.float64), 0.0)
    return np.minimum(x, np.finfo(np.float32).max)


def rule(p, q, drafts, u, lens):
    """p [B, T+1, V], q [B, T, V] as the type holds them, fp64."""
    B, T, V = q.shape
    n_new, tokens = np.zeros(B, np.int32), np.full((B, T + 1), -1, np.int32)
    p, q = clean(p), clean(q)
    for b in range(B):
        n = T if lens is None else min(max(int(lens[b]), 0), T)
        a = 0
        while a < n:
            x = int(drafts[b, a])
            if not (0 <= x < V and Fraction(float(u[b, a])) * Fraction(q[b, a, x]) < Fraction(p[b, a, x])):
                break
            a += 1
        w = np.maximum(p[b, a] - q[b, a], 0) if a < n else p[b, a]
        if not w.any():
            w = p[b, a]
        cum = np.cumsum(w)
        over = np.nonzero(cum > max(float(u[b, T]), 0.0) * cum[-1])[0]
        pick = over[0] if len(over) else (np.nonzero(w)[0][-1] if w.any() else 0)
        tokens[b, :a] = drafts[b, :a]
        tokens[b, a] = pick
        n_new[b] = a + 1
    return n_new, tokens


def run(p, q, drafts, u, lens, **kw):
    torch, ob = _mods()
    dev = lambda x: None if x is None else x.cuda() if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda()
    n, t = ob.verify_drafts(dev(p), dev(q), dev(drafts), dev(u), draft_lens=dev(lens), **kw)
    return n.cpu().numpy(), t.cpu().numpy()


def rows(B, T, V, io, seed, near=0.7):
    torch, _ = _mods()
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(B, T + 1, V, generator=g) * 3
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :T] + near * torch.randn(B, T, V, generator=g), -1)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[io]
    drafts = torch.multinomial(q.reshape(B * T, V), 1, generator=g).view(B, T).int() if T else torch.zeros(B, 0, dtype=torch.int32)
    return p.to(dt), q.to(dt), drafts, torch.rand(B, T + 1, generator=g)


@pytest.mark.parametrize("io", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (2, 3, 2), (5, 4, 17), (3, 0, 1000), (7, 5, 4095), (4, 2, 4096), (4, 7, 4097),
                                   (3, 12, 8193), (2, 300, 33), (6, 3, 32001), (1, 4, 200003)])
@pytest.mark.parametrize("ragged", [False, True])
def test_rule(io, B, T, V, ragged):
    p, q, drafts, u = rows(B, T, V, io, B * 7919 + V)
    lens = np.random.default_rng(V).integers(-1, T + 2, size=B).astype(np.int32) if ragged else None
    got = run(p, q, drafts, u, lens)
    want = rule(p.double().numpy(), q.double().numpy(), drafts.numpy(), u.numpy(), lens)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_more_pieces_than_threads():
    """2^20 + 3 tokens are 257 pieces; the row's weight sits in single tokens at both ends and at the pieces' edges."""
    torch, _ = _mods()
    V = (1 << 20) + 3
    at = np.array([0, 4095, 4096, 255 * 4096, 256 * 4096 - 1, 256 * 4096, V - 1])
    p = np.zeros((len(at) * 2, 1, V), np.float32)
    p[:, 0, at] = np.arange(1, len(at) + 1, dtype=np.float32)
    total, below = p[0, 0, at].sum(), np.concatenate([[0], np.cumsum(p[0, 0, at])])
    u = np.concatenate([below[:-1] / total, np.nextafter((below[1:] / total).astype(np.float32), np.float32(0))]).astype(np.float32)[:, None]
    got = run(p, np.zeros((len(at) * 2, 0, V), np.float32), np.zeros((len(at) * 2, 0), np.int32), u, None)
    want = rule(p.astype(np.float64), np.zeros((len(at) * 2, 0, V)), np.zeros((len(at) * 2, 0), np.int32), u, None)
    assert np.array_equal(got[1], want[1]) and (got[0] == 1).all()


def test_borders_are_exact():
    """Dyadic rows: u p and u q fall on the borders exactly; a token starts where the running sum has passed."""
    V = 8
    p = np.full((9, 2, V), 0.125, np.float32)
    q = np.full((9, 1, V), 0.25, np.float32)
    u = np.zeros((9, 2), np.float32)
    u[:, 0] = 0.5                                    # 0.5 * 0.25 < 0.125 does not hold: every draft falls
    u[:8, 1] = np.arange(8) / 8                       # the rest is all zero, so the row itself is drawn from
    u[8, 1] = 1.0                                    # (outside [0, 1): the last)
    n, t = run(p, q, np.zeros((9, 1), np.int32), u, None)
    assert (n == 1).all() and t[:, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 7] and (t[:, 1] == -1).all()
    u[:, 0] = np.nextafter(np.float32(0.5), np.float32(0))
    assert (run(p, q, np.zeros((9, 1), np.int32), u, None)[0] == 2).all()


def test_rows_that_are_no_probabilities():
    V = 5000
    rng = np.random.default_rng(2)
    p, q = rng.random((6, 2, V)).astype(np.float32), rng.random((6, 1, V)).astype(np.float32)
    drafts, u = np.full((6, 1), 7, np.int32), np.full((6, 2), 0.5, np.float32)
    p[0] = 0                                          # nothing to draw from: token 0
    p[1, 0], q[1, 0] = q[1, 0], p[1, 0]
    p[1, 0, ::3], q[1, 0, 1::3] = np.nan, -1.0
    p[2, :, 4999], q[2, 0, 3] = np.inf, np.inf
    q[3] = p[3, :1]                                   # equal rows: every draft stands
    drafts[4] = V                                     # outside the vocabulary
    drafts[5] = -1
    got = run(p, q, drafts, u, None)
    want = rule(p, q, drafts, u, None)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    assert got[1][0, 0] == 0 and got[0][3] == 2 and got[0][4] == got[0][5] == 1 and got[1][2, got[0][2] - 1] == 4999


def test_unaligned_rows_given_outputs_workspace_stream_and_graph():
    torch, ob = _mods()
    V, B, T = 1003, 3, 2
    p, q, drafts, u = rows(B, T, V, "bf16", 9)
    want = rule(p.double().numpy(), q.double().numpy(), drafts.numpy(), u.numpy(), None)
    store = torch.zeros(p.numel() + 1, dtype=p.dtype, device="cuda")
    store[1:] = p.flatten().cuda()
    dp, dq, dd, du = store[1:].view(p.shape), q.cuda(), drafts.cuda(), u.cuda()
    n, tok = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, T + 1, dtype=torch.int32, device="cuda")
    ws = torch.full((ob.verify_workspace_bytes(B, V),), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ob.verify_drafts(dp, dq, dd, du, n_new=n, tokens=tok, workspace=ws, stream=s)
    s.synchronize()
    assert np.array_equal(n.cpu().numpy(), want[0]) and np.array_equal(tok.cpu().numpy(), want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.verify_drafts(dp, dq, dd, du, n_new=n, tokens=tok, workspace=ws)
    for step in range(4):
        du.copy_(torch.rand(B, T + 1, generator=torch.Generator().manual_seed(step)))
        eager = ob.verify_drafts(dp, dq, dd, du)
        graph.replay()
        torch.cuda.synchronize()
        want = rule(p.double().numpy(), q.double().numpy(), drafts.numpy(), du.cpu().numpy(), None)
        for g in ((n, tok), eager):
            assert np.array_equal(g[0].cpu().numpy(), want[0]) and np.array_equal(g[1].cpu().numpy(), want[1])


def test_what_comes_out_is_distributed_as_the_target():
    """20000 steps of one draft over 6 tokens: the first token's frequencies are the target's, within six standard
    deviations of a binomial."""
    torch, ob = _mods()
    B = 20000
    g = torch.Generator().manual_seed(4)
    p = torch.tensor([0.05, 0.3, 0.1, 0.25, 0.2, 0.1])
    q = torch.tensor([0.3, 0.1, 0.1, 0.05, 0.15, 0.3])
    drafts = torch.multinomial(q, B, replacement=True, generator=g).view(B, 1).int()
    n, t = run(p.expand(B, 2, 6).contiguous(), q.expand(B, 1, 6).contiguous(), drafts, torch.rand(B, 2, generator=g), None)
    freq = np.bincount(t[:, 0], minlength=6) / B
    sigma = np.sqrt(p.numpy() * (1 - p.numpy()) / B)
    assert (np.abs(freq - p.numpy()) <= 6 * sigma).all()
    stand = np.minimum(p.numpy(), q.numpy()).sum()
    assert abs((n == 2).mean() - stand) <= 6 * np.sqrt(stand * (1 - stand) / B)
