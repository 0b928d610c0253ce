"""oscar_rope against the turn in 64 bits: types, pairings, partial and odd rotary widths, axes, far and negative
positions, strided rows, in place, inverse, gradients."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def _mods():
    import torch
    from paper_2605_19660_amd import binding as ob
    return torch, ob, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def reference(x, pos, inv, axes, adjacent, inverse):
    """x [n, heads, 128] fp64, pos [axes, n] int, inv fp32; the angle as an exact product, reduced in extended
    precision (64 bits of mantissa hold a 31-bit position times a 24-bit frequency)."""
    half = len(inv)
    a = pos[axes].T.astype(np.longdouble) * inv.astype(np.longdouble)
    a = np.remainder(a, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)[:, None]
    c, s = np.cos(a), np.sin(a) * (-1 if inverse else 1)
    y = x.copy()
    i = (np.arange(half) * 2, np.arange(half) * 2 + 1) if adjacent else (np.arange(half), np.arange(half) + half)
    y[..., i[0]] = x[..., i[0]] * c - x[..., i[1]] * s
    y[..., i[1]] = x[..., i[1]] * c + x[..., i[0]] * s
    return y, i


def check(got, x, pos, inv, axes, io, adjacent=False, inverse=False):
    """One rounding of the result to its type, and the turn's own error: the angle is off by at most
    2^-24 of half a turn from its rounding to fp32 and, beyond 2^24, 2^-52 of its number of turns twice
    (product, division by 2 pi); sine and cosine by 2 steps of fp32, products and sum by 3 half steps."""
    want, (i, j) = reference(x, pos, inv, axes, adjacent, inverse)
    err = np.abs(got - want)
    size = np.abs(x[..., i]) + np.abs(x[..., j])
    turns = np.abs(pos).max() * np.abs(inv).max() / 6.28
    fp32 = size * (np.pi * 2.0 ** -24 + 2 * np.pi * turns * 2.0 ** -52 + 4 * 2.0 ** -23 + 3 * 2.0 ** -24)
    for k in (i, j):
        bound = np.abs(want[..., k]) * HALF_STEP[io] * 1.001 + fp32 * 1.01 + (2.0 ** -25 if io == "f16" else 0)
        assert (err[..., k] <= bound).all(), (err[..., k] - bound).max()
    rest = np.setdiff1d(np.arange(128), np.concatenate([i, j]))
    assert np.array_equal(got[..., rest], x[..., rest])


def inputs(n, hq, hk, io, axes, rot, first, seed):
    torch, ob, types = _mods()
    rng = np.random.default_rng(seed)
    x = [torch.from_numpy(rng.standard_normal((n, h, 128)).astype(np.float32)).to(types[io]) for h in (hq, hk)]
    pos = (first + rng.integers(0, 5000, size=(axes, n))).astype(np.int32)
    inv = (10000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    axis = rng.integers(0, axes, size=rot // 2).astype(np.uint8)
    return x, pos, inv, axis


@pytest.mark.parametrize("io", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("n,hq,hk,axes,rot,first", [
    (1, 32, 8, 1, 128, 0), (5, 28, 4, 3, 128, 131072), (3, 7, 1, 2, 64, 1 << 20), (2, 1, 1, 4, 2, 7), (9, 5, 3, 3, 90, -300),
    (4, 3, 2, 1, 126, 2 ** 31 - 5001), (3, 40, 40, 2, 32, -2 ** 31), (2051, 3, 1, 3, 96, 99), (2049, 1, 2, 1, 24, 5)])
def test_rope(io, adjacent, n, hq, hk, axes, rot, first):
    torch, ob, _ = _mods()
    (q, k), pos, inv, axis = inputs(n, hq, hk, io, axes, rot, first, n + rot)
    dev = lambda a: torch.from_numpy(a).cuda()
    gq, gk = ob.rope(q.cuda(), k.cuda(), dev(pos), dev(inv), axes=bytes(axis), adjacent=adjacent)
    for g, x in ((gq, q), (gk, k)):
        check(g.cpu().double().numpy(), x.double().numpy(), pos, inv, axis, io, adjacent)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("adjacent,rot", [(False, 128), (True, 64), (False, 90)])
def test_rows_of_a_projection_in_place_one_side_and_inverse(io, adjacent, rot):
    torch, ob, types = _mods()
    n, hq, hk = 37, 12, 4
    (q, k), pos, inv, axis = inputs(n, hq, hk, io, 2, rot, 1000, 5)
    fused = torch.full((n, (hq + 2 * hk) * 128), 7.0, dtype=types[io], device="cuda")
    fq, fk = fused[:, :hq * 128].view(n, hq, 128), fused[:, hq * 128:(hq + hk) * 128].view(n, hk, 128)
    fq.copy_(q)
    fk.copy_(k)
    p, i = torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda()
    want = ob.rope(q.cuda(), k.cuda(), p, i, axes=bytes(axis), adjacent=adjacent)
    got = ob.rope(fq, fk, p, i, axes=bytes(axis), adjacent=adjacent)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    only_k = ob.rope(None, fk, p, i, axes=bytes(axis), adjacent=adjacent)
    assert only_k[0] is None and torch.equal(only_k[1], want[1])
    ob.rope(fq, None, p, i, axes=bytes(axis), adjacent=adjacent, out_q=fq)
    assert torch.equal(fq, want[0]) and torch.equal(fk.cpu(), k) and bool((fused[:, (hq + hk) * 128:] == 7).all())
    back = ob.rope(want[0], want[1], p, i, axes=bytes(axis), adjacent=adjacent, inverse=True)
    check(back[0].cpu().double().numpy(), want[0].cpu().double().numpy(), pos, inv, axis, io, adjacent, True)
    # batched positions [batch, T]
    b4 = ob.rope(q[:36].view(4, 9, hq, 128).cuda(), None, p[:, :36].contiguous(), i, axes=bytes(axis), adjacent=adjacent)[0]
    assert b4.shape == (4, 9, hq, 128) and torch.equal(b4.view(36, hq, 128), want[0][:36])


def test_infinities_stay_in_their_pairs():
    torch, ob, _ = _mods()
    q = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    q[0, 0, 100], q[0, 0, 5] = float("inf"), float("nan")
    inv = torch.full((32,), 0.1, device="cuda")
    for adjacent in (False, True):
        y = ob.rope(q, None, torch.tensor([3], dtype=torch.int32, device="cuda"), inv, adjacent=adjacent)[0][0, 0].cpu()
        bad = [5, 4] if adjacent else [5, 37]
        assert set(torch.nonzero(~torch.isfinite(y)).flatten().tolist()) == set(bad + [100]) and y[100] == float("inf")


def test_gradient():
    """The gradient of sum(w . rope(x)) is the inverse turn of w: against the formula and against differences."""
    torch, ob, _ = _mods()
    (q, _), pos, inv, axis = inputs(3, 2, 1, "f32", 2, 64, 50, 11)
    p, i = torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda()
    w = torch.randn(q.shape, generator=torch.Generator().manual_seed(1))
    grad = ob.rope(w.cuda(), None, p, i, axes=bytes(axis), inverse=True)[0].cpu().double().numpy()
    check(grad, w.double().numpy(), pos, inv, axis, "f32", False, True)
    f = lambda x: float((reference(x, pos, inv, axis, False, False)[0] * w.double().numpy()).sum())
    x = q.double().numpy()
    for at in ((0, 0, 0), (2, 1, 33), (1, 0, 63), (1, 1, 127)):
        d = np.zeros_like(x)
        d[at] = 0.5
        assert abs((f(x + d) - f(x - d)) - grad[at]) <= 1e-5      # linear: the difference is exact


def test_on_another_stream_and_in_a_graph():
    torch, ob, _ = _mods()
    (q, k), pos, inv, axis = inputs(64, 8, 2, "bf16", 2, 128, 0, 3)
    q, k, p, i = q.cuda(), k.cuda(), torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda()
    want = ob.rope(q, k, p, i, axes=bytes(axis))
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ob.rope(q, k, p, i, axes=bytes(axis), out_q=oq, out_k=ok, stream=s)
    s.synchronize()
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.rope(q, k, p, i, axes=bytes(axis), out_q=oq, out_k=ok)
    for step in range(3):
        p += 1
        want = ob.rope(q, k, p, i, axes=bytes(axis))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
