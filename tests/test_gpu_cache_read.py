"""oscar_cache_read against the cache's numbers in 64 bits: formats, types, ranges that start and end anywhere
(inside pages, in the window, before and behind the sequence), rows left alone, bad pages."""
import numpy as np
import pytest

from cache_numbers import filled_cache, hadamard, numbers, torch_type

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def read(c, starts, T, out, which="kv", fill=-77.0):
    import torch
    from paper_2605_19660_amd import binding as ob
    shape = (c.batch, T, c.cfg.n_kv_heads, 128)
    k, v = (torch.full(shape, fill, dtype=torch_type(out), device="cuda") if x in which else None for x in "kv")
    s = None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda")
    assert ob.cache_read(c, s, k=k, v=v) == (k, v)
    return [None if x is None else x.double().cpu().numpy() for x in (k, v)]


def check(c, starts, T, out, held=None):
    """Values: (c - z) is exact and its product rounds once in fp32 (zero added: once more), then once to the
    type.  Keys: the same for K_u, the rotation's 7 stages and the factor n / sqrt(128) (rounded, multiplied)
    each round once: at most 10 half steps of fp32 of the channels' absolute sum through the rotation."""
    got_k, got_v = read(c, starts, T, out)
    H = hadamard()
    rotated = c.cfg.rotation == 0
    for b, s in enumerate(numbers(c)):
        start = 0 if starts is None else starts[b]
        n = s["n"].shape[1]
        t = np.arange(start, start + T)
        there = (t >= 0) & (t < n)
        if held is not None:
            there &= held(b, t)
        assert (got_k[b, ~there] == -77).all() and (got_v[b, ~there] == -77).all()
        if not there.any():
            continue
        t = t[there]
        v, vmag = s["vc"] + s["vb"], np.abs(s["vc"]) + np.abs(s["vb"])
        k, kmag = s["kc"] + s["kb"], np.abs(s["kc"]) + np.abs(s["kb"])
        kmag = np.maximum(np.abs(k), kmag if c.cfg.zp_mode else np.abs(k)) * s["n"][..., None]
        k = k * s["n"][..., None]
        if rotated:
            k, kmag = k @ H, kmag @ np.abs(H)
        tiny = 2.0 ** -25 if out == "f16" else 0.0
        for got, want, fp32 in ((got_v, v, 3 * 2.0 ** -24 * (vmag if c.cfg.zp_mode else np.abs(v))),
                                (got_k, k, 10 * 2.0 ** -24 * kmag)):
            g, w, f = got[b, there], want[:, t].transpose(1, 0, 2), fp32[:, t].transpose(1, 0, 2)
            bound = (np.abs(w) + f) * HALF_STEP[out] * 1.001 + f * 1.001 + tiny
            assert (np.abs(g - w) <= bound).all(), (b, (np.abs(g - w) - bound).max())


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bits,kg,vg,io,meta,zp_min", [
    (2, 128, 32, "bf16", "f16", False), (4, 128, 32, "f16", "f16", False), (2, 32, 64, "f16", "f16", True),
    (4, 64, 128, "bf16", "f32", False), (2, 64, 32, "f32", "f32", True), (4, 32, 128, "f32", "f16", True),
    (2, 128, 128, "f32", "f32", False)])
def test_formats(bits, kg, vg, io, meta, zp_min, out):
    c = filled_cache([700, 128, 1, 0, 383], hk=3, hq=3, bits=bits, kg=kg, vg=vg, io=io, meta=meta, zp_min=zp_min,
                     scattered=True, seed=bits * kg + vg)
    check(c, None, 701, out)
    check(c, [129, 100, 0, -5, 300], 260, out)


@pytest.mark.parametrize("starts,T", [
    ([0, 0, 0], 1), ([127, 128, 129], 1), ([127, 128, 129], 2), ([1, 255, 383], 130), ([384, 100, 500], 128),
    ([-3, -500, -499], 500), ([510, 511, 512], 9), ([2 ** 31 - 1, -2 ** 31, 0], 600), ([640, 0, 5], 100000 // 100)])
def test_ranges(starts, T):
    # a full window of 128 waits in sequence 1 (decode rule), the others' windows are ragged
    c = filled_cache([512, 384, 500], steps=[(3, 128, 12)], hk=2, scattered=True, pages=6)
    check(c, starts, T, "bf16")


@pytest.mark.parametrize("kw", [dict(rotation=False), dict(scale=1), dict(scale=2), dict(scale=3, rotation=False), dict(norm_scope=1)])
def test_switches(kw):
    c = filled_cache([300, 200], **kw)
    check(c, [20, 100], 250, "f32")


def test_one_side_and_bad_pages():
    import torch
    c = filled_cache([600, 600], hk=2, pages=5)
    both = read(c, [5, 130], 500, "bf16")
    assert np.array_equal(read(c, [5, 130], 500, "bf16", "k")[0], both[0])
    assert np.array_equal(read(c, [5, 130], 500, "bf16", "v")[1], both[1])
    table = c.block_table.clone()
    full = numbers(c)
    c.block_table[0, 1], c.block_table[1, 3], c.block_table[1, 0] = -1, c.num_pages, 2 ** 31 - 1
    got = read(c, None, 600, "bf16")
    c.block_table.copy_(table)
    want = read(c, None, 600, "bf16")
    gone = np.zeros((2, 600), bool)
    gone[0, 128:256] = gone[1, 384:512] = gone[1, :128] = True
    for g, w in zip(got, want):
        assert (g[gone] == -77).all() and np.array_equal(g[~gone], w[~gone])
    assert len(full) == 2


def test_layer_views_streams_and_graphs():
    import torch
    from paper_2605_19660_amd import binding as ob
    cfg = ob.Config(4, 2)
    m = ob.MultiLayerCache(cfg, 2, 4, 3)
    k = torch.randn(3, 2, 300, 2, 128, device="cuda").bfloat16()
    for l in range(3):
        ob.quantize_append(m.layer(l), k[l], k[l].flip(0), eager=True)
    plain = ob.Cache(cfg, 2, 4)
    ob.quantize_append(plain, k[1], k[1].flip(0), eager=True)
    want = read(plain, [3, 40], 300, "bf16")
    assert all(np.array_equal(a, b) for a, b in zip(read(m.layer(1), [3, 40], 300, "bf16"), want))
    out_k, out_v = (torch.zeros(2, 64, 2, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    at = torch.tensor([0, 128], dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ob.cache_read(plain, at, k=out_k, v=out_v, stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.cache_read(plain, at, k=out_k, v=out_v)
    for step in range(3):
        at += 29
        e = [torch.zeros_like(out_k), torch.zeros_like(out_v)]
        ob.cache_read(plain, at, k=e[0], v=e[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(e[0], out_k) and torch.equal(e[1], out_v)
