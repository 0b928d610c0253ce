"""oscar_draft_attn against attention in 64 bits over the cache's numbers: head layouts, formats, types, lengths of
nothing, one token, page and window edges, ragged new tokens, splits, odd rows, stale NaNs, other streams, graphs."""
import numpy as np
import pytest

from cache_numbers import filled_cache, hadamard, numbers, torch_type

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -11                       # half a step of fp16, relative
HALF_STEP = {"bf16": 2.0 ** -8, "f16": HALF}


def attention(c, q, k_new, v_new, new_lens, io, scale=None):
    """The output in 64 bits and how far the kernel's may be from it, per element.

    Roundings, each at most HALF of the number rounded and independent of the others: a query's channel once, its
    product with a key's step once, and the key's zero term once; a probability once, its product with a value's
    step once, and the value's zero term once.  (New tokens: the probability, and the value where bf16 has it
    below fp16's normal range.)  An error that is a sum of independent ones h_j each bounded in size stays within
    6 sqrt(sum h_j^2) but for 3e-8 of cases (Hoeffding's bound at 6: 2 exp(-18)); queries and steps are shared
    between tokens, so over tokens the errors are added up as they are.  The output is then rounded once."""
    H = hadamard()
    scale = scale or 1 / np.sqrt(128.0)
    B, T, hq, _ = q.shape
    hk = k_new.shape[2]
    g = hq // hk
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b, s in enumerate(numbers(c)):
        for h in range(hq):
            kv = h // g
            qr = q[b, :, h] @ H if c.cfg.rotation == 0 else q[b, :, h]
            n = s["n"][kv] * scale
            old = (qr @ (s["kc"][kv] + s["kb"][kv]).T) * n
            e_old = 6 * HALF * np.sqrt((qr ** 2) @ ((4 * s["kc"][kv] ** 2) + 4 * s["kb"][kv] ** 2).T) * n
            for t in range(T if new_lens is None else max(0, min(int(new_lens[b]), T))):
                new = (q[b, t, h] @ k_new[b, :t + 1, kv].T) * scale
                lg = np.concatenate([old[t], new])
                e = np.concatenate([e_old[t], np.zeros(t + 1)]) + 1e-5 * (1 + np.abs(lg))   # fp32 sums and exponentials
                p = np.exp(lg - lg.max())
                p /= p.sum()
                v = np.concatenate([s["vc"][kv] + s["vb"][kv], v_new[b, :t + 1, kv]])
                vc = np.concatenate([s["vc"][kv], v_new[b, :t + 1, kv]])
                vb = np.concatenate([s["vb"][kv], np.zeros((t + 1, 128))])
                o = p @ v
                out[b, t, h] = o
                d = (p * np.expm1(2 * e)) @ np.abs(v - o)
                d += 6 * HALF * np.sqrt((p ** 2) @ (4 * vc ** 2 + 4 * vb ** 2 + v ** 2)) + 2.0 ** -25 * (p.sum() + 1)
                d += 1e-5 * (p @ (np.abs(vc) + np.abs(vb)))
                tol[b, t, h] = d + (np.abs(o) + d) * HALF_STEP[io] + 2.0 ** -25
    return out, tol


def inputs(c, T, io, seed=1, qmul=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    B, hq, hk = c.batch, c.cfg.n_q_heads, c.cfg.n_kv_heads
    mk = lambda h, m: (torch.randn(B, T, h, 128, generator=g) * m).to(torch_type(io)).cuda()
    return mk(hq, qmul), mk(hk, 1.0), mk(hk, 1.0)


def check(c, T, io, new_lens=None, splits=0, scale=0.0, seed=1, qmul=1.0, hint=None):
    import torch
    from paper_2605_19660_amd import binding as ob
    q, k, v = inputs(c, T, io, seed, qmul)
    want, tol = attention(c, *(x.double().cpu().numpy() for x in (q, k, v)), new_lens, io, scale or None)
    lens = None
    if new_lens is not None:
        lens = torch.tensor(new_lens, dtype=torch.int32, device="cuda")
        for b, n in enumerate(new_lens):              # what lies behind the new tokens does not count
            q[b, max(n, 0):], k[b, max(n, 0):], v[b, max(n, 0):] = float("nan"), float("nan"), float("inf")
    hint = int(c.seq_lens.max()) if hint is None else hint
    got = ob.draft_attn(c, q, k, v, new_lens=lens, scale=scale, max_seq_len_hint=hint, num_splits=splits, out=torch.full_like(q, 55.0))
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.isfinite(err).all() and (err <= tol).all(), (err.max(), (err / np.maximum(tol, 1e-30)).max())
    again = ob.draft_attn(c, q, k, v, new_lens=lens, scale=scale, max_seq_len_hint=hint, num_splits=splits)
    assert torch.equal(got, again)
    return got, want


FORMATS = [(2, 128, 32, "bf16", "f16", False), (4, 128, 32, "f16", "f16", False), (2, 32, 64, "f16", "f16", True),
           (4, 64, 128, "bf16", "f32", False), (2, 64, 32, "bf16", "f32", True), (4, 32, 32, "f16", "f16", True),
           (2, 32, 128, "f16", "f32", False), (4, 128, 64, "bf16", "f16", True)]


@pytest.mark.parametrize("bits,kg,vg,io,meta,zp_min", FORMATS)
@pytest.mark.parametrize("T,splits", [(3, 1), (9, 0), (4, 3)])
def test_formats(bits, kg, vg, io, meta, zp_min, T, splits):
    c = filled_cache([700, 128, 1, 0, 383], hk=2, hq=8, bits=bits, kg=kg, vg=vg, io=io, meta=meta, zp_min=zp_min,
                     scattered=True, seed=bits * kg + vg)
    check(c, T, io, splits=splits)


@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (4, 2), (3, 1), (20, 4), (6, 1), (14, 2), (8, 1)])
@pytest.mark.parametrize("T", [1, 2, 5, 17])
def test_heads_and_tokens(hq, hk, T):
    check(filled_cache([300, 257], hk=hk, hq=hq), T, "bf16", new_lens=[T, max(T - 2, 0)])


@pytest.mark.parametrize("T", [31, 32, 33, 64, 65, 130])
@pytest.mark.parametrize("splits", [1, 2])
def test_many_new_tokens(T, splits):
    check(filled_cache([130, 40], hk=1, hq=4, io="f16"), T, "f16", new_lens=[T, T - 31], splits=splits)


@pytest.mark.parametrize("lens,steps", [
    ([0, 0], ()), ([1, 127], ()), ([128, 129], ()), ([256, 255], ((128, 1),)), ([383, 0], ((1, 128),)),
    ([0, 640], ((31, 128), (1, 0))), ([1279, 1290], ())])
@pytest.mark.parametrize("splits", [1, 4, 11])
def test_lengths(lens, steps, splits):
    check(filled_cache(lens, steps=steps, scattered=True), 4, "bf16", splits=splits)


def test_new_lens_of_every_size_and_none():
    c = filled_cache([200, 0, 129, 64, 300, 0], hq=4, hk=2)
    got, _ = check(c, 6, "bf16", new_lens=[0, 0, -4, 6, 9, 1])
    assert not got[:3].any() and bool(got[3].any()) and bool(got[4].any()) and not got[5, 1:].any()


@pytest.mark.parametrize("gain", [3e-4, 30.0, 3e3])
@pytest.mark.parametrize("io,meta", [("bf16", "f16"), ("f16", "f32")])
def test_value_sizes(gain, io, meta):
    """Value steps far below and above 2, where the probabilities' scale has to give way; in one sequence the large
    values come late, so that what is summed already has to be rescaled."""
    c = filled_cache([600, 1500], io=io, meta=meta, gain=gain, steps=((20, 100),))
    check(c, 3, io, splits=1)
    check(c, 3, io, splits=2)


@pytest.mark.parametrize("qmul,scale", [(12.0, 0.0), (1.0, 0.5), (0.01, 0.0), (1.0, 1e-3)])
def test_sharp_and_flat(qmul, scale):
    check(filled_cache([900, 131], hk=2, hq=8), 5, "bf16", qmul=qmul, scale=scale)


@pytest.mark.parametrize("kw", [dict(rotation=False), dict(scale=1), dict(scale=2), dict(scale=3, rotation=False), dict(norm_scope=1)])
def test_switches(kw):
    check(filled_cache([400, 200], **kw), 4, "bf16")


def test_what_later_new_tokens_hold_does_not_reach_earlier_rows():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([200], hq=4, hk=2)
    q, k, v = inputs(c, 5, "bf16")
    want = ob.draft_attn(c, q, k, v, num_splits=1)
    k[:, 3:], v[:, 3:], v[:, 4] = float("inf"), float("inf"), float("nan")
    assert torch.equal(ob.draft_attn(c, q, k, v, num_splits=1)[:, :3], want[:, :3])


def test_one_new_token_is_close_to_the_decode_step():
    """The same token appended first (its key then rounded to fp16 by norm and direction) and attended to by
    decode_attn: both within their tolerances of the same attention."""
    import torch
    from paper_2605_19660_amd import binding as ob
    a, b = (filled_cache([900, 140], hk=2, hq=8) for _ in range(2))
    q, k, v = inputs(a, 1, "bf16")
    got = ob.draft_attn(a, q, k, v, max_seq_len_hint=900).float()
    ob.quantize_append(b, k, v)
    want = ob.decode_attn(b, q[:, 0].contiguous(), max_seq_len_hint=901)
    assert float((got[:, 0] - want).norm() / want.norm()) <= 2.0 ** -8 + 1e-3 + 2.0 ** -9


def test_pages_that_are_none_are_left_out():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([640, 640], hk=2, hq=4, pages=6)
    q, k, v = inputs(c, 3, "bf16")
    c.block_table[0, 4], c.block_table[0, 3] = -1, c.num_pages
    got = ob.draft_attn(c, q, k, v, num_splits=2)
    c.seq_lens[0] = 384
    want = ob.draft_attn(c, q, k, v, num_splits=2)
    assert torch.allclose(got.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -9)


def test_streams_workspaces_and_graphs():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([1000, 900], hk=2, hq=8, pages=10)
    q, k, v = inputs(c, 4, "bf16")
    lens = torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    ws = torch.full((ob.draft_workspace_bytes(c.cfg, 2, 4, 3),), 255, dtype=torch.uint8, device="cuda")
    out, want = torch.zeros_like(q), ob.draft_attn(c, q, k, v, new_lens=lens, num_splits=3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ob.draft_attn(c, q, k, v, new_lens=lens, num_splits=3, out=out, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.draft_attn(c, q, k, v, new_lens=lens, num_splits=3, out=out, workspace=ws)
    for step in range(3):
        ob.quantize_append(c, k, v, new_lens=lens)
        q.mul_(0.9)
        want = ob.draft_attn(c, q, k, v, new_lens=lens, num_splits=3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
