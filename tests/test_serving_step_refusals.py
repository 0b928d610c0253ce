"""Arguments that plan_step, the calls of the 8-bit cache and sample refuse, at the C ABI and in the binding, and what
their host-only helpers say (no GPU needed: nothing is enqueued when a check fails)."""
import ctypes as C

import pytest

from paper_2605_19660_amd import binding as ob

P = 1 << 20          # stands for a device pointer: 16-byte aligned, never read on the host
BIG = 2 ** 31 - 1


def plan(**kw):
    a = dict(lens=P, keep=None, want=P, batch=4, table=P, max_pages=8, num_pages=32, ps=128, free=P, n_free=P, n_rows=10, lens_out=P,
             new_lens=P, n_free_out=P, row_starts=P, positions=P, row_seq=P, slots=P)
    a.update(kw)
    return ob.lib().oscar_plan_step(*[a[n] for n in ("lens", "keep", "want", "batch", "table", "max_pages", "num_pages", "ps", "free",
                                                     "n_free", "n_rows", "lens_out", "new_lens", "n_free_out", "row_starts", "positions",
                                                     "row_seq", "slots")], None)


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(batch=(1 << 20) + 1), dict(max_pages=0), dict(num_pages=0), dict(ps=0), dict(n_rows=-1), dict(lens=None),
    dict(want=None), dict(table=None), dict(free=None), dict(n_free=None), dict(lens_out=None), dict(new_lens=None), dict(n_free_out=None),
    dict(row_starts=None), dict(num_pages=1 << 24, ps=128), dict(max_pages=1 << 24), dict(ps=BIG, num_pages=2),
])
def test_plan_step_refuses(bad):
    assert plan(**bad) == ob.ERR_INVALID_ARG


def q8(**kw):
    c = ob.CQ8Cache(*[kw.get(n, d) for n, d in (("batch", 2), ("max_pages", 4), ("num_pages", 8), ("n_kv_heads", 2), ("head_dim", 128),
                                                ("page_size", 128), ("block", 32), ("io", ob.BF16))])
    for name in ("k_codes", "v_codes", "k_scales", "v_scales", "win_k", "win_v", "block_table"):
        setattr(c, name, kw.get(name, P))
    return c


BAD_SIZES = [(dict(batch=0), ob.ERR_INVALID_ARG), (dict(batch=65536), ob.ERR_INVALID_ARG), (dict(max_pages=0), ob.ERR_INVALID_ARG),
             (dict(max_pages=1 << 24), ob.ERR_INVALID_ARG), (dict(num_pages=0), ob.ERR_INVALID_ARG), (dict(num_pages=1 << 24), ob.ERR_INVALID_ARG),
             (dict(n_kv_heads=0), ob.ERR_INVALID_ARG), (dict(n_kv_heads=65536), ob.ERR_INVALID_ARG), (dict(head_dim=64), ob.ERR_UNSUPPORTED),
             (dict(head_dim=0), ob.ERR_INVALID_ARG), (dict(page_size=64), ob.ERR_UNSUPPORTED), (dict(block=16), ob.ERR_UNSUPPORTED),
             (dict(block=0), ob.ERR_INVALID_ARG), (dict(block=256), ob.ERR_UNSUPPORTED), (dict(io=ob.F32), ob.ERR_UNSUPPORTED),
             (dict(io=3), ob.ERR_INVALID_ARG)]
BAD_CACHE = BAD_SIZES + [({n: None}, ob.ERR_INVALID_ARG) for n in ("k_codes", "v_codes", "k_scales", "v_scales", "win_k", "win_v", "block_table")] + [
    ({n: P + 8}, ob.ERR_INVALID_ARG) for n in ("k_codes", "v_codes", "win_k", "win_v")]


def append(c, k=P, v=P, ks=256, vs=256, rows=8, T=4, starts=None, new=None, lens=P):
    return ob.lib().oscar_q8_append(k, v, ks, vs, rows, T, starts, new, lens, C.byref(c) if c is not None else None, None)


def attn(c, q=P, qs=1024, rows=8, hq=8, T=4, starts=None, new=None, lens=P, out=P, dt=ob.BF16, hint=1000, splits=1, ws=None, wb=0):
    return ob.lib().oscar_q8_attn(q, qs, rows, hq, T, starts, new, lens, C.byref(c) if c is not None else None, out, dt, 0.0, hint, splits,
                                  ws, wb, None)


def read(c, lens=P, starts=None, T=3, k=P, v=P, dt=ob.BF16):
    return ob.lib().oscar_q8_read(C.byref(c) if c is not None else None, lens, starts, T, k, v, dt, None)


@pytest.mark.parametrize("bad,code", BAD_CACHE)
def test_the_calls_refuse_caches(bad, code):
    c = q8(**bad)
    assert append(c) == code and attn(c) == code and read(c) == code


@pytest.mark.parametrize("bad,code", BAD_SIZES)
def test_sizes_refuse(bad, code):
    assert ob.lib().oscar_q8_sizes(C.byref(q8(**bad)), C.byref(ob.CQ8PoolSizes())) == code


def test_sizes():
    out = ob.CQ8PoolSizes()
    c = q8(k_codes=None, block_table=None, batch=3, num_pages=7, n_kv_heads=5, block=64)
    assert ob.lib().oscar_q8_sizes(C.byref(c), C.byref(out)) == ob.OK
    assert out.codes == 7 * 5 * 128 * 128 and out.scales == 7 * 5 * 2 * 4 and out.window == 3 * 5 * 2 * 64 * 128 * 2
    assert out.block_table == 3 * 4 * 4 and out.page_bytes_per_kv_head == 2 * (16384 + 8)
    assert ob.lib().oscar_q8_sizes(C.byref(c), None) == ob.ERR_INVALID_ARG
    assert ob.lib().oscar_q8_sizes(None, C.byref(out)) == ob.ERR_INVALID_ARG


def test_append_refuses():
    c = q8()
    assert append(None) == ob.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(rows=-1), dict(k=None), dict(v=None), dict(lens=None), dict(k=P + 8), dict(v=P + 2), dict(ks=248), dict(vs=260),
               dict(ks=-256), dict(T=BIG)):
        assert append(c, **kw) == ob.ERR_INVALID_ARG, kw
    assert append(c, T=0) == ob.OK and append(c, rows=0, k=None) == ob.OK


def test_attn_refuses():
    c = q8()
    assert attn(None) == ob.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(rows=-1), dict(q=None), dict(out=None), dict(lens=None), dict(q=P + 8), dict(out=P + 4), dict(qs=1016),
               dict(qs=1028), dict(hq=0), dict(hq=7), dict(dt=ob.F16), dict(dt=5), dict(hint=-1), dict(splits=-1), dict(splits=513), dict(T=BIG)):
        assert attn(c, **kw) == ob.ERR_INVALID_ARG, kw
    assert attn(c, hq=130, qs=130 * 128) == ob.ERR_UNSUPPORTED
    need = ob.lib().oscar_q8_workspace_bytes(C.byref(c), 8, 4, 3)
    assert need == 2 * 4 * 8 * 3 * 130 * 4
    for kw in (dict(), dict(ws=P, wb=need - 1), dict(ws=P + 8, wb=need)):
        assert attn(c, splits=3, **kw) == ob.ERR_WORKSPACE, kw
    assert attn(c, T=0) == ob.OK and attn(c, rows=0) == ob.OK


def test_read_refuses():
    c = q8()
    assert read(None) == ob.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(lens=None), dict(dt=3), dict(k=None, v=None), dict(k=P + 8), dict(v=P + 4), dict(T=BIG)):
        assert read(q8(n_kv_heads=128), **kw) == ob.ERR_INVALID_ARG, kw
    assert read(c, T=0) == ob.OK


def test_split_count():
    L = ob.lib()
    splits = lambda hq, T, n, **kw: L.oscar_q8_auto_splits(C.byref(q8(**kw)), hq, T, n)
    assert L.oscar_q8_workspace_bytes(C.byref(q8()), 8, 4, 1) == 0      # one split writes the output itself
    assert splits(8, 1, 0) == 1 and splits(7, 1, 1000) == 1 and splits(8, 0, 1000) == 1
    for batch, T, n in ((1, 1, 1000), (8, 1, 32768), (1, 5, 131072), (64, 1, 8192), (2, 500, 8192), (1, 1, BIG)):
        s = splits(32, T, n, batch=batch, n_kv_heads=8)
        assert 1 <= s <= min(512, (n + 127) // 128)


def test_split_count_of_the_longest_lengths():
    """Bounds up to 2^31 - 1 count as many splits as bounds a page below."""
    splits = lambda T, n: ob.lib().oscar_q8_auto_splits(C.byref(q8(batch=1, n_kv_heads=8)), 32, T, n)
    for T in (1, 5, 40):
        assert [splits(T, n) for n in (BIG, BIG - 126, BIG - 127)] == [splits(T, BIG - 255)] * 3 and splits(T, BIG) > 1


def sample(x=P, stride=1000, batch=2, vocab=1000, dt=ob.F32, temp=None, k=None, p=None, m=None, u=P, tokens=P, probs=None,
           ws=P, wb=None):
    wb = ob.sample_workspace_bytes(batch, vocab) if wb is None else wb
    return ob.lib().oscar_sample(x, stride, batch, vocab, dt, temp, k, p, m, u, tokens, probs, ws, wb, None)


def test_sample_refuses():
    for kw in (dict(x=None), dict(u=None), dict(tokens=None), dict(batch=-1), dict(vocab=0), dict(vocab=(1 << 22) + 1, stride=1 << 23), dict(dt=3), dict(dt=-1),
               dict(stride=999), dict(x=P + 2), dict(x=P + 1, dt=ob.BF16), dict(batch=65536)):
        assert sample(**kw) == ob.ERR_INVALID_ARG, kw
    need = ob.sample_workspace_bytes(2, 1000)
    assert need > 0 and ob.sample_workspace_bytes(0, 5) == 0 and ob.sample_workspace_bytes(1, 0) == 0
    for kw in (dict(ws=None), dict(ws=P + 8), dict(wb=need - 1)):
        assert sample(**kw) == ob.ERR_WORKSPACE, kw
    assert sample(batch=0, x=None) == ob.OK


def test_the_binding_checks_shapes_and_types():
    """What the binding asserts before it asks the library, on CPU tensors where the check comes first."""
    import torch
    cache = type("C", (), dict(batch=2, n_kv_heads=2, io_dtype=ob.BF16, block=32))()
    x = torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16)
    rows = ob._step_rows
    assert rows(cache, x, 2, None, None) == (6, 3, 256) and rows(cache, x[0], 2, x, 5) == (3, 5, 256)
    for bad in (lambda: rows(cache, x.float(), 2, None, None), lambda: rows(cache, x, 4, None, None), lambda: rows(cache, x[:1], 2, None, None),
                lambda: rows(cache, x, 2, None, 4), lambda: rows(cache, x[0], 2, x, None), lambda: rows(cache, x, 2, x, 3),
                lambda: rows(cache, x[:, :2, :, ::2], 2, None, None)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(ob.OscarError) as e:
        ob.q8_read(cache, None)
    assert e.value.status == ob.ERR_INVALID_ARG
