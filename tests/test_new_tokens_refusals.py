"""Arguments that rope, cache_read, draft_attn and verify_drafts refuse, at the C ABI and in the binding, and
what their host-only helpers say (no GPU needed: nothing is enqueued when a check fails)."""
import ctypes as C

import pytest

from paper_2605_19660_amd import binding as ob

P = 1 << 20          # stands for a device pointer: 16-byte aligned, never read on the host


def rope(**kw):
    a = dict(q=P, k=P, q_out=P, k_out=P, n=4, hq=8, hk=2, qs=1024, ks=256, qos=1024, kos=256, pos=P, inv=P, axis=None,
             axes=1, rot=128, dt=ob.BF16, flags=0)
    a.update(kw)
    return ob.lib().oscar_rope(a["q"], a["k"], a["q_out"], a["k_out"], a["n"], a["hq"], a["hk"], a["qs"], a["ks"], a["qos"],
                               a["kos"], a["pos"], a["inv"], a["axis"], a["axes"], a["rot"], a["dt"], a["flags"], None)


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(hq=-1), dict(hk=-1), dict(axes=0), dict(axes=5), dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2),
    dict(dt=3), dict(dt=-1), dict(flags=4), dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(pos=None),
    dict(inv=None), dict(q=P + 2), dict(k_out=P + 8), dict(qs=1028), dict(kos=260), dict(qs=1016), dict(kos=128),
    dict(qs=-1024), dict(axes=2), dict(axis=bytes([0] * 63 + [1])), dict(axes=3, axis=bytes([3] + [0] * 63)), dict(hq=65537),
    dict(dt=ob.F32, qs=1026),
])
def test_rope_refuses(bad):
    assert rope(**bad) == ob.ERR_INVALID_ARG


def test_rope_with_nothing_to_do():
    assert rope(n=0) == ob.OK
    assert rope(hq=0, hk=0, q=None, k=None, q_out=None, k_out=None) == ob.OK
    assert rope(n=0, axes=4, axis=bytes([3] * 64)) == ob.OK


def test_axes_of_pairs():
    assert ob.rope_axes([2, 3]) == bytes([0, 0, 1, 1, 1])
    assert ob.rope_axes([3, 1, 2], interleaved=True) == bytes([0, 1, 2, 0, 2, 0])


def cache_struct(**kw):
    cfg = dict(n_q_heads=8, n_kv_heads=2)
    cfg.update({k: v for k, v in kw.items() if hasattr(ob.Config(1, 1), k)})
    c = ob.CCache()
    c.cfg = ob.Config(**cfg).c()
    c.batch, c.max_pages_per_seq, c.num_pages = kw.get("batch", 2), kw.get("max_pages", 4), kw.get("num_pages", 8)
    for name, t in ob.CCache._fields_:
        if t is C.c_void_p:
            setattr(c, name, None if kw.get("null") == name else P)
    return c


BAD_CACHE = [(dict(bits=3), ob.ERR_UNSUPPORTED), (dict(head_dim=64), ob.ERR_UNSUPPORTED), (dict(batch=0), ob.ERR_INVALID_ARG),
             (dict(max_pages=0), ob.ERR_INVALID_ARG), (dict(num_pages=0), ob.ERR_INVALID_ARG),
             (dict(n_q_heads=7), ob.ERR_INVALID_ARG)] + [
    (dict(null=n), ob.ERR_INVALID_ARG) for n in ("k_codes", "k_meta", "k_norms", "v_codes", "v_meta", "res_k", "res_v",
                                                 "res_norm", "block_table", "seq_lens", "res_lens")]


def read(c=None, starts=None, T=3, k=P, v=P, dt=ob.BF16):
    return ob.lib().oscar_cache_read(C.byref(c) if c is not None else None, starts, T, k, v, dt, None)


@pytest.mark.parametrize("bad,code", BAD_CACHE)
def test_cache_read_refuses_caches(bad, code):
    assert read(cache_struct(**bad)) == code


def test_cache_read_refuses():
    c = cache_struct()
    assert read(None) == ob.ERR_INVALID_ARG
    for kw in (dict(T=-1), dict(dt=3), dict(k=None, v=None), dict(k=P + 2), dict(v=P + 8)):
        assert read(c, **kw) == ob.ERR_INVALID_ARG, kw
    assert read(cache_struct(batch=65536)) == ob.ERR_INVALID_ARG
    assert read(c, T=0) == ob.OK


def draft(c, q=P, k=P, v=P, T=4, lens=None, out=P, hint=1000, splits=1, ws=None, wb=0):
    return ob.lib().oscar_draft_attn(q, k, v, T, lens, C.byref(c) if c is not None else None, out, 0.0, hint, splits, ws, wb, None)


@pytest.mark.parametrize("bad,code", BAD_CACHE + [(dict(io_dtype=ob.F32), ob.ERR_UNSUPPORTED)])
def test_draft_attn_refuses_caches(bad, code):
    assert draft(cache_struct(**bad)) == code


def test_draft_attn_refuses():
    c = cache_struct()
    assert draft(None) == ob.ERR_INVALID_ARG
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(T=-1), dict(hint=-1), dict(splits=-1),
               dict(splits=513), dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8), dict(T=1 << 30)):
        assert draft(c, **kw) == ob.ERR_INVALID_ARG, kw
    need = ob.draft_workspace_bytes(ob.Config(8, 2), 2, 4, 3)
    assert need == 2 * 4 * 8 * 3 * 130 * 4
    for kw in (dict(), dict(ws=P, wb=need - 1), dict(ws=P + 4, wb=need)):
        assert draft(c, splits=3, **kw) == ob.ERR_WORKSPACE, kw
    assert draft(c, T=0) == ob.OK


def test_draft_helpers():
    cfg = ob.Config(32, 8)
    assert ob.draft_workspace_bytes(cfg, 8, 4, 1) == 0                 # one split writes the output itself
    for batch, T, ctx in ((1, 1, 0), (1, 4, 1000), (8, 8, 32768), (64, 500, 100), (1, 5, 1 << 20)):
        s = ob.draft_auto_splits(cfg, batch, T, ctx)
        assert 1 <= s <= 512 and s <= (max(1, (ctx + 127) // 128) + 4 + (T + 31) // 32 + 3) // 4     # a piece of work a wave
    assert ob.draft_auto_splits(ob.Config(32, 8, io_dtype=ob.F32), 1, 4, 1000) == 1


def verify(p=P, q=P, drafts=P, lens=None, u=P, batch=2, T=3, vocab=1000, dt=ob.F32, n=P, tok=P, ws=P, wb=None):
    if wb is None:
        wb = ob.verify_workspace_bytes(batch, vocab)
    return ob.lib().oscar_verify_drafts(p, q, drafts, lens, u, batch, T, vocab, dt, n, tok, ws, wb, None)


def test_verify_drafts_refuses():
    for kw in (dict(p=None), dict(q=None), dict(drafts=None), dict(u=None), dict(n=None), dict(tok=None), dict(batch=-1),
               dict(batch=65536), dict(T=-1), dict(T=4097), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dt=3), dict(p=P + 2),
               dict(q=P + 1)):
        assert verify(**kw) == ob.ERR_INVALID_ARG, kw
    need = ob.verify_workspace_bytes(2, 1000)
    assert need > 0 and ob.verify_workspace_bytes(0, 10) == 0 and ob.verify_workspace_bytes(1, 0) == 0
    for kw in (dict(ws=None), dict(wb=need - 1), dict(ws=P + 8)):
        assert verify(**kw) == ob.ERR_WORKSPACE, kw
    assert verify(batch=0) == ob.OK


def test_host_tensors_are_refused(monkeypatch):
    import torch
    monkeypatch.setattr(ob, "_current_device", lambda: 0)
    x, i = torch.zeros(2, 3, 4, 128), torch.zeros(6, dtype=torch.int32)
    with pytest.raises(AssertionError, match="current device"):
        ob.rope(x, None, i, torch.ones(64))
    with pytest.raises(AssertionError, match="current device"):
        ob.verify_drafts(torch.rand(2, 4, 10), torch.rand(2, 3, 10), i.view(2, 3), torch.rand(2, 4))


def test_grids_past_what_a_launch_takes_are_refused():
    assert rope(n=4 * ((1 << 24) - 1) + 1, hk=0) == ob.ERR_INVALID_ARG
    assert draft(cache_struct(batch=65535, n_q_heads=128, n_kv_heads=128), splits=512, ws=P, wb=1 << 60) == ob.ERR_INVALID_ARG
    assert draft(cache_struct(batch=1, n_q_heads=8, n_kv_heads=1), T=1 << 22, splits=2, ws=P, wb=1 << 60) == ob.ERR_INVALID_ARG
