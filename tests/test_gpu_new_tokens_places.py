"""rope, cache_read, draft_attn and verify_drafts where their memory is unusual: far into large pools and tensors
(byte offsets past 32 bits), made on a stream that is not the current one, or not on the current device."""
import pytest

from cache_numbers import filled_cache

pytestmark = pytest.mark.gpu


def far_copy(c, pages, at):
    """The same cache with its pages at `at`, `at` + 1, .. of a pool of `pages`."""
    import torch
    from paper_2605_19660_amd import binding as ob
    far = ob.Cache(c.cfg, c.batch, c.c.max_pages_per_seq, num_pages=pages)
    for name in ("k_codes", "k_meta", "k_norms", "v_codes", "v_meta"):
        src, dst = getattr(c, name), getattr(far, name)
        dst.view(torch.uint8).view(pages, -1)[at:at + c.num_pages] = src.view(torch.uint8).view(c.num_pages, -1)
    for name in ("res_k", "res_v", "res_norm", "seq_lens", "res_lens"):
        getattr(far, name).copy_(getattr(c, name))
    far.block_table.copy_(c.block_table + at)
    return far


def test_pages_past_4_gib():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([700, 300], hk=8, hq=32, bits=4, scattered=True)
    far = far_copy(c, 66000, 65700)      # 64 KB of codes a page, of keys and of values
    assert far.k_codes.numel() * far.k_codes.element_size() > 1 << 32
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(2, 5, h, 128, generator=g).bfloat16().cuda() for h in (32, 8, 8))
    for splits in (1, 3):
        assert torch.equal(ob.draft_attn(far, q, k, v, num_splits=splits), ob.draft_attn(c, q, k, v, num_splits=splits))
    new = lambda: [torch.zeros(2, 700, 8, 128, device="cuda") for _ in range(2)]
    for a, b in zip(ob.cache_read(far, None, *new()), ob.cache_read(c, None, *new())):
        assert torch.equal(a, b) and float(a.abs().sum()) > 0


def test_read_into_rows_past_4_gib():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([700, 300], hk=8, hq=8)
    T = 600_000
    k = torch.zeros(2, T, 8, 128, device="cuda")
    starts = torch.tensor([10, 200 - T], dtype=torch.int32, device="cuda")
    ob.cache_read(c, starts, k=k)
    want = torch.zeros(2, 700, 8, 128, device="cuda")
    ob.cache_read(c, None, k=want)
    assert torch.equal(k[0, :690], want[0, 10:]) and torch.equal(k[1, T - 200:], want[1, :200])
    assert not k[0, 690:].any() and not k[1, :T - 200].any()


def test_rope_of_tokens_past_4_gib():
    import torch
    from paper_2605_19660_amd import binding as ob
    g = torch.Generator().manual_seed(2)
    x = torch.randn(3, 4, 128, generator=g).bfloat16().cuda()
    pos, inv = torch.tensor([7, 1 << 30, -5], dtype=torch.int32, device="cuda"), torch.rand(64, generator=g).cuda()
    room = torch.empty((1 << 32) + 512, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided((3, 4, 128), (1 << 31, 128, 1))
    far.copy_(x)
    ob.rope(far, None, pos, inv, out_q=far)
    assert torch.equal(far, ob.rope(x, None, pos, inv)[0])


def test_rows_of_probabilities_past_4_gib():
    import torch
    from paper_2605_19660_amd import binding as ob
    B, T, V = 4200, 1, (1 << 19) + 3
    p, q = (torch.zeros(B, t, V, dtype=torch.bfloat16, device="cuda") for t in (T + 1, T))
    drafts = torch.full((B, T), 17, dtype=torch.int32, device="cuda")
    u = torch.full((B, T + 1), 0.5, device="cuda")
    p[B - 1, 0, 17], q[B - 1, 0, 17], p[B - 1, 1, V - 1] = 0.5, 0.5, 1.0
    p[B - 2, 0, V - 2] = 1.0
    n, tokens = (x.cpu() for x in ob.verify_drafts(p, q, drafts, u))
    assert n[-1] == 2 and tokens[-1].tolist() == [17, V - 1] and n[-2] == 1 and tokens[-2].tolist() == [V - 2, -1]
    assert (n[:-2] == 1).all() and (tokens[:-2] == torch.tensor([0, -1])).all()


def calls():
    """name, call(stream) -> result made by the call"""
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([700, 300], hk=2, hq=8)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(2, 40, h, 128, generator=g).bfloat16().cuda() for h in (8, 2, 2))
    pos, inv = torch.arange(80, dtype=torch.int32, device="cuda"), torch.rand(64, generator=g).cuda()
    p, d = (torch.rand(2, t, 5000, generator=g).cuda() for t in (4, 3))
    x, u = torch.randint(0, 5000, (2, 3), generator=g).int().cuda(), torch.rand(2, 4, generator=g).cuda()
    outs = [torch.zeros_like(k) for _ in range(2)]
    return [("rope", lambda **kw: ob.rope(q, k, pos, inv, **kw)),
            ("draft_attn", lambda **kw: (ob.draft_attn(c, q, k, v, num_splits=3, **kw),)),
            ("verify_drafts", lambda **kw: ob.verify_drafts(p, d, x, u, **kw)),
            ("cache_read", lambda **kw: ob.cache_read(c, None, *outs, **kw))]


def test_what_a_call_makes_belongs_to_its_stream():
    """Blocks that the current stream gave back, with its writes to them still to come, are not handed to a call on
    another stream."""
    import torch
    s = torch.cuda.Stream()
    for name, call in calls():
        print(name, flush=True)
        if name == "cache_read":
            continue              # makes nothing
        want = [x.clone() for x in call()]
        torch.cuda.synchronize()
        given_back = [torch.empty_like(x) for _ in range(8) for x in want]
        torch.cuda._sleep(20_000_000)
        for x in given_back:
            x.fill_(9)
        del given_back, x
        got = call(stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


def test_tensors_of_another_device_are_refused(monkeypatch):
    from paper_2605_19660_amd import binding as ob
    for name, call in calls():
        call()
        with monkeypatch.context() as m:
            m.setattr(ob, "_current_device", lambda: 1)
            with pytest.raises(AssertionError, match="current device"):
                call()


def test_one_layer_of_many():
    """A layer behind a shared block table answers as a cache of its own does."""
    import torch
    from paper_2605_19660_amd import binding as ob
    cfg = ob.Config(8, 2)
    m, plain = ob.MultiLayerCache(cfg, 2, 4, 3), ob.Cache(cfg, 2, 4)
    g = torch.Generator().manual_seed(4)
    k = torch.randn(3, 2, 300, 2, 128, generator=g).bfloat16().cuda()
    for l in range(3):
        ob.quantize_append(m.layer(l), k[l], k[l].flip(0), eager=True)
    ob.quantize_append(plain, k[1], k[1].flip(0), eager=True)
    q, kn, vn = (torch.randn(2, 5, h, 128, generator=g).bfloat16().cuda() for h in (8, 2, 2))
    for splits in (1, 2):
        assert torch.equal(ob.draft_attn(m.layer(1), q, kn, vn, num_splits=splits), ob.draft_attn(plain, q, kn, vn, num_splits=splits))


def test_nothing_to_do():
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([140], hk=2, hq=8)
    empty = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    assert ob.draft_attn(c, empty(1, 0, 8, 128), empty(1, 0, 2, 128), empty(1, 0, 2, 128)).shape == (1, 0, 8, 128)
    assert ob.cache_read(c, None, k=empty(1, 0, 2, 128))[0].shape == (1, 0, 2, 128)
    pos, inv = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    assert ob.rope(empty(0, 8, 128), None, pos, inv)[0].shape == (0, 8, 128)
    n, tokens = ob.verify_drafts(torch.empty(0, 4, 10, device="cuda"), torch.empty(0, 3, 10, device="cuda"),
                                 torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda"))
    assert n.shape == (0,) and tokens.shape == (0, 4)


@pytest.mark.parametrize("bits,heads", [(2, 3), (4, 1)])
def test_a_long_piece_attends_to_itself(bits, heads):
    """Many blocks of rows, the last of 16 rows and fewer, over a short cache: against the short call's rows, whose
    causal past is the same."""
    import torch
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([150], hk=1, hq=heads, bits=bits)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(1, 1500, h, 128, generator=g).bfloat16().cuda() for h in (heads, 1, 1))
    got = ob.draft_attn(c, q, k, v, num_splits=1)
    for n in (7, 40, 333, 1024):
        part = ob.draft_attn(c, q[:, :n].contiguous(), k[:, :n].contiguous(), v[:, :n].contiguous(), num_splits=1)
        # the same sums; which rows share a tile decides when its reference moves (whole powers of two, fp16 operands:
        # 2^-11 of each probability), and the outputs are rounded to bf16
        err = (got[:, :n].double() - part.double()).abs()
        assert bool((err <= 2.0 ** -8 * part.double().abs() + 2.0 ** -10 * float(v.abs().max())).all())
