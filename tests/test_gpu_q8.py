"""oscar_q8_append and oscar_q8_read against the definition of the 8-bit cache: codes, scales and windows bit by bit, at
any cut of a sequence into calls."""
import numpy as np
import pytest

from q8_numbers import D, counted, dev, ints, packed_rows, padded_rows, scattered_cache, stands_for, tokens, torch_type

pytestmark = pytest.mark.gpu


def places():
    t, c = np.meshgrid(np.arange(128), np.arange(D), indexing="ij")
    k = ((t // 16 * 2 + c // 64) * 4 + c % 64 // 16) * 256 + t % 16 * 16 + c % 16
    v = (((t // 32 * 4 + c // 32) * 4 + t % 16 // 4) * 16 + c % 16) * 16 + c % 32 // 16 * 8 + t % 32 // 16 * 4 + t % 4
    return k, v


def append(ob, c, x, old, new, io, packed=False, T=None):
    """Appends tokens old[b] .. old[b] + new[b] - 1 of (keys, values) x to every sequence."""
    lens, T = np.asarray(old) + np.asarray(new), max(1, max(new)) if T is None else T
    if packed:
        (k, starts), (v, _) = (packed_rows(y, old, new, spare=2) for y in x)
        ob.q8_append(c, dev(k, io), dev(v, io), ints(lens), new_lens=ints(new), row_starts=ints(starts), max_new=T)
    else:
        k, v = (dev(padded_rows(y, old, new, T), io) for y in x)
        ob.q8_append(c, k, v, ints(lens), new_lens=None if all(n == T for n in new) else ints(new))


def check(ob, c, x, lens, io):
    """Pages, scales and window as the definition has them; and everything else as it was (no number)."""
    import torch
    block, H = c.block, c.n_kv_heads
    table = c.block_table.cpu().numpy()
    for y, codes, scales, win, place in zip(x, (c.k_codes, c.v_codes), (c.k_scales, c.v_scales), (c.win_k, c.win_v), places()):
        value = codes.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)
        scale, win = scales.double().cpu().numpy(), win.double().cpu().numpy()
        untouched = np.ones(value.shape[0], bool)
        for b, n in enumerate(lens):
            done = n // block * block
            for h in range(H):
                want, s = stands_for(y[b, :n, h], block, io)
                for t in range(0, done, block):
                    page, at = table[b, t // 128], t % 128
                    untouched[page] = False
                    assert scale[page, h, at // block] == s[t // block]
                    assert np.array_equal(value[page, h][place[at:at + block]] * s[t // block], want[t:t + block])
                late = np.arange(max(done - block, 0), n)
                assert np.array_equal(win[b, h, late % (2 * block)], counted(y[b, late, h], io))
        assert np.isnan(value[untouched]).all() and np.isnan(scale[untouched]).all()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("io,block", [("bf16", 32), ("f16", 32), ("bf16", 64), ("f16", 128), ("bf16", 128)])
def test_appends_of_any_cut_hold_what_the_definition_says(io, block, packed):
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(block + packed)
    lens = [700, 128, 0, 259]
    x = [tokens(rng, 4, 701, 3, io, wild=True) for _ in "kv"]
    for cuts in ([[1.0] * 4], [[0.37] * 4, [0.0, 0.5, 0.0, 0.5], [0.999, 0.7, 0.0, 0.9], [1.0] * 4], None):
        c = scattered_cache(ob, 3, 4, 6, block, io, rng)
        old = [0] * 4
        if cuts is None:     # single tokens and pieces around a block's length
            while old != lens:
                new = [min(n - o, int(rng.choice([0, 1, 1, block - 1, block, block + 1, 2 * block + 3]))) for o, n in zip(old, lens)]
                append(ob, c, x, old, new, io, packed)
                old = [o + n for o, n in zip(old, new)]
        else:
            for cut in cuts:
                to = [max(o, int(n * f)) for o, n, f in zip(old, lens, cut)]
                append(ob, c, x, old, [t - o for o, t in zip(old, to)], io, packed)
                old = to
        check(ob, c, x, lens, io)


@pytest.mark.parametrize("block", [32, 64, 128])
def test_every_length_of_two_appends(block):
    """All residues of the first append, and second ones across none, one and several block ends."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(block)
    B = block + 1
    x = [tokens(rng, B, 6 * block, 1, "bf16") for _ in "kv"]
    first = list(range(B))
    for add in (1, block // 2, block, block + 1, 2 * block, 3 * block + 1, 4 * block):
        c = scattered_cache(ob, 1, B, 6 * block // 128 + 1, block, "bf16", rng)
        append(ob, c, x, [0] * B, first, "bf16")
        append(ob, c, x, first, [add] * B, "bf16", packed=add % 2 == 1)
        check(ob, c, x, [n + add for n in first], "bf16")


@pytest.mark.parametrize("io", ["bf16", "f16"])
def test_what_is_no_number(io):
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(3)
    x = [tokens(rng, 2, 100, 2, io) for _ in "kv"]
    for y in x:
        y[0, 3, 0, 5], y[0, 40, 1, 7], y[0, 70, 0, 9], y[0, 99, 1, 127] = np.nan, np.inf, -np.inf, np.nan
        y[1, 10, 0, :] = np.nan
        if io == "bf16":
            y[1, 50, 1, 0] = 2.0 ** 100
            y[1, 64:96, 1] = 2.0 ** -120
    c = scattered_cache(ob, 2, 2, 1, 32, io, rng)
    append(ob, c, x, [0, 0], [90, 97], io)
    append(ob, c, x, [90, 97], [10, 1], io)
    check(ob, c, x, [100, 98], io)


def test_lengths_taken_back_and_gone_on_from():
    """Tokens that do not stand: the next append says a smaller length, and its tokens take their places; up to a whole
    block back, over a block that was coded already."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(5)
    for block in (32, 128):
        for back in (1, block // 2, block):
            for start in (block - 1, block, 2 * block + 5, 3 * block):
                keep = start + block + 7 - back     # the length that stands
                x = [tokens(rng, 1, 6 * block, 2, "bf16") for _ in "kv"]
                c = scattered_cache(ob, 2, 1, 8, block, "bf16", rng)
                append(ob, c, x, [0], [start], "bf16")
                append(ob, c, x, [start], [block + 7], "bf16")
                for y in x:                          # other tokens come instead
                    y[:, keep:] = tokens(rng, 1, 6 * block - keep, 2, "bf16")
                for n in (1, 3, block, 5):
                    append(ob, c, x, [keep], [n], "bf16")
                    keep += n
                check(ob, c, x, [keep], "bf16")


def test_rows_of_any_stride_beside_each_other():
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(8)
    B, T, H = 2, 70, 2
    x = [tokens(rng, B, T, H, "bf16") for _ in "kv"]
    m = torch.full((B * T, 8 + (4 + 2 * H) * D + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    k, v = (m[:, 8 + (4 + i * H) * D:8 + (4 + (i + 1) * H) * D].view(B, T, H, D) for i in (0, 1))
    k.copy_(dev(x[0], "bf16")), v.copy_(dev(x[1], "bf16"))
    c = scattered_cache(ob, H, B, 1, 64, "bf16", rng)
    ob.q8_append(c, k, v, ints([T] * B))
    check(ob, c, x, [T] * B, "bf16")


def test_rows_that_are_not_there_and_pages_that_are_none():
    """Tokens in pages that are no page are dropped, rows past n_rows are not read, everything around stays."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(9)
    x = [tokens(rng, 2, 400, 2, "bf16") for _ in "kv"]
    c = scattered_cache(ob, 2, 2, 3, 32, "bf16", rng)
    c.block_table[0, 1], c.block_table[1, 0], c.block_table[1, 2] = -1, 9, 2 ** 31 - 1
    keep = c.block_table.cpu().numpy().copy()
    append(ob, c, x, [0, 0], [400, 384], "bf16")     # (400: past the table's end)
    assert np.array_equal(c.block_table.cpu().numpy(), keep)
    value = c.k_codes.view(torch.float8_e4m3fn).float()
    written = ~torch.isnan(value).flatten(1).all(1)
    assert sorted(written.nonzero().flatten().tolist()) == sorted([keep[0, 0], keep[0, 2], keep[1, 1]])
    k = torch.full((2, 400, 2, D), 7.0, device="cuda")
    ob.q8_read(c, ints([400, 384]), k=k)
    got = k.cpu().numpy()
    for b in range(2):
        want = np.full((400, 2, D), 7.0)
        for h in range(2):
            y, _ = stands_for(x[0][b, :[400, 384][b], h], 32, "bf16")
            want[:len(y), h] = y
        for p in range(4):
            if p == 3 or not 0 <= keep[b, p] < c.num_pages:
                want[p * 128:min((p + 1) * 128, [384, 384][b])] = 7.0
        assert np.array_equal(got[b], want), b
    # rows that do not exist
    c = scattered_cache(ob, 2, 2, 2, 32, "bf16", rng)
    k, v = (dev(y[:, :40].reshape(80, 2, D), "bf16") for y in x)
    ob.q8_append(c, k, v, ints([40, 40]), new_lens=ints([40, 40]), row_starts=ints([70, -3]), max_new=40)
    assert np.array_equal(c.win_k[0, 0, 32:34].double().cpu().numpy(), np.zeros((2, D)))


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("io,block", [("bf16", 32), ("f16", 64), ("f16", 128)])
def test_read(io, block, out):
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(11)
    B, H, lens = 5, 3, [500, 1, 129, 0, 383]
    x = [tokens(rng, B, 500, H, io, wild=io == "bf16") for _ in "kv"]
    c = scattered_cache(ob, H, B, 4, block, io, rng)
    append(ob, c, x, [0] * B, lens, io)
    for T, starts in ((500, None), (1, [499, 0, 128, 0, 5]), (77, [40, -3, 100, 0, 350]), (33, [-50, -32, 31, 32, 33]), (600, [1, 2, 3, 4, 2 ** 31 - 1])):
        k, v = (torch.full((B, T, H, D), 3.0, dtype=torch_type(out), device="cuda") for _ in "kv")
        ob.q8_read(c, ints(lens), starts=None if starts is None else ints(starts), k=k, v=v)
        for y, got in zip(x, (k, v)):
            want = torch.full((B, T, H, D), 3.0, dtype=torch.float64)
            for b, n in enumerate(lens):
                s = 0 if starts is None else starts[b]
                for h in range(H):
                    z = torch.from_numpy(stands_for(y[b, :n, h], block, io)[0])
                    for i in range(max(s, 0), min(n, s + T)):
                        want[b, i - s, h] = z[i]
            assert torch.equal(got.cpu(), want.to(torch_type(out)))
        only = torch.full((B, T, H, D), 3.0, dtype=torch_type(out), device="cuda")
        ob.q8_read(c, ints(lens), starts=None if starts is None else ints(starts), v=only)
        assert torch.equal(only, v)


def test_a_pool_past_4_gib():
    """Pages whose codes lie past 2^32 bytes."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(13)
    H, pages = 8, 2 ** 32 // (8 * 16384) + 5
    x = [tokens(rng, 1, 300, H, "bf16") for _ in "kv"]
    c = ob.Q8Cache(H, 1, 3, num_pages=pages, block_table=ints([[pages - 1, 0, pages - 2]]))
    append(ob, c, x, [0], [300], "bf16")
    k, v = (torch.zeros(1, 300, H, D, device="cuda") for _ in "kv")
    ob.q8_read(c, ints([300]), k=k, v=v)
    for y, got in zip(x, (k, v)):
        for h in range(H):
            assert np.array_equal(got[0, :, h].double().cpu().numpy(), stands_for(y[0, :, h], 32, "bf16")[0])
    assert bool(c.k_codes[1:pages - 2].any()) is False and bool(c.v_codes[1:pages - 2].any()) is False


def test_the_largest_fp16_numbers_come_back_finite():
    """A block of an fp16 cache with numbers from 63488 on holds 65536 for them, which is no fp16 number: read as fp16 they are
    65504, as bf16 and fp32 what the codes say; infinities the same way."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(21)
    x = [tokens(rng, 2, 70, 2, "f16") for _ in "kv"]
    for y in x:
        y[0, :, 0, ::5] = rng.choice([65504.0, -65504.0, 63488.0, -63488.0, 63456.0, -63456.0, 61440.0], size=y[0, :, 0, ::5].shape)
        y[1, [3, 40, 66], 1, 9], y[1, [4, 50, 67], 1, 10] = np.inf, -np.inf
    c = scattered_cache(ob, 2, 2, 1, 32, "f16", rng)
    append(ob, c, x, [0, 0], [70, 68], "f16")
    check(ob, c, x, [70, 68], "f16")
    for out in ("f16", "bf16", "f32"):
        k, v = (torch.full((2, 70, 2, D), 3.0, dtype=torch_type(out), device="cuda") for _ in "kv")
        ob.q8_read(c, ints([70, 68]), k=k, v=v)
        for y, got in zip(x, (k, v)):
            want = np.full((2, 70, 2, D), 3.0)
            for b, n in enumerate([70, 68]):
                for h in range(2):
                    want[b, :n, h] = stands_for(y[b, :n, h], 32, "f16")[0]
            assert (np.abs(want) == 65536.0).any() and (np.abs(want) == 65504.0).any()
            if out == "f16":
                want = np.clip(want, -65504.0, 65504.0)
            assert torch.equal(got.cpu(), torch.from_numpy(want).to(torch_type(out))), out


@pytest.mark.parametrize("block", [32, 64, 128])
def test_lengths_taken_back_again_and_again(block):
    """Lengths that go back and forth as far as the cache allows: to f and above, f = n / block * block - block of the
    longest append that ended at n, or to a multiple of block below, which f is then.  After every change what is read is
    what a cache of that length holds."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(100 + block)
    B, H, most = 6, 2, 7 * block
    x = [tokens(rng, B, most, H, "bf16") for _ in "kv"]
    c = scattered_cache(ob, H, B, most // 128 + 1, block, "bf16", rng)
    n, f = np.zeros(B, int), np.zeros(B, int)

    def holds():
        k, v = (torch.zeros(B, most, H, D, device="cuda") for _ in "kv")
        ob.q8_read(c, ints(n), k=k, v=v)
        for y, got in zip(x, (k, v)):
            got = got.double().cpu().numpy()
            for b in range(B):
                for h in range(H):
                    assert np.array_equal(got[b, :n[b], h], stands_for(y[b, :n[b], h], block, "bf16")[0]), (b, n[b], f[b])

    for i in range(60):
        new = np.array([min(most - n[b], int(rng.choice([0, 1, 2, 7, block // 2, block, block + 3, 3 * block]))) for b in range(B)])
        append(ob, c, x, n, new, "bf16", packed=i % 2 == 1)
        n += new
        f = np.maximum(f, np.where(new > 0, n // block * block - block, 0))
        holds()
        for b in range(B):
            r = rng.random()
            if r < 0.2:
                n[b] = f[b] = int(rng.integers(0, f[b] // block + 1)) * block     # a multiple of block, below f or f
            elif r < 0.7:
                n[b] = int(rng.choice([f[b], rng.integers(f[b], n[b] + 1)]))
            for y in x:                                                          # other tokens come instead
                y[b, n[b]:] = tokens(rng, 1, most, H, "bf16")[0, n[b]:]
        holds()
