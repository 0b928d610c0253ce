"""oscar_q8_attn against attention in 64 bits over what the definition says the cache holds."""
import numpy as np
import pytest

from q8_numbers import D, dev, ints, packed_rows, padded_rows, scattered_cache, stands_for, tokens, torch_type
from test_gpu_q8 import append

pytestmark = pytest.mark.gpu


def attention(q, x, lens, new, block, io, out, scale=0.0, left_out=None):
    """Per sequence: outputs of its new tokens in 64 bits and how far off a result may be.

    With p_j the softmax of the true logits s_j: a computed weight is p_j (1 + d_j), which moves the output by at most
    2 max|d| sum p_j |v_j| (numerator and sum).  d: a logit adds 128 exact products in fp32, at worst one after
    the other, 2^-24 a step of their absolute sum (128 of them), and is multiplied by the scale, multiplied out and
    subtracted from the reference (4 more); 2^-22 of the exponential; 2^-17 of the two limbs.  Sums over n tokens in
    fp32: 32 to a matrix product that adds them and then its result to the sum, 64 steps for the joins."""
    # half a step of the output's type relative to the value (8 and 11 significant bits), behind one of fp32
    half = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[out] + 2.0 ** -24
    tiny = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}[out]
    result = []
    hq, hk = q.shape[2], x[0].shape[2]
    g, c = hq // hk, scale or 1 / np.sqrt(D)
    for b, (n, m) in enumerate(zip(lens, new)):
        o, tol = np.zeros((m, hq, D)), np.zeros((m, hq, D))
        k, v = ([stands_for(y[b, :n, h], block, io)[0] for h in range(hk)] for y in x)
        is_there = np.ones(n, bool)
        for p in (left_out or {}).get(b, ()):
            is_there[p * 128:(p + 1) * 128] = np.arange(n)[p * 128:(p + 1) * 128] >= n // block * block
        for t in range(m):
            see = np.nonzero(is_there[:n - m + t + 1])[0]
            if len(see) == 0:
                continue
            for h in range(hq):
                kk, vv = k[h // g][see], v[h // g][see]
                s = c * (kk @ q[b, t, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                o[t, h] = p @ vv
                size = c * (np.abs(kk) @ np.abs(q[b, t, h]))
                d = (132 * 2.0 ** -24) * size[p > 1e-9].max() + 2.0 ** -22 + 2.0 ** -17 + (len(see) * 33 / 32 + 64) * 2.0 ** -24
                tol[t, h] = 2 * d * (p @ np.abs(vv)) + half * np.abs(o[t, h]) + tiny + 1e-9 * np.abs(vv).max()
        result.append((o, tol))
    return result


def run(ob, c, q, lens, new, io, out, packed=False, stride=0, fill=7.0, **kw):
    """Outputs by sequence; what no sequence owns has to stay."""
    import torch
    T = max(1, max(new))
    if packed:
        rows, starts = packed_rows(q, [0] * len(new), new, spare=3)
    else:
        rows, starts = padded_rows(q, [0] * len(new), new, T), None
    r = dev(rows, io)
    if stride:
        wide = torch.full((r.shape[0] * (1 if packed else r.shape[1]), r.shape[-2] * D + stride), float("nan"), dtype=r.dtype, device="cuda")
        wide = wide[:, :r.shape[-2] * D].view(*r.shape)
        wide.copy_(r)
        r = wide
    o = torch.full(rows.shape, fill, dtype=torch_type(out), device="cuda")
    got = ob.q8_attn(c, r, ints(lens), new_lens=None if not packed and all(n == T for n in new) else ints(new),
                     row_starts=None if starts is None else ints(starts), max_new=T, out=o, **kw)
    assert got is o
    o = o.double().cpu().numpy()
    parts = [o[starts[b]:starts[b] + n] if packed else o[b, :n] for b, n in enumerate(new)]
    rest = o[starts[-1]:] if packed else np.concatenate([o[b, n:] for b, n in enumerate(new)])
    assert (rest == fill).all()
    return parts


def compare(got, want):
    for b, (y, (o, tol)) in enumerate(zip(got, want)):
        assert np.isfinite(y).all(), b
        off = np.abs(y - o) - tol
        assert (off <= 0).all(), (b, float(off.max()), float(np.abs(y - o).max()))


CASES = [
    # lens, new, (q heads, kv heads), block, io, out
    ([1, 2, 31, 32, 33, 127, 128, 129], [1] * 8, (8, 2), 32, "bf16", "bf16"),
    ([1, 64, 127, 128, 200, 255, 256, 383], [1] * 8, (8, 2), 128, "f16", "f16"),
    ([1000, 64, 513, 95], [1] * 4, (7, 1), 32, "bf16", "f32"),
    ([1000, 64, 513, 95], [1] * 4, (28, 4), 64, "f16", "f32"),
    ([700, 5, 40, 0, 33], [5, 5, 0, 0, 3], (8, 2), 32, "bf16", "bf16"),
    ([300, 65, 40], [64, 65, 1], (4, 4), 64, "bf16", "f32"),
    ([300, 129, 40], [130 - 1, 129, 9], (12, 2), 32, "f16", "f16"),
    ([260, 70], [70, 70], (20, 4), 128, "bf16", "bf16"),
    ([150], [33], (32, 1), 32, "bf16", "f32"),
    ([90], [2], (64, 1), 32, "f16", "f16"),
    ([200, 100], [100, 100], (1, 1), 64, "f16", "f32"),
    ([2049], [1], (3, 3), 32, "bf16", "f32"),
    # 17 .. 32 rows, a workgroup each
    ([300, 17, 129, 6], [6, 6, 2, 6], (8, 2), 32, "f16", "f32"),
    ([515, 260], [2, 2], (32, 2), 64, "f16", "f16"),
    ([1030, 31], [9, 9], (9, 3), 128, "bf16", "bf16"),
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lens,new,heads,block,io,out", CASES)
def test_against_64_bits(lens, new, heads, block, io, out, packed):
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(len(lens) + sum(lens) + packed)
    B, S = len(lens), max(lens)
    x = [tokens(rng, B, S, heads[1], io) for _ in "kv"]
    q = tokens(rng, B, max(1, max(new)), heads[0], io)
    c = scattered_cache(ob, heads[1], B, S // 128 + 2, block, io, rng)
    append(ob, c, x, [0] * B, lens, io)
    want = attention(q, x, lens, new, block, io, out)
    for splits in (0, 1, 2, 5):
        compare(run(ob, c, q, lens, new, io, out, packed, num_splits=splits, max_seq_len_hint=S), want)


@pytest.mark.parametrize("io", ["bf16", "f16"])
def test_values_of_all_sizes_beside_a_token_that_takes_the_softmax(io):
    """A key that answers the query takes nearly all of the softmax, with values of 0 there: what is left is
    the others', however small their weights and scales are; blocks' scales lie far apart."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(2)
    lens, new = [290, 290], [1, 2]
    x = [tokens(rng, 2, 290, 1, io) for _ in "kv"]
    q = tokens(rng, 2, 2, 4, io)
    for b, at in ((0, 17), (1, 280)):     # in a page, and in the window
        x[0][b, :, 0] = 0.01 * rng.integers(-3, 4, size=(290, D))
        x[0][b, at, 0] = 4.0 * np.sign(q[b, 0, 0])
        x[1][b, 32:64] *= 2.0 ** -10
        x[1][b, 64:96] *= 2.0 ** (6 if io == "f16" else 30)
        x[1][b, at] = 0.0
    x = [dev(y, io).double().cpu().numpy() for y in x]
    c = scattered_cache(ob, 1, 2, 3, 32, io, rng)
    append(ob, c, x, [0, 0], lens, io)
    for out in ("f32", io):
        want = attention(q, x, lens, new, 32, io, out)
        for splits in (1, 3):
            compare(run(ob, c, q, lens, new, io, out, num_splits=splits), want)


@pytest.mark.parametrize("order", ["rising", "falling", "far"])
def test_logits_that_move_the_reference(order):
    """Logits of hundreds, so that the running reference moves often or every later token vanishes."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(4)
    n = 700
    x = [tokens(rng, 1, n, 1, "bf16") for _ in "kv"]
    q = np.ones((1, 3, 2, D))
    q[:, :, 1] = -1.0
    level = {"rising": np.linspace(-30, 30, n), "falling": np.linspace(30, -30, n), "far": np.where(np.arange(n) == 333, 60.0, 0.0)}[order]
    x[0][0, :, 0] = 0.2 * x[0][0, :, 0] + level[:, None]
    x = [dev(y, "bf16").double().cpu().numpy() for y in x]
    c = scattered_cache(ob, 1, 1, 6, 32, "bf16", rng)
    append(ob, c, x, [0], [n], "bf16")
    want = attention(q, x, [n], [3], 32, "bf16", "f32")
    for splits in (1, 4):
        compare(run(ob, c, q, [n], [3], "bf16", "f32", num_splits=splits), want)


def test_scale_and_rows_of_any_stride():
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(6)
    lens, new = [200, 77], [3, 20]
    x = [tokens(rng, 2, 200, 2, "bf16") for _ in "kv"]
    q = tokens(rng, 2, 20, 6, "bf16")
    c = scattered_cache(ob, 2, 2, 2, 64, "bf16", rng)
    append(ob, c, x, [0, 0], lens, "bf16")
    for scale in (0.25, 1e-3):
        want = attention(q, x, lens, new, 64, "bf16", "bf16", scale=scale)
        for packed in (False, True):
            compare(run(ob, c, q, lens, new, "bf16", "bf16", packed, stride=40, scale=scale), want)


def test_pages_that_are_none_are_left_out_and_rows_that_see_nothing_are_zeros():
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(7)
    lens, new = [500, 128, 260], [2, 1, 132]
    x = [tokens(rng, 3, 500, 2, "bf16") for _ in "kv"]
    q = tokens(rng, 3, 132, 4, "bf16")
    c = scattered_cache(ob, 2, 3, 4, 32, "bf16", rng)
    append(ob, c, x, [0] * 3, lens, "bf16")
    c.block_table[0, 0], c.block_table[0, 2], c.block_table[1, 0], c.block_table[2, 0] = -1, c.num_pages, 2 ** 31 - 1, -2 ** 31
    want = attention(q, x, lens, new, 32, "bf16", "f32", left_out={0: [0, 2], 1: [0], 2: [0]})
    assert not want[1][0].any()
    for splits in (0, 1, 3):
        got = run(ob, c, q, lens, new, "bf16", "f32", num_splits=splits, max_seq_len_hint=500)
        compare(got, want)
        assert not got[1].any()


def test_lengths_below_the_new_tokens_and_rows_past_the_end():
    """A length that does not count its new tokens: the rows before its first token see nothing.  Rows past n_rows are
    not touched."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(8)
    x = [tokens(rng, 2, 40, 1, "bf16") for _ in "kv"]
    q = tokens(rng, 2, 5, 2, "bf16")
    c = scattered_cache(ob, 1, 2, 1, 32, "bf16", rng)
    append(ob, c, x, [0, 0], [3, 40], "bf16")
    out = torch.full((8, 2, D), 7.0, device="cuda")
    for splits in (1, 2):
        out.fill_(7.0)
        ob.q8_attn(c, dev(q.reshape(10, 2, D)[:8], "bf16"), ints([3, 40]), row_starts=ints([0, 6]), max_new=5, out=out, num_splits=splits)
        got = out.double().cpu().numpy()
        assert not got[:2].any() and (got[5] == 7.0).all()
        want = attention(q, x, [3], [3], 32, "bf16", "f32")[0]
        q2 = q.copy()
        q2[0, :3] = q.reshape(10, 2, D)[2:5]
        o, tol = attention(q2, x, [3], [3], 32, "bf16", "f32")[0]
        assert (np.abs(got[2:5] - o) <= tol).all()
        q2[1, :5] = 0
        q2[1, :2] = q.reshape(10, 2, D)[6:8]
        o, tol = attention(q2[1:], [y[1:] for y in x], [40], [5], 32, "bf16", "f32")[0]
        assert (np.abs(got[6:8] - o[:2]) <= tol[:2]).all()


def test_later_tokens_do_not_touch_earlier_rows():
    """Rows of a piece of a prompt are the bits of the same rows when the tokens behind them are others."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(9)
    n, T = 300, 100
    x = [tokens(rng, 1, n, 2, "bf16") for _ in "kv"]
    q = tokens(rng, 1, T, 4, "bf16")
    outs = []
    for other in (False, True):
        if other:
            for y in x:
                y[:, 256:] = 1000.0 * tokens(rng, 1, n - 256, 2, "bf16")   # (a whole block of codes and the window)
            x = [dev(y, "bf16").double().cpu().numpy() for y in x]
        c = scattered_cache(ob, 2, 1, 3, 32, "bf16", np.random.default_rng(0))
        append(ob, c, x, [0], [n], "bf16")
        outs.append(run(ob, c, q, [n], [T], "bf16", "f32", num_splits=1)[0][:56])
    assert np.array_equal(*outs)


def test_the_same_call_gives_the_same_bits_and_may_share_a_workspace_in_order():
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(10)
    lens = [900, 130, 77]
    x = [tokens(rng, 3, 900, 2, "bf16") for _ in "kv"]
    c = scattered_cache(ob, 2, 3, 8, 32, "bf16", rng)
    append(ob, c, x, [0] * 3, lens, "bf16")
    q1, q2 = (dev(tokens(rng, 3, 1, 8, "bf16"), "bf16") for _ in range(2))
    ws = torch.empty(ob.q8_workspace_bytes(c, 8, 1, 4), dtype=torch.uint8, device="cuda")
    ws.view(torch.int32).fill_(0x7fc00000)
    first = [ob.q8_attn(c, q, ints(lens), num_splits=4, workspace=ws) for q in (q1, q2, q1)]
    assert torch.equal(first[0], first[2]) and not torch.equal(first[0], first[1])


def test_a_long_sequence_of_many_splits():
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(12)
    n = 40000
    x = [tokens(rng, 1, n, 1, "bf16") for _ in "kv"]
    c = scattered_cache(ob, 1, 1, n // 128 + 1, 64, "bf16", rng)
    append(ob, c, x, [0], [n], "bf16")
    q = tokens(rng, 1, 3, 5, "bf16")
    want = attention(q, x, [n], [3], 64, "bf16", "f32")
    for splits in (0, 7, 512):
        compare(run(ob, c, q, [n], [3], "bf16", "f32", num_splits=splits, max_seq_len_hint=n), want)


def test_another_stream():
    """Everything the call makes belongs to the stream it is told."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(14)
    lens = [600, 300]
    x = [tokens(rng, 2, 600, 2, "bf16") for _ in "kv"]
    s = torch.cuda.Stream()
    c = scattered_cache(ob, 2, 2, 5, 32, "bf16", rng)
    k, v, q = dev(padded_rows(x[0], [0, 0], lens, 600), "bf16"), dev(padded_rows(x[1], [0, 0], lens, 600), "bf16"), tokens(rng, 2, 1, 4, "bf16")
    n, qd = ints(lens), dev(q, "bf16")
    torch.cuda.synchronize()
    ob.q8_append(c, k, v, n, new_lens=n, stream=s)
    out = ob.q8_attn(c, qd, n, max_seq_len_hint=600, num_splits=3, stream=s)
    s.synchronize()
    compare([out[b].double().cpu().numpy() for b in range(2)], attention(q, x, lens, [1, 1], 32, "bf16", "bf16"))


def test_lengths_of_any_size_stay_inside_their_tensors():
    """Lengths up to 2^31 - 1 and below 0: what no page or window holds is left out."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(16)
    x = [tokens(rng, 5, 300, 1, "bf16") for _ in "kv"]
    c = scattered_cache(ob, 1, 5, 2, 32, "bf16", rng, poison=False)
    append(ob, c, x, [0] * 5, [300] * 5, "bf16")
    lens = ints([2 ** 31 - 1, 2 ** 31 - 4097, -1, -2 ** 31, 300])
    guard = torch.full((7, 3, 4, D), 7.0, device="cuda")
    for splits in (1, 3):
        out = guard[1:6]
        out.fill_(7.0)
        ob.q8_attn(c, dev(tokens(rng, 5, 3, 4, "bf16"), "bf16"), lens, out=out, num_splits=splits)
        assert (guard[0] == 7.0).all() and (guard[6] == 7.0).all()
        assert not out[2:4].any() and torch.isfinite(out).all() and out[4].any()
    before = [y.clone() for y in (c.k_codes, c.v_codes, c.block_table)]
    k = torch.full((5, 40, 1, D), 7.0, device="cuda")
    ob.q8_read(c, lens, starts=ints([2 ** 31 - 30, 0, 0, 0, 280]), k=k)
    assert (k[2:4] == 7.0).all()
    rows = dev(tokens(rng, 5, 3, 1, "bf16"), "bf16")
    ob.q8_append(c, rows, rows, lens)       # (past the table's end: the window only)
    assert all(torch.equal(y, z) for y, z in zip(before, (c.k_codes, c.v_codes, c.block_table)))


@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_logits_of_any_size(sign):
    """Scaled logits of 2^29 in size and their neighbours: whoever has the largest takes the row."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(17)
    x = [tokens(rng, 1, 100, 1, "bf16") for _ in "kv"]
    x[0][...] = 2.0 ** 12 * rng.choice([1.0, 1.0078125], size=x[0].shape)
    x[0][0, 97] = 2.0 ** 12 * (1.0 if sign < 0 else 1.0078125)          # in the window: it is the largest
    q = sign * 2.0 ** 13 * np.ones((1, 1, 1, D))
    c = scattered_cache(ob, 1, 1, 1, 32, "bf16", rng)
    append(ob, c, x, [0], [100], "bf16")
    k = stands_for(x[0][0, :, 0], 32, "bf16")[0]
    logits = k @ q[0, 0, 0] / np.sqrt(D)
    best = np.nonzero(logits == logits.max())[0]
    got = run(ob, c, q, [100], [1], "bf16", "f32")[0]
    assert 2.0 ** 28 < abs(logits).max() < 2.0 ** 30
    # (equal logits share the row; the next is thousands below)
    want = stands_for(x[1][0, :, 0], 32, "bf16")[0][best].mean(0)
    assert (np.abs(got[0, 0] - want) <= 2.0 ** -16 * np.abs(x[1][0, best, 0]).max(0) + 2.0 ** -24).all()


def test_captured_and_replayed_over_growing_lengths():
    """One graph of append and attention, replayed while the lengths on the device grow past block and page ends, with
    eager work between; every replay is the eager call's bits."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(18)
    B, H, HQ, first = 3, 2, 6, [120, 30, 250]
    x = [tokens(rng, B, 400, H, "bf16") for _ in "kv"]
    a, b = (scattered_cache(ob, H, B, 4, 32, "bf16", np.random.default_rng(0)) for _ in range(2))
    for c in (a, b):
        append(ob, c, x, [0] * B, first, "bf16")
    k, v, q = (torch.zeros(B, 1, n, D, dtype=torch.bfloat16, device="cuda") for n in (H, H, HQ))
    lens, out = ints(first), torch.zeros(B, 1, HQ, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(ob.q8_workspace_bytes(b, HQ, 1, 3), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.q8_append(b, k, v, lens)
        ob.q8_attn(b, q, lens, out=out, num_splits=3, workspace=ws)
    n = np.array(first)
    for i in range(140):
        n += 1
        k.copy_(dev(np.stack([x[0][j, n[j] - 1] for j in range(B)])[:, None], "bf16"))
        v.copy_(dev(np.stack([x[1][j, n[j] - 1] for j in range(B)])[:, None], "bf16"))
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        lens.copy_(torch.from_numpy(n))
        graph.replay()
        ob.q8_append(a, k, v, lens)
        want = ob.q8_attn(a, q, lens, num_splits=3)
        assert torch.equal(out, want), i
    compare([out[j].double().cpu().numpy() for j in range(B)], attention(q.double().cpu().numpy(), x, list(n), [1] * B, 32, "bf16", "bf16"))


@pytest.mark.parametrize("heads", [(2, 1), (20, 1)])
def test_the_largest_fp16_numbers_stay_finite(heads):
    """Values of an fp16 cache whose codes stand for 65536: an output that is one of them, or nearly, is 65504 as fp16."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(22)
    lens, new = [64, 40, 33], [1, 2, 1]
    x = [tokens(rng, 3, 64, 1, "f16") for _ in "kv"]
    x[1][0, :, 0, :4] = [65504.0, -65504.0, 63488.0, np.inf]      # every token has it
    x[1][1, 7, 0, :2] = 65504.0, -np.inf                          # one that takes the softmax
    x[1][2, :, 0, :2] = 63488.0, -63488.0
    q = tokens(rng, 3, 2, heads[0], "f16")
    x[0][1, :, 0] = 0.01 * rng.integers(-3, 4, size=(64, D))
    x[0][1, 7, 0] = 4.0 * np.sign(q[1, 0, 0])
    q[1, :] = q[1, 0, 0]
    x = [dev(y, "f16").double().cpu().numpy() for y in x]
    c = scattered_cache(ob, 1, 3, 1, 32, "f16", rng)
    append(ob, c, x, [0] * 3, lens, "f16")
    for out in ("f16", "f32"):
        want = attention(q, x, lens, new, 32, "f16", out)
        assert max(np.abs(o).max() for o, _ in want) > 65520.0     # (what rounds to infinity)
        if out == "f16":
            want = [(np.clip(o, -65504.0, 65504.0), tol) for o, tol in want]
        for splits in (1, 2):
            compare(run(ob, c, q, lens, new, "f16", out, num_splits=splits), want)


@pytest.mark.parametrize("rows", [1, 20])
def test_fp16_values_of_the_window_enter_as_they_are(rows):
    """A token of logit 0 and 30 of one weight just above 1/2, with a value whose last three bits the products take apart.

    The weight w = (1 + 2^-9 (1 - 2^-7)) / 2 is two bf16 limbs exactly, 1/2 and 2^-10 (1 - 2^-7); the computed one is within 2^-22 (the
    exponential) and 2^-23 (scale and logit, each rounded) of it, less than half a step (2^-19) of the lower limb, so that the limbs are
    the exact ones and only their sum is off by as much.  A product adds 32 numbers, 2^-24 each at worst; the sum of the
    weights and the division take 12 steps.  Without the lower limbs' product with the value's last bits, 3 2^-10, the output is
    too small by 2^-9 3 2^-10 = 2^-17.4 of itself."""
    from paper_2605_19660_amd import binding as ob
    w, value = (1.0 + 2.0 ** -9 * (1.0 - 2.0 ** -7)) / 2.0, 1.0 + 3.0 * 2.0 ** -10
    x = [np.zeros((1, 31, 1, D)) for _ in "kv"]
    x[0][0, 1:, 0, 0], x[1][0, 1:, 0] = -1.0, value
    q = np.zeros((1, 1, rows, D))
    q[..., 0] = 1.0
    c = scattered_cache(ob, 1, 1, 1, 32, "f16", np.random.default_rng(0))
    append(ob, c, x, [0], [31], "f16")
    got = run(ob, c, q, [31], [1], "f16", "f32", scale=-np.log(w))[0][0]
    off = np.abs(got / (30 * w * value / (30 * w + 1.0)) - 1.0)
    assert (off <= (32 + 12) * 2.0 ** -24 + 1.5 * 2.0 ** -22).all(), float(off.max())


def test_a_scale_below_the_smallest_number():
    """Keys of 2^-105 in blocks of scale 2^-100, and a softmax_scale of 2^-70: the scale of their logits is below every fp32 number, and
    all tokens weigh the same, those that a row does not see nothing."""
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(23)
    lens, new = [64, 200], [9, 33]
    x = [tokens(rng, 2, 200, 1, "bf16") for _ in "kv"]
    x[0][...] = 2.0 ** -105 * rng.choice([1.0, -1.0], size=x[0].shape)
    q = tokens(rng, 2, 33, 2, "bf16")
    c = scattered_cache(ob, 1, 2, 2, 32, "bf16", rng)
    append(ob, c, x, [0, 0], lens, "bf16")
    for scale in (2.0 ** -70, 1e-40):
        want = attention(q, x, lens, new, 32, "bf16", "f32", scale=scale)
        for splits in (1, 2):
            compare(run(ob, c, q, lens, new, "bf16", "f32", num_splits=splits, scale=scale), want)
