"""A serving step over a paged 8-bit cache: its operators, for timing and for comparing results.

A server plans a step on the GPU from what its requests hold and want (`plan_step`: pages given back
and handed out, block tables, where every row of the step goes), puts the new keys and values into the
cache (`q8_append`: e4m3 numbers with one power-of-two scale for each block of tokens and kv head, the
last tokens in 16 bits), attends from all new tokens (`q8_attn`), reads history back for code that wants
16-bit keys and values (`q8_read`) and draws the next tokens from the logits (`sample`).

With ``own`` set `run` makes the calls of ``paper_2605_19660_amd.binding``; without it the same results
come from elementary torch operations in 32 bits (64 for the weights and sums that decide a token),
rounded once.  `exact` works in 64 bits from the numbers before they are laid out in pages.
"""
import math

import numpy as np
import torch

own = False

D = PAGE = 128
IO = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"f32": 0, "bf16": 1, "f16": 2}
HEADS = [(32, 8), (28, 4), (8, 8), (16, 2), (20, 4), (6, 2), (32, 1)]

PLAN = {"kind": "plan", "batch": 8, "context": 1000, "pages": 64, "prompt": 0, "prompts": 0, "short": False}
CACHE = {"batch": 1, "context": 1000, "q_heads": 32, "kv_heads": 8, "block": 32, "io": "bf16", "ragged": False,
         "scattered": False}
WRITE = {"kind": "write", "tokens": 1, "packed": False, **CACHE}
READ = {"kind": "read", "tokens": 1000, "out": "bf16", **CACHE}
ATTN = {"kind": "attn", "tokens": 1, "packed": False, **CACHE}
SAMPLE = {"kind": "sample", "batch": 1, "vocab": 32000, "io": "f32", "top_k": 0, "top_p": 1.0, "min_p": 0.0,
          "greedy": False, "mixed": False, "probs": False}


def listed():
    return [
        # eight users' next token: launch and latency are all there is
        {**PLAN, "name": "plan-b8-decode"},
        # a large server: 480 answers go on, some end, 32 prompts' pieces come in, and the pages run short
        {**PLAN, "name": "plan-b512-mixed", "batch": 512, "context": 8192, "pages": 128, "prompt": 1000, "prompts": 32,
         "short": True},
        # one user's next token joins the window, and is read back
        {**WRITE, "name": "write-b1-token"},
        # prompts of four users, side by side in one matrix, into empty caches
        {**WRITE, "name": "write-b4-8k-prompts", "batch": 4, "context": 8192, "tokens": 8192, "ragged": True, "packed": True,
         "scattered": True, "block": 64},
        # one user's short history
        {**READ, "name": "read-b1-1k"},
        # a batch of contexts handed to 32-bit code
        {**READ, "name": "read-b4-16k-f32", "batch": 4, "context": 16384, "tokens": 16384, "io": "f16", "out": "f32",
         "ragged": True, "scattered": True},
        # one user's next token over a short context
        {**ATTN, "name": "attn-b1-1k"},
        # the batched server's decoding step
        {**ATTN, "name": "attn-b8-32k", "batch": 8, "context": 32768},
        # one very long document, seven query heads a kv head, four drafts behind the last token, larger blocks
        {**ATTN, "name": "attn-b1-128k-g7-t5", "context": 131001, "tokens": 5, "q_heads": 28, "kv_heads": 4, "block": 128},
        # pieces of prompts and single tokens of ragged sequences in one packed batch
        {**ATTN, "name": "attn-b8-4k-packed-t500-f16", "batch": 8, "context": 4100, "tokens": 500, "io": "f16", "ragged": True,
         "scattered": True, "packed": True},
        # one user's draw; and a batch with a large vocabulary, every row with its own settings, the distribution kept
        {**SAMPLE, "name": "sample-b1-32000-top-p", "top_p": 0.9},
        {**SAMPLE, "name": "sample-b64-128003-mixed-probs", "batch": 64, "vocab": 128003, "top_k": 50, "top_p": 0.95,
         "min_p": 0.02, "greedy": True, "mixed": True, "probs": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "write", "read", "attn", "attn", "attn", "sample", "sample"])
    if kind == "plan":
        batch, pages = _log_int(rng, 1, 512), _log_int(rng, 2, 256)
        context = _log_int(rng, 1, pages * PAGE)
        return {**PLAN, "batch": batch, "pages": pages, "context": context, "prompt": _log_int(rng, 2, min(1000, pages * PAGE)),
                "prompts": rng.randint(0, min(batch, 32)), "short": rng.random() < 0.5}
    if kind == "sample":
        vocab = _log_int(rng, 1000, 200000)
        return {**SAMPLE, "vocab": vocab, "batch": _log_int(rng, 1, max(1.01, min(256, 8000000 / vocab))),
                "io": rng.choice(["f32", "f32", "bf16", "f16"]), "top_k": rng.choice([0, 1, _log_int(rng, 2, 1000)]),
                "top_p": rng.choice([1.0, 0.5, 0.9, 0.95, 0.99]), "min_p": rng.choice([0.0, 0.0, 0.02, 0.1]),
                "greedy": rng.random() < 0.2, "mixed": rng.random() < 0.5, "probs": rng.random() < 0.3}
    heads = rng.choice(HEADS)
    c = {"q_heads": heads[0], "kv_heads": heads[1], "block": rng.choice([32, 32, 64, 128]), "io": rng.choice(["bf16", "bf16", "f16"]),
         "ragged": rng.random() < 0.5, "scattered": rng.random() < 0.5}
    # 1 .. 131072 tokens a sequence, 1 .. 64 sequences, at most half of the largest cache
    most = 131072 if kind == "attn" else 32768
    c["context"] = rng.choice([1, 127, 128] + [_log_int(rng, 100, most) for _ in range(4)])
    full = {"write": 16384, "read": 32768, "attn": 131072}[kind] * 8 // heads[1]
    c["batch"] = min(64, _log_int(rng, 1, max(1.01, full / c["context"])))
    if kind == "read":
        return {**READ, **c, "tokens": c["context"] if rng.random() < 0.5 else _log_int(rng, 1, c["context"]),
                "out": rng.choice([c["io"], "f32"])}
    c["packed"] = rng.random() < 0.5
    if kind == "write":
        c["tokens"] = c["context"] if rng.random() < 0.5 else min(c["context"], _log_int(rng, 1, 32))
        return {**WRITE, **c}
    c["tokens"] = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 16, 600)])
    # the logits of the plain form are held whole
    while c["batch"] > 1 and c["batch"] * heads[0] * c["tokens"] * c["context"] > 1 << 29:
        c["batch"] //= 2
    while c["tokens"] > 1 and c["batch"] * heads[0] * c["tokens"] * c["context"] > 1 << 29:
        c["tokens"] //= 2
    c["tokens"] = min(c["tokens"], c["context"])
    return {**ATTN, **c}


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + what)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).cuda()


def _lengths(case, seed):
    """Tokens of every sequence after the step, and its new ones."""
    rng = np.random.default_rng([seed, 1])
    B, T = case["batch"], case["tokens"]
    n, new = np.full(B, case["context"]), np.full(B, T)
    if case["ragged"]:
        # the same spread of lengths whatever the seed, dealt out by it
        low = max(1, case["context"] // 2)
        n = low + (np.arange(B) + 1) * (case["context"] - low) // B
        if case["kind"] == "attn":
            # pieces of prompts, single tokens between them
            new = np.where(np.arange(B) % 2 == B % 2, min(T, 1), (np.arange(B) + 1) * T // B)
        if case["kind"] == "write" and T == case["context"]:
            new = n
        order = rng.permutation(B)
        n, new = n[order], np.minimum(new, n)[order]
    return n, np.minimum(new, n)


def _tokens(case, seed):
    """Keys and values of every token, [batch, token, kv head, channel] of the io type."""
    g = _gen(seed, 1)
    B, S, H = case["batch"], case["context"], case["kv_heads"]
    gain = torch.ones(H, D, device="cuda")
    gain[:, ::37] = 8.0                                       # outlier channels
    out = []
    for gains in (gain, gain.flip(1)):
        x = _randn(g, B, S, H, D)
        x *= torch.exp(0.5 * _randn(g, B, S, 1, 1))
        x *= gains
        out.append(x.to(IO[case["io"]]))
        del x
    return out


def _coded(x, block):
    """e4m3 numbers and scales of [..., tokens, head, channel], tokens in whole blocks: what the numbers
    stand for is code * scale, scale the smallest power of two that keeps the block's largest below 448."""
    y = x.float().unflatten(-3, (-1, block))
    m, e = torch.frexp(y.abs().amax((-3, -1), keepdim=True))
    e = torch.where(m > 0, e - 9 + (m > 0.875), torch.zeros_like(e))
    scale = ((e + 127) << 23).int().view(torch.float32)
    return (y / scale).to(torch.float8_e4m3fn).flatten(-4, -3), scale


def _places():
    """Where a page keeps the codes of [token][channel], keys and values (see the library's header)."""
    t, c = np.meshgrid(np.arange(PAGE), np.arange(D), indexing="ij")
    k = ((t // 16 * 2 + c // 64) * 4 + c % 64 // 16) * 256 + t % 16 * 16 + c % 16
    v = (((t // 32 * 4 + c // 32) * 4 + t % 16 // 4) * 16 + c % 16) * 16 + c % 32 // 16 * 8 + t % 32 // 16 * 4 + t % 4
    return k, v


def _pools(case, seed, held, tokens):
    """Pools that hold the first `held` tokens of every sequence, and the block table."""
    B, H, block = case["batch"], case["kv_heads"], case["block"]
    P = (case["context"] + PAGE - 1) // PAGE
    total = B * P
    perm = np.random.default_rng([seed, 4]).permutation(total) if case["scattered"] else np.arange(total)
    page = torch.from_numpy(perm).cuda()
    io = IO[case["io"]]
    p = {"block_table": _dev(perm.reshape(B, P))}
    held_gpu = torch.from_numpy(held).cuda()
    done = held_gpu // block * block
    at = torch.arange(P * PAGE, device="cuda")
    for name, x, place in zip("kv", tokens, _places()):
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, P * PAGE - x.shape[1]))
        codes, scale = _coded(x, block)
        ready = (at[None] < done[:, None])[:, :, None, None]
        codes = torch.where(ready, codes.view(torch.uint8), torch.zeros((), dtype=torch.uint8, device="cuda"))
        pool = torch.empty(total, H, PAGE * D, dtype=torch.uint8, device="cuda")
        order = torch.from_numpy(np.argsort(place.reshape(-1))).cuda()
        pool[page] = codes.view(B, P, PAGE, H, D).permute(0, 1, 3, 2, 4).reshape(total, H, -1)[..., order]
        p[name + "_codes"] = pool
        scales = torch.empty(total, H, PAGE // block, device="cuda")
        scale = torch.where(ready[:, ::block], scale[:, :, 0], torch.ones((), device="cuda"))
        scales[page] = scale[..., 0].view(B, P, PAGE // block, H).transpose(2, 3).reshape(total, H, -1)
        p[name + "_scales"] = scales
        # the window: tokens of the last whole block and behind it, at their place modulo two blocks
        win = torch.zeros(B, 2 * block, H, D, dtype=io, device="cuda")
        first = (done - block).clamp(min=0)[:, None] + torch.arange(2 * block, device="cuda")
        inside = first < held_gpu[:, None]
        b = torch.arange(B, device="cuda")[:, None].expand_as(first)
        win[b[inside], first[inside] % (2 * block)] = x[b[inside], first[inside]]
        p["win_" + name] = win.transpose(1, 2).contiguous()
        del codes, x, win
    return p


def _handle(case, pools):
    """The library's cache object over these pools, which a program keeps beside them."""
    from paper_2605_19660_amd import binding as ob
    B, P = pools["block_table"].shape
    cache = ob.Q8Cache(case["kv_heads"], B, P, block=case["block"], io_dtype=CODE[case["io"]])
    for name, t in pools.items():
        dst = getattr(cache, name)
        dst.copy_(t.view(dst.shape))
    return cache


def _starts(case, seed):
    n, _ = _lengths(case, seed)
    rng = np.random.default_rng([seed, 5])
    return np.array([rng.integers(0, max(1, x - case["tokens"] + 1)) for x in n], np.int32)


def _rows_of(case, new):
    """First row of every sequence, and how many rows there are (a packed batch has a few that belong to nobody)."""
    if not case["packed"]:
        return None, case["batch"] * case["tokens"]
    return np.concatenate([[0], np.cumsum(new)]), int(new.sum()) + 3


def _rows(case, new, x):
    """[batch, T, ...] rows as the step has them."""
    starts, n = _rows_of(case, new)
    if starts is None:
        return x
    out = x.new_zeros(n, *x.shape[2:])
    b = np.repeat(np.arange(len(new)), new)
    t = np.arange(new.sum()) - np.repeat(starts[:-1], new)
    out[:len(b)] = x[torch.from_numpy(b).cuda(), torch.from_numpy(t).cuda()]
    return out


def _queries(case, seed):
    return _randn(_gen(seed, 4), case["batch"], case["tokens"], case["q_heads"], D).to(IO[case["io"]])


def _new_tokens(case, lens, new, x):
    """The tokens of the step, [batch, T, kv head, channel]."""
    at = (lens - new)[:, None] + np.arange(case["tokens"])
    at = torch.from_numpy(np.minimum(at, case["context"] - 1)).cuda()
    return x[torch.arange(case["batch"], device="cuda")[:, None], at]


def _plan_inputs(case, seed):
    rng = np.random.default_rng([seed, 2])
    B, P = case["batch"], case["pages"]
    lens = rng.integers((case["context"] + 1) // 2, case["context"] + 1, size=B)
    lens = np.minimum(lens, P * PAGE - 1)
    want = np.ones(B, np.int64)
    some = rng.permutation(B)[:case["prompts"]]
    lens[some] = rng.integers(0, max(1, lens.min() // 2) + 1, size=len(some))
    want[some] = rng.integers(1, case["prompt"] + 1, size=len(some))
    rows = B + case["prompts"] * case["prompt"] * 2 // 5            # (hardly enough, as a step's limit is)
    keep = lens.copy()
    if B > 8:
        want[rng.integers(0, B, size=B // 16)] = 0              # idle
        ends = rng.integers(0, B, size=B // 16)                 # answers that are complete
        keep[ends], want[ends] = 0, 0
        back = rng.integers(0, B, size=B // 4)                  # drafts that did not stand, in the last page
        room = np.maximum(lens[back] - 1, 0) % PAGE
        keep[back] = np.where(keep[back] > 0, lens[back] - np.minimum(room, 3), keep[back])
    held = (lens + PAGE - 1) // PAGE
    need = np.where(want > 0, (keep + want + PAGE - 1) // PAGE - (keep + PAGE - 1) // PAGE, 0).sum()
    total = B * P
    perm = rng.permutation(total)
    spare = min(total - held.sum(), int(need * 0.8) if case["short"] else need + 16)
    table = np.full((B, P), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(held)])
    for b in range(B):
        table[b, :held[b]] = perm[at[b]:at[b + 1]]
    free = np.zeros(total, np.int32)
    free[:spare] = perm[at[-1]:at[-1] + spare]
    return lens, keep, want, table, free, spare, rows


def _logits(case, seed):
    g = _gen(seed, 3)
    B, V = case["batch"], case["vocab"]
    # a few likely tokens, a long tail
    rank = torch.argsort(torch.rand(B, V, device="cuda", generator=g), -1).float()
    x = (1.5 * _randn(g, B, V) - 1.2 * torch.log1p(rank)).to(IO[case["io"]])
    rng = np.random.default_rng([seed, 7])
    temp = rng.uniform(0.6, 1.3, size=B)
    if case["greedy"]:
        temp[rng.integers(0, B, size=(B + 7) // 8)] = 0.0
    k, p, m = np.full(B, case["top_k"]), np.full(B, case["top_p"]), np.full(B, case["min_p"])
    if case["mixed"]:
        k, p, m = (np.where(rng.random(B) < 0.5, a, none) for a, none in ((k, 0), (p, 1.0), (m, 0.0)))
    return x, {"temperature": _dev(temp, np.float32), "top_k": _dev(k), "top_p": _dev(p, np.float32),
               "min_p": _dev(m, np.float32), "u": torch.rand(B, device="cuda", generator=g)}


def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case}
    if kind == "plan":
        lens, keep, want, table, free, n_free, rows = _plan_inputs(case, seed)
        e = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
        B = case["batch"]
        return {**s, "lens": _dev(lens), "keep": _dev(keep), "want": _dev(want), "table": _dev(table), "free": _dev(free),
                "n_free": _dev([n_free]), "n_rows": rows,
                "out": {"lens_out": e(B), "new_lens": e(B), "n_free_out": e(1), "row_starts": e(B + 1), "positions": e(rows),
                        "row_seq": e(rows), "slots": e(rows)}}
    if kind == "sample":
        s["logits"], s["how"] = _logits(case, seed)
        return s
    lens, new = _lengths(case, seed)
    tokens = _tokens(case, seed)
    pools = _pools(case, seed, lens - new if kind == "write" else lens, tokens)
    s["lens"] = _dev(lens)
    if kind != "read":
        starts, n = _rows_of(case, new)
        s["new_lens"] = _dev(new) if case["ragged"] or case["packed"] else None
        s["row_starts"] = None if starts is None else _dev(starts)
    if kind in ("read", "write"):
        s["starts"] = _dev(_starts(case, seed) if kind == "read" else lens - new)
        out = IO[case["out" if kind == "read" else "io"]]
        s["k"] = torch.zeros(case["batch"], case["tokens"], case["kv_heads"], D, device="cuda", dtype=out)
        s["v"] = torch.zeros_like(s["k"])
    if kind == "write":
        s["k_new"], s["v_new"] = (_rows(case, new, _new_tokens(case, lens, new, x)) for x in tokens)
    if kind == "attn":
        s["q"] = _rows(case, new, _queries(case, seed))
        s["out"] = torch.zeros_like(s["q"])
    if own:
        s["cache"] = _handle(case, pools)
    else:
        s["pools"] = pools
        s["places"] = tuple(torch.from_numpy(x).cuda() for x in _places())
    return s


# ---- one pass ----------------------------------------------------------------------------------

def _held(s, name, at, there):
    """Keys or values at positions `at` [batch, n], in 32 bits: [batch, n, kv head, channel], zeros where there is none."""
    c, p = s["case"], s["pools"]
    block = c["block"]
    dev = at.device
    b = torch.arange(c["batch"], device=dev)[:, None]
    h = torch.arange(c["kv_heads"], device=dev)
    at = torch.where(there, at, torch.zeros_like(at))
    page = p["block_table"].long()[b, at // PAGE]
    where = s["places"][0 if name == "k" else 1][at % PAGE]
    codes = p[name + "_codes"][page[:, :, None, None], h[:, None], where[:, :, None, :]]
    scale = p[name + "_scales"][page[:, :, None], h, (at % PAGE // block)[:, :, None]]
    x = codes.view(torch.float8_e4m3fn).float() * scale[..., None]
    coded = (at < (s["lens"].long() // block * block)[:, None])[:, :, None, None]
    win = p["win_" + name][b[:, :, None], h, (at % (2 * block))[:, :, None]].float()
    return torch.where(there[:, :, None, None], torch.where(coded, x, win), torch.zeros((), device=dev))


def _padded(s, x):
    """Rows of the step as [batch, T, ...], and which of them there are."""
    c = s["case"]
    B, T = c["batch"], c["tokens"]
    t = torch.arange(T, device=x.device)
    n = torch.full((B,), T, device=x.device) if s["new_lens"] is None else s["new_lens"].long()
    there = t < n[:, None]
    if s["row_starts"] is None:
        return x, there, n, None
    row = torch.where(there, s["row_starts"].long()[:B, None] + t, torch.zeros((), dtype=torch.long, device=x.device))
    return x[row], there, n, row


def _plain_read(s):
    c = s["case"]
    at = s["starts"].long()[:, None] + torch.arange(c["tokens"], device="cuda")
    there = at < s["lens"][:, None]
    out = []
    for n in "kv":
        out.append(torch.where(there[:, :, None, None], _held(s, n, at, there).to(s[n].dtype), s[n]))
    return tuple(out)


def _plain_write(s):
    c, p = s["case"], s["pools"]
    B, T, H, block = c["batch"], c["tokens"], c["kv_heads"], c["block"]
    lens = s["lens"].long()
    blocks = (T + block - 2) // block + 1
    for name in "kv":
        x, there, n, _ = _padded(s, s[name + "_new"])
        dev = x.device
        b = torch.arange(B, device=dev)[:, None]
        old = lens - n
        first = old // block * block
        at = first[:, None] + torch.arange(blocks * block, device=dev)
        win = p["win_" + name]
        before = win.transpose(1, 2)[b, at % (2 * block)]
        mine = (at - old[:, None]).clamp(min=0, max=T - 1)
        y = torch.where((at < old[:, None])[:, :, None, None], before, x[b, mine])
        # whole blocks become codes in their pages
        codes, scale = _coded(y, block)
        end = at[:, ::block] + block
        whole = (end <= lens[:, None]) & (n > 0)[:, None]
        hold = (at // PAGE).clamp(max=p["block_table"].shape[1] - 1)
        page = p["block_table"].long()[b, hold]
        where = s["places"][0 if name == "k" else 1][at % PAGE]
        pool = p[name + "_codes"].view(-1)
        index = (page[:, :, None, None] * H + torch.arange(H, device=dev)[:, None]) * (PAGE * D) + where[:, :, None, :]
        keep = whole.repeat_interleave(block, 1)[:, :, None, None].expand_as(index)
        pool[index[keep]] = codes.view(torch.uint8)[keep]
        index = (page[:, ::block, None] * H + torch.arange(H, device=dev)) * (PAGE // block) + (at[:, ::block] % PAGE // block)[:, :, None]
        keep = whole[:, :, None].expand_as(index)
        p[name + "_scales"].view(-1)[index[keep]] = scale[:, :, 0, :, 0][keep]
        # and the last tokens go into the window
        late = (at >= old[:, None]) & (at < lens[:, None]) & (at >= (lens // block * block - block)[:, None])
        bb = b.expand_as(at)[late]
        win[bb, :, at[late] % (2 * block)] = y[late]
    return _plain_read(s)


def _plain_attn(s):
    c = s["case"]
    B, T, hq, hk, S = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"], c["context"]
    g = hq // hk
    q, there, n, row = _padded(s, s["q"])
    at = torch.arange(S, device=q.device)
    held = at < s["lens"][:, None]
    k, v = (_held(s, x, at.expand(B, S), held).transpose(1, 2).contiguous() for x in "kv")
    q = q.float().view(B, T, hk, g, D).permute(0, 2, 1, 3, 4).reshape(B, hk, T * g, D)
    logits = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (1 / math.sqrt(D))
    mine = (s["lens"] - n)[:, None] + torch.arange(T, device=q.device)
    logits.masked_fill_((at > mine[:, :, None]).repeat_interleave(g, 1)[:, None], float("-inf"))
    logits -= logits.amax(-1, keepdim=True)
    e = torch.exp_(logits)
    out = torch.matmul(e, v) / e.sum(-1, keepdim=True)
    out = out.view(B, hk, T, g, D).permute(0, 2, 1, 3, 4).reshape(B, T, hq, D).to(s["q"].dtype)
    if row is None:
        return torch.where(there[:, :, None, None], out, s["out"])
    whole = s["out"].clone()
    whole[row[there]] = out[there]
    return whole


def _plain_plan(s):
    lens, keep, want, table = (s[x].long() for x in ("lens", "keep", "want", "table"))
    B, P = table.shape
    dev = lens.device
    N = s["free"].numel()
    keep, col = torch.minimum(keep, lens), torch.arange(P, device=dev)
    held, kept = (lens + PAGE - 1) // PAGE, (keep + PAGE - 1) // PAGE
    # pages that come back, on top of the stack
    back = (col >= kept[:, None]) & (col < held[:, None])
    to = torch.where(back, s["n_free"] + back.flatten().cumsum(0).view(B, P) - 1, N)
    free = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter(0, to.flatten(), s["table"].flatten())
    pages = s["n_free"].long() + back.sum()
    # who takes part
    need = (keep + want + PAGE - 1) // PAGE - kept
    fits = (want > 0) & (keep + want <= P * PAGE)
    need = need * fits
    ok = fits & ((need == 0) | (need.cumsum(0) <= pages))
    ok &= (want * ok).cumsum(0) <= s["n_rows"]
    n, need = want * ok, need * ok
    first = need.cumsum(0) - need
    given = (col >= kept[:, None]) & (col < (kept + need)[:, None])
    which = pages - 1 - (first[:, None] + col - kept[:, None])
    table = torch.where(given, free[which.clamp(min=0, max=N)], s["table"])
    # the rows
    starts = torch.cat([n.new_zeros(1), n.cumsum(0)])
    row = torch.arange(s["n_rows"], device=dev)
    seq = torch.searchsorted(starts[1:], row, right=True)
    real = row < starts[-1]
    b = seq.clamp(max=B - 1)
    pos = keep[b] + row - starts[b]
    slot = table[b, (pos // PAGE).clamp(min=0, max=P - 1)].long() * PAGE + pos % PAGE
    i = lambda x: torch.where(real, x, torch.full_like(x, -1)).int()
    return ((keep + n).int(), n.int(), (pages - need.sum()).int(), table, free[:N], starts.int(), i(pos), i(seq), i(slot))


def _plain_sample(s):
    c, how = s["case"], s["how"]
    x = s["logits"].double()
    B, V = x.shape
    j = torch.arange(V, device=x.device)
    temp = how["temperature"].double()[:, None]
    top, order = torch.sort(x, dim=-1, descending=True, stable=True)
    w = torch.exp((top - top[:, :1]) / torch.where(temp > 0, temp, torch.ones_like(temp)))
    k = how["top_k"].long()[:, None]
    k = torch.where(k > 0, k, torch.full_like(k, V))
    k = torch.where(temp > 0, k, torch.ones_like(k))
    w = torch.where(j < k, w, torch.zeros_like(w))
    before = w.cumsum(-1) - w
    p, m = how["top_p"].double()[:, None], how["min_p"].double()[:, None]
    stays = (p >= 1) | (before < p * w.sum(-1, keepdim=True))
    stays &= w >= m
    stays[:, 0] = True
    w = torch.where(stays, w, torch.zeros_like(w))
    w = torch.zeros_like(w).scatter_(-1, order, w)
    cum = w.cumsum(-1)
    pick = (cum <= how["u"].double()[:, None] * cum[:, -1:]).sum(-1)
    token = torch.minimum(pick, V - 1 - (w > 0).flip(-1).long().argmax(-1)).int()
    return (token, (w / cum[:, -1:]).float()) if c["probs"] else token


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2605_19660_amd import binding as ob
        c = s["case"]
        if kind == "plan":
            p = ob.plan_step(s["lens"], s["want"], s["table"], s["free"], s["n_free"], n_rows=s["n_rows"], keep=s["keep"], **s["out"])
            return (p.lens, p.new_lens, p.n_free, s["table"], s["free"], p.row_starts, p.positions, p.row_seq, p.slots)
        if kind == "sample":
            token, probs = ob.sample(s["logits"], s["how"]["u"], temperature=s["how"]["temperature"],
                                     top_k=s["how"]["top_k"] if c["top_k"] else None,
                                     top_p=s["how"]["top_p"] if c["top_p"] < 1 else None,
                                     min_p=s["how"]["min_p"] if c["min_p"] else None, probs=c["probs"])
            return (token, probs) if c["probs"] else token
        if kind == "write":
            ob.q8_append(s["cache"], s["k_new"], s["v_new"], s["lens"], new_lens=s["new_lens"], row_starts=s["row_starts"],
                         max_new=c["tokens"])
        if kind in ("read", "write"):
            return ob.q8_read(s["cache"], s["lens"], starts=s["starts"], k=s["k"], v=s["v"])
        return ob.q8_attn(s["cache"], s["q"], s["lens"], new_lens=s["new_lens"], row_starts=s["row_starts"], max_new=c["tokens"],
                          out=s["out"], max_seq_len_hint=c["context"])
    return {"plan": _plain_plan, "write": _plain_write, "read": _plain_read, "attn": _plain_attn, "sample": _plain_sample}[kind](s)


# ---- what a pass cannot do without -------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    if kind == "plan":
        rows = c["batch"] + c["prompts"] * c["prompt"] / 2
        return {"bytes": int(c["batch"] * 24 + rows * 12 + rows / PAGE * 8), "flops": int(40 * c["batch"] + 10 * rows)}
    if kind == "sample":
        e = 4 if c["io"] == "f32" else 2
        n = c["batch"] * c["vocab"]
        return {"bytes": n * (e + 4 * c["probs"]) + 24 * c["batch"], "flops": 20 * n}
    share = 0.75 if c["ragged"] else 1.0                      # lengths are spread over context / 2 .. context
    B, T, hq, hk = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    coded = 2 * D + 8 / c["block"]                            # bytes of a token and kv head
    if kind == "read":
        n = B * min(T, c["context"] * share) * hk
        return {"bytes": int(n * (coded + 2 * D * (4 if c["out"] == "f32" else 2))), "flops": int(n * 2 * D)}
    if kind == "write":
        n = B * min(T, c["context"] * share) * hk
        return {"bytes": int(n * (coded + 2 * 2 * D * 2)), "flops": int(n * 6 * D)}
    rows = B * T * (0.4 if c["ragged"] and T > 1 else 1.0)
    cached = B * c["context"] * share * hk * coded
    return {"bytes": int(cached + 4 * rows * hq * D), "flops": int(4 * D * rows * hq * max(1, c["context"] * share - T / 2))}


# ---- the same in 64 bits, from the numbers before they are laid out ------------------------------

def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None
    if kind == "sample":
        return _exact_sample(case, seed)
    lens, new = _lengths(case, seed)
    if kind == "attn" and int((lens * new).sum()) * case["q_heads"] > 1 << 30:
        return None
    values = [_stands_for(x, lens, case["block"]) for x in _tokens(case, seed)]
    if kind == "attn":
        return _exact_attn(case, seed, lens, new, *values)
    starts = _starts(case, seed) if kind == "read" else lens - new
    out = []
    for x in values:
        y = torch.zeros(case["batch"], case["tokens"], case["kv_heads"], D, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            part = x[b, starts[b]:min(n, starts[b] + case["tokens"])]
            y[b, :len(part)] = part
        out.append(y)
    return tuple(out)


def _power(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _stands_for(x, lens, block):
    """What the cache holds of [batch, token, kv head, channel], in 64 bits: tokens of whole blocks rounded to
    four significant bits, or to multiples of 2^-9 of the block's scale below its normal numbers."""
    y = x.double()
    for b, n in enumerate(lens):
        n = int(n) // block * block
        z = y[b, :n].unflatten(0, (-1, block))
        top = z.abs().amax((1, 3), keepdim=True)
        scale = _power(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)))
        scale = torch.where(top > 0, scale, torch.ones_like(scale))
        r = z / scale
        step = _power(torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3)
        y[b, :n] = (torch.round(r / step) * step * scale).flatten(0, 1)
    return y


def _exact_attn(case, seed, lens, new, k, v):
    B, T, hq, hk = case["batch"], case["tokens"], case["q_heads"], case["kv_heads"]
    g = hq // hk
    q = _queries(case, seed).double()
    starts, n_rows = _rows_of(case, new)
    out = torch.zeros(n_rows, hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, m = int(lens[b]), int(new[b])
        if m == 0:
            continue
        row = b * T if starts is None else int(starts[b])
        later = torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None]
        for h in range(hq):
            logits = (q[b, :m, h] @ k[b, :n, h // g].t() / math.sqrt(D)).masked_fill(later, -math.inf)
            out[row:row + m, h] = torch.softmax(logits, -1) @ v[b, :n, h // g]
    return out.view(B, T, hq, D) if starts is None else out


def _exact_sample(case, seed):
    x, how = _logits(case, seed)
    x = x.double().cpu().numpy()
    temp, k, p, m, u = (how[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "u"))
    tokens, probs = [], np.zeros_like(x)
    for b, row in enumerate(x):
        order = np.argsort(-row, kind="stable")
        if temp[b] <= 0:
            order = order[:1]
        elif k[b] > 0:
            order = order[:int(k[b])]
        w = np.exp((row[order] - row[order[0]]) / (temp[b] if temp[b] > 0 else 1.0))
        if p[b] < 1:
            count = 1 + int(np.searchsorted(np.cumsum(w), p[b] * w.sum()))
            order, w = order[:count], w[:count]
        few = np.sort(order[w >= min(m[b], 1.0)])
        w = np.exp((row[few] - row.max()) / (temp[b] if temp[b] > 0 else 1.0))
        cum = np.cumsum(w)
        tokens.append(few[min(np.searchsorted(cum, u[b] * cum[-1], side="right"), len(few) - 1)])
        probs[b, few] = w / cum[-1]
    tokens = torch.tensor(tokens, dtype=torch.int32)
    return (tokens, torch.from_numpy(probs)) if case["probs"] else tokens
