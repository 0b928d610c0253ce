"""A decoding step with drafted tokens over the packed cache: its operators, for timing and for
comparing results.

A server that drafts tokens puts positions on the queries and keys of the last token and its drafts
(`rope`), attends from all of them over the packed cache and, causally, over themselves
(`draft_attn`), decides which drafts stand (`verify_drafts`) and appends the keys and values of those
(`quantize_append` with the counts); what the cache holds is read back for code that wants 16-bit
keys and values (`cache_read`).

With ``own`` set `run` makes the calls of ``paper_2605_19660_amd.binding``; without it the same
results come from elementary torch operations in 32 bits (64 for angles and for the sums that decide
a token), rounded once.  `exact` works in 64 bits from the quantized numbers themselves, before they
are packed into pages.
"""
import math

import numpy as np
import torch

own = False

D = R = 128
IO = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"f32": 0, "bf16": 1, "f16": 2}
HEADS = [(32, 8), (28, 4), (8, 8), (16, 2), (20, 4), (6, 2)]

CACHE = {"batch": 1, "context": 1000, "q_heads": 32, "kv_heads": 8, "bits": 2, "k_group": 128,
         "v_group": 32, "io": "bf16", "meta": "f16", "zp_min": False, "ragged": False, "scattered": False}
ROPE = {"kind": "rope", "tokens": 1, "q_heads": 32, "kv_heads": 8, "io": "bf16", "axes": 1, "interleaved": False,
        "rotary": 128, "adjacent": False, "inverse": False, "fused": False, "first": 1000}
READ = {"kind": "read", "tokens": 1000, "out": "bf16", **CACHE}
DRAFT = {"kind": "draft", "tokens": 4, **CACHE}
VERIFY = {"kind": "verify", "batch": 1, "drafts": 4, "vocab": 32000, "io": "f32", "ragged": False}


def listed():
    return [
        # one user's next token: launch and latency are all there is
        {**ROPE, "name": "rope-1-token"},
        # a long mixed prompt, positions in time, height and width dealt out pair by pair, q and k as the
        # projection left them, beside v in one matrix
        {**ROPE, "name": "rope-32k-three-axes-fused", "tokens": 32768, "q_heads": 28, "kv_heads": 4, "axes": 3,
         "interleaved": True, "fused": True, "first": 0},
        # an fp32 model with partial rotary: positions taken off again (also the gradient's direction)
        {**ROPE, "name": "rope-2999-f32-inverse", "tokens": 2999, "io": "f32", "rotary": 64, "adjacent": True,
         "inverse": True, "first": 120000},
        # one user's short history
        {**READ, "name": "read-b1-1k"},
        # the largest: a batch of long contexts handed to 16-bit code
        {**READ, "name": "read-b4-32k", "batch": 4, "context": 32768, "tokens": 32768},
        # pieces out of the middle of ragged 4-bit caches with the finer groups, pages in any order, fp32 out
        {**READ, "name": "read-b8-900-of-4k-int4", "batch": 8, "context": 4096, "tokens": 900, "bits": 4, "k_group": 32,
         "io": "f16", "out": "f32", "ragged": True, "scattered": True},
        # one user, three drafts behind the last token
        {**DRAFT, "name": "draft-b1-1k-t4"},
        # the batched server, seven drafts
        {**DRAFT, "name": "draft-b8-32k-t8", "batch": 8, "context": 32768, "tokens": 8},
        # one very long document, seven query heads a kv head, four drafts, groups of 32 tokens
        {**DRAFT, "name": "draft-b1-128k-g7-t5", "context": 131001, "tokens": 5, "q_heads": 28, "kv_heads": 4, "k_group": 32},
        # a piece of a prompt attending over 4-bit ragged caches before it is appended
        {**DRAFT, "name": "draft-b2-8k-t500-int4-f16", "batch": 2, "context": 8100, "tokens": 500, "bits": 4, "io": "f16",
         "ragged": True, "scattered": True},
        # verification for one user, and for a batch with a large vocabulary and ragged drafts
        {**VERIFY, "name": "verify-b1-32000"},
        {**VERIFY, "name": "verify-b64-128003-ragged", "batch": 64, "drafts": 7, "vocab": 128003, "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "read", "read", "draft", "draft", "draft", "verify"])
    heads = rng.choice(HEADS)
    if kind == "rope":
        axes = rng.choice([1, 1, 2, 3, 4])
        return {**ROPE, "tokens": _log_int(rng, 1, 30000), "q_heads": heads[0], "kv_heads": heads[1],
                "io": rng.choice(["bf16", "bf16", "f16", "f32"]), "axes": axes,
                "interleaved": rng.random() < 0.5, "rotary": rng.choice([128, 128, 64, 32, 90]),
                "adjacent": rng.random() < 0.3, "inverse": rng.random() < 0.2, "fused": rng.random() < 0.5,
                "first": rng.choice([0, 1000, 131072, 1000000])}
    if kind == "verify":
        drafts = rng.randint(1, 12)
        vocab = _log_int(rng, 1000, 200000)
        return {**VERIFY, "batch": _log_int(rng, 1, min(64, max(1, 60000000 // (vocab * drafts)) + 1)),
                "drafts": drafts, "vocab": vocab, "io": rng.choice(["f32", "f32", "bf16", "f16"]),
                "ragged": rng.random() < 0.5}
    c = {"q_heads": heads[0], "kv_heads": heads[1], "bits": rng.choice([2, 2, 4]), "k_group": rng.choice([128, 128, 32, 64]),
         "v_group": rng.choice([32, 32, 64, 128]), "io": rng.choice(["bf16", "bf16", "f16"]),
         "meta": rng.choice(["f16", "f16", "f32"]), "zp_min": rng.random() < 0.2, "ragged": rng.random() < 0.5,
         "scattered": rng.random() < 0.5}
    # 1 .. 131072 tokens a sequence, 1 .. 64 sequences, at most half the largest cache
    c["context"] = rng.choice([1, 127, _log_int(rng, 100, 131072), _log_int(rng, 100, 131072), _log_int(rng, 100, 131072)])
    most = 131072 * 8 // heads[1] // 2
    c["batch"] = min(64, _log_int(rng, 1, max(1.01, most / c["context"])))
    if kind == "read":
        return {**READ, **c, "tokens": c["context"] if rng.random() < 0.5 else _log_int(rng, 1, c["context"]),
                "out": rng.choice([c["io"], "f32"])}
    c["tokens"] = _log_int(rng, 1, 16) if rng.random() < 0.7 else _log_int(rng, 16, 600)
    # the logits of the plain form are held whole
    while c["batch"] > 1 and c["batch"] * heads[0] * c["tokens"] * (c["context"] + c["tokens"]) > 1 << 29:
        c["batch"] //= 2
    while c["tokens"] > 1 and c["batch"] * heads[0] * c["tokens"] * (c["context"] + c["tokens"]) > 1 << 29:
        c["tokens"] //= 2
    return {**DRAFT, **c}


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 64 + what)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _lengths(case, seed):
    """Tokens and window tokens of every sequence: after a prompt the window holds what is left of the
    last block, after a decoding step a full block can still wait in it."""
    rng = np.random.default_rng([seed, 1])
    n = np.full(case["batch"], case["context"])
    if case["ragged"]:
        n = rng.integers(max(1, case["context"] // 2), case["context"] + 1, size=case["batch"])
        n[rng.integers(case["batch"])] = case["context"]
    res = n % R
    res[(res == 0) & (rng.random(case["batch"]) < 0.5)] = R
    return n, res


def _quantize(x, bits, dim, meta, zp_min):
    """Codes, step and zero of x over `dim`, the parameters rounded to the metadata's type."""
    lo, hi = x.amin(dim, keepdim=True), x.amax(dim, keepdim=True)
    step = (hi - lo) / (2 ** bits - 1)
    step = torch.where(step > 0, step, torch.ones_like(step)).to(meta).float()
    zero = lo.to(meta).float() if zp_min else torch.round(-lo / step).to(meta).float()
    codes = (x - zero) / step if zp_min else x / step + zero
    return torch.round(codes).clamp(0, 2 ** bits - 1).to(torch.uint8), step, zero


def _history(case, seed):
    """What the cache holds, as numbers: codes [batch, page, kv head, token, channel] with their
    parameters, and the window."""
    g = _gen(seed, 1)
    B, H, bits = case["batch"], case["kv_heads"], case["bits"]
    meta = IO[case["meta"]]
    n, res = _lengths(case, seed)
    pages = int(((n - res) // R).max())
    P = max(pages, 1)
    h = {"lens": n, "res": res, "pages": P}
    k = _randn(g, B, P, H, R, D)
    k /= k.norm(dim=-1, keepdim=True)
    G = case["k_group"]
    codes, step, zero = _quantize(k.view(B, P, H, R // G, G, D), bits, 4, meta, case["zp_min"])
    del k
    h["k_codes"], h["k_step"], h["k_zero"] = codes.view(B, P, H, R, D), step[:, :, :, :, 0], zero[:, :, :, :, 0]
    h["k_norm"] = (torch.exp(0.5 * _randn(g, B, P, H, R)) * math.sqrt(D)).to(meta).float()
    gain = torch.ones(H, D, device="cuda")
    gain[:, ::37] = 8.0                                       # outlier channels
    v = _randn(g, B, P, H, R, D)
    v *= torch.exp(0.5 * _randn(g, B, P, 1, R, 1))
    v *= gain[:, None, :]
    G = case["v_group"]
    codes, step, zero = _quantize(v.view(B, P, H, R, D // G, G), bits, 5, meta, case["zp_min"])
    del v
    h["v_codes"], h["v_step"], h["v_zero"] = codes.view(B, P, H, R, D), step[..., 0], zero[..., 0]
    rk = _randn(g, B, H, R, D)
    h["res_k"] = (rk / rk.norm(dim=-1, keepdim=True)).to(torch.float16)
    h["res_norm"] = (torch.exp(0.5 * _randn(g, B, H, R)) * math.sqrt(D)).to(meta)
    h["res_v"] = (_randn(g, B, H, R, D) * gain[:, None, :]).to(IO[case["io"]])
    return h


def _slots(bits):
    """Order of 32 codes in a chunk: position kk * 8 + e of the operand holds code number slot."""
    kk, e = np.meshgrid(np.arange(4), np.arange(8), indexing="ij")
    s = 16 * (kk // 2) + 4 * (kk % 2) + e // 2 + 8 * (e % 2) if bits == 2 else 8 * kk + e // 2 + 4 * (e % 2)
    return s


def _pack_bits(u, bits):
    """[..., 32] codes to [..., 4 * bits] bytes, code number u at bit u * bits."""
    per = 8 // bits
    w = u.view(*u.shape[:-1], 32 // per, per)
    shift = torch.arange(per, device=u.device, dtype=torch.uint8) * bits
    return (w << shift).sum(-1, dtype=torch.uint8)


def _pack(case, h, seed):
    """The page pools as the library lays them out, and the block table."""
    B, P, H, bits = case["batch"], h["pages"], case["kv_heads"], case["bits"]
    meta = IO[case["meta"]]
    slots = _slots(bits)
    chan = torch.from_numpy((32 * np.arange(4)[:, None] + slots.reshape(-1)[None]).reshape(-1)).cuda()
    tok = (torch.arange(R).view(8, 16).t().reshape(-1)).cuda()            # position (t % 16) * 8 + t / 16
    # keys: [page][tile pair][n][quarter][tile of the pair][code]
    x = h["k_codes"].view(B * P, H, 4, 2, 16, 4, 32).permute(0, 1, 2, 4, 5, 3, 6).contiguous()
    k_codes = _pack_bits(x, bits).view(B * P, H, -1)
    # values: [page][tile pair][n][token % 4][tile of the pair][code], token 16 e + 4 kk + quarter
    x = h["v_codes"].view(B * P, H, 8, 4, 4, 4, 2, 16)                     # e kk q4 | pair tile n
    x = x.permute(0, 1, 5, 7, 4, 6, 3, 2).reshape(B * P, H, 4, 16, 4, 2, 32)
    back = torch.from_numpy(np.argsort(slots.reshape(-1))).cuda()
    v_codes = _pack_bits(x[..., back].contiguous(), bits).view(B * P, H, -1)
    k_meta = torch.stack([h["k_step"], h["k_zero"]], 3).to(meta)[..., chan].contiguous()
    v_meta = torch.stack([h["v_step"], h["v_zero"]], 3).to(meta)             # [B, P, H, 2, token, group]
    v_meta = v_meta.transpose(-1, -2)[..., tok].contiguous()
    k_norms = h["k_norm"].to(meta)[..., tok].contiguous()
    total = B * P
    perm = np.random.default_rng([seed, 4]).permutation(total) if case["scattered"] else np.arange(total)
    at = torch.from_numpy(np.argsort(perm)).cuda()                          # logical page held by a physical one
    raw = lambda t: t.view(total, -1).view(torch.uint8)[at].contiguous().view(-1)
    return {"k_codes": raw(k_codes), "k_meta": raw(k_meta), "k_norms": raw(k_norms), "v_codes": raw(v_codes),
            "v_meta": raw(v_meta), "res_k": h["res_k"], "res_v": h["res_v"], "res_norm": h["res_norm"],
            "block_table": torch.from_numpy(perm.astype(np.int32).reshape(B, P)).cuda(),
            "seq_lens": torch.from_numpy(h["lens"].astype(np.int32)).cuda(),
            "res_lens": torch.from_numpy(h["res"].astype(np.int32)).cuda()}


def _handle(case, pools):
    """The library's cache object over these pools, which a program keeps beside them."""
    from paper_2605_19660_amd import binding as ob
    B, P = pools["block_table"].shape
    cfg = ob.Config(case["q_heads"], case["kv_heads"], bits=case["bits"], k_group=case["k_group"], v_group=case["v_group"],
                    io_dtype=CODE[case["io"]], meta_dtype=CODE[case["meta"]],
                    zp_mode=ob.ZP_MIN if case["zp_min"] else ob.ZP_INT)
    cache = ob.Cache(cfg, B, P)
    for name, t in pools.items():
        dst = getattr(cache, name)
        dst.copy_(t.view(torch.uint8).view(-1) if dst.dtype == torch.uint8 else t)
    return cache


def _starts(case, seed):
    n, _ = _lengths(case, seed)
    rng = np.random.default_rng([seed, 5])
    return np.array([rng.integers(0, max(1, x - case["tokens"] + 1)) for x in n], np.int32)


def _axis_of_pair(case):
    pairs, axes = case["rotary"] // 2, case["axes"]
    if case["interleaved"]:
        return np.arange(pairs) % axes
    share = np.full(axes, pairs // axes)
    share[0] += pairs - share.sum()
    return np.repeat(np.arange(axes), share)


def _rope_inputs(case, seed):
    g = _gen(seed, 2)
    n, hq, hk, io = case["tokens"], case["q_heads"], case["kv_heads"], IO[case["io"]]
    if case["fused"]:
        x = _randn(g, n, (hq + 2 * hk) * D).to(io)
        q, k = x[:, :hq * D].view(n, hq, D), x[:, hq * D:(hq + hk) * D].view(n, hk, D)
    else:
        q, k = _randn(g, n, hq, D).to(io), _randn(g, n, hk, D).to(io)
    rng = np.random.default_rng([seed, 6])
    pos = case["first"] + np.arange(n) + rng.integers(0, 100)
    pos = np.stack([pos] + [case["first"] + rng.integers(0, 400, size=n) for _ in range(case["axes"] - 1)])
    r = case["rotary"]
    inv = (10000.0 ** (-np.arange(0, r, 2) / r)).astype(np.float32)
    return q, k, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(inv).cuda()


def _probabilities(case, seed):
    g = _gen(seed, 3)
    B, T, V, io = case["batch"], case["drafts"], case["vocab"], IO[case["io"]]
    logits = _randn(g, B, T + 1, V) * 3.0
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :T] + 0.7 * _randn(g, B, T, V), -1)
    del logits
    u = torch.rand(B, T, 1, device="cuda", generator=g, dtype=torch.float64)
    cum = q.double().cumsum(-1)
    drafts = torch.searchsorted(cum, u * cum[..., -1:], right=True).clamp(max=V - 1).view(B, T).int()
    lens = None
    if case["ragged"]:
        lens = torch.from_numpy(np.random.default_rng([seed, 7]).integers(0, T + 1, size=B).astype(np.int32)).cuda()
    u = torch.rand(B, T + 1, device="cuda", generator=g)
    return p.to(io), q.to(io), drafts, u, lens


def prepare(case, seed):
    kind = case["kind"]
    if kind == "rope":
        q, k, pos, inv = _rope_inputs(case, seed)
        axes = _axis_of_pair(case)
        return {"case": case, "q": q, "k": k, "pos": pos, "inv_freq": inv, "axes": bytes(axes.tolist()),
                "axis_index": torch.from_numpy(axes).cuda()}
    if kind == "verify":
        p, q, drafts, u, lens = _probabilities(case, seed)
        return {"case": case, "p": p, "q": q, "drafts": drafts, "u": u, "lens": lens}
    pools = _pack(case, _history(case, seed), seed)
    s = {"case": case, "pools": pools, "slots": torch.from_numpy(_slots(case["bits"]).reshape(-1)).cuda(),
         "hadamard": _hadamard(torch.float32)}
    if own:
        s["cache"] = _handle(case, pools)
        s["pools"] = None
    B, T, hq, hk, io = case["batch"], case["tokens"], case["q_heads"], case["kv_heads"], IO[case["io"]]
    if kind == "read":
        s["starts"] = torch.from_numpy(_starts(case, seed)).cuda()
        s["k"] = torch.zeros(B, T, hk, D, device="cuda", dtype=IO[case["out"]])
        s["v"] = torch.zeros_like(s["k"])
        return s
    s.update(_draft_inputs(case, seed))
    return s


def _draft_inputs(case, seed):
    g = _gen(seed, 4)
    B, T, hq, hk, io = case["batch"], case["tokens"], case["q_heads"], case["kv_heads"], IO[case["io"]]
    new = None
    if case["ragged"]:
        new = torch.from_numpy(np.random.default_rng([seed, 8]).integers(0, T + 1, size=B).astype(np.int32)).cuda()
    return {"q": _randn(g, B, T, hq, D).to(io), "k_new": _randn(g, B, T, hk, D).to(io), "v_new": _randn(g, B, T, hk, D).to(io),
            "new_lens": new}


# ---- one pass ----------------------------------------------------------------------------------

def _hadamard(dtype):
    i = torch.arange(D, device="cuda")
    bits = i[:, None] & i[None, :]
    odd = sum((bits >> s) & 1 for s in range(7)) % 2
    return (1 - 2 * odd).to(dtype) / math.sqrt(D)


def _unpack_bits(b, bits):
    per = 8 // bits
    shift = torch.arange(per, device=b.device, dtype=torch.uint8) * bits
    return ((b[..., None] >> shift) & (2 ** bits - 1)).flatten(-2)


def _dequantized(s):
    """Every sequence's packed and window tokens in 32 bits, keys in the rotated basis with their norms:
    [batch, kv head, token, channel] with the window behind the pages, and which places hold a token."""
    c, t = s["case"], s["pools"]
    B, P = t["block_table"].shape
    H, bits, meta = c["kv_heads"], c["bits"], IO[c["meta"]]
    page = t["block_table"].long().view(-1)
    take = lambda name: t[name].view(B * P, H, -1)[page]
    slots = s["slots"]
    back = torch.argsort(slots)
    x = _unpack_bits(take("k_codes").view(B * P, H, 4, 16, 4, 2, 4 * bits), bits)
    codes = x.permute(0, 1, 2, 5, 3, 4, 6).reshape(B, P, H, R, D)
    m = take("k_meta").view(meta).view(B, P, H, 2, R // c["k_group"], 4, 32)[..., back].flatten(-2).float()
    step, zero = (y.repeat_interleave(c["k_group"], 3) for y in m.unbind(3))
    k = codes.float() * step + zero if c["zp_min"] else (codes.float() - zero) * step
    norm = take("k_norms").view(meta).view(B, P, H, 16, 8).transpose(-1, -2).reshape(B, P, H, R).float()
    k *= norm[..., None]
    x = _unpack_bits(take("v_codes").view(B * P, H, 4, 16, 4, 2, 4 * bits), bits)[..., slots]
    codes = x.view(B * P, H, 4, 16, 4, 2, 4, 8).permute(0, 1, 7, 6, 4, 2, 5, 3).reshape(B, P, H, R, D)
    m = take("v_meta").view(meta).view(B, P, H, 2, D // c["v_group"], 16, 8).transpose(-1, -2).flatten(-2).float()
    step, zero = (y.transpose(-1, -2).repeat_interleave(c["v_group"], 4) for y in m.unbind(3))
    v = codes.float() * step + zero if c["zp_min"] else (codes.float() - zero) * step
    k = torch.cat([k.transpose(1, 2).reshape(B, H, P * R, D), t["res_k"].float() * t["res_norm"].float()[..., None]], 2)
    v = torch.cat([v.transpose(1, 2).reshape(B, H, P * R, D), t["res_v"].float()], 2)
    i = torch.arange((P + 1) * R, device=k.device)
    packed = (t["seq_lens"] - t["res_lens"])[:, None]
    held = torch.where(i < P * R, i < packed, i - P * R < t["res_lens"][:, None])
    return k, v, held, packed


def _plain_read(s):
    c = s["case"]
    k, v, _, packed = _dequantized(s)
    B, T, P = c["batch"], c["tokens"], s["pools"]["block_table"].shape[1]
    k = torch.matmul(k, s["hadamard"])
    at = s["starts"].long()[:, None] + torch.arange(T, device=k.device)
    there = at < s["pools"]["seq_lens"][:, None]
    at = torch.where(at < packed, at, at - packed + P * R).clamp(max=(P + 1) * R - 1)
    pick = lambda x: torch.where(there[:, :, None, None], x.transpose(1, 2)[torch.arange(B, device=k.device)[:, None], at],
                                 torch.zeros((), device=k.device)).to(IO[c["out"]])
    return pick(k), pick(v)


def _plain_draft(s):
    c = s["case"]
    k, v, held, _ = _dequantized(s)
    B, T, hq, hk = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    g, scale = hq // hk, 1 / math.sqrt(D)
    q = s["q"].float().view(B, T, hk, g, D).permute(0, 2, 1, 3, 4).reshape(B, hk, T * g, D)
    k_new, v_new = (s[n].float().transpose(1, 2) for n in ("k_new", "v_new"))
    old = torch.matmul(torch.matmul(q, s["hadamard"]), k.transpose(-1, -2)) * scale
    old.masked_fill_(~held[:, None, None, :], float("-inf"))
    new = torch.matmul(q, k_new.transpose(-1, -2).contiguous()) * scale
    t = torch.arange(T, device=q.device)
    new.masked_fill_((t[None, :] > t[:, None]).repeat_interleave(g, 0), float("-inf"))
    p = torch.softmax(torch.cat([old, new], -1), -1)
    v = torch.where(held[:, None, :, None], v, torch.zeros((), device=v.device))
    out = torch.matmul(p[..., :old.shape[-1]], v) + torch.matmul(p[..., old.shape[-1]:], v_new)
    out = out.view(B, hk, T, g, D).permute(0, 2, 1, 3, 4).reshape(B, T, hq, D)
    if s["new_lens"] is not None:
        out = out * (t < s["new_lens"][:, None])[:, :, None, None]
    return out.to(IO[c["io"]])


def _plain_rope(s):
    c = s["case"]
    r = c["rotary"]
    angle = s["pos"].double()[s["axis_index"]].t() * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin

    def turn(x):
        y = x.float()
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["adjacent"] else (y[..., :r // 2], y[..., r // 2:r])
        a, b = a * cos - b * sin, b * cos + a * sin
        ab = torch.stack([a, b], -1).flatten(-2) if c["adjacent"] else torch.cat([a, b], -1)
        return torch.cat([ab, y[..., r:]], -1).to(x.dtype)
    return turn(s["q"]), turn(s["k"])


def _plain_verify(s):
    p, q, drafts, u, lens = s["p"], s["q"], s["drafts"], s["u"], s["lens"]
    B, T, V = q.shape
    t = torch.arange(T, device=p.device)
    n = torch.full((B,), T, device=p.device) if lens is None else lens.long()
    x = drafts.long()[..., None]
    px, qx = (y.gather(-1, x)[..., 0].double() for y in (p[:, :T], q))
    stands = (u[:, :T].double() * qx < px) & (t < n[:, None])
    a = stands.long().cumprod(1).sum(1)
    b = torch.arange(B, device=p.device)
    target = p[b, a].double()
    rest = (target - q[b, a.clamp(max=T - 1)].double() * (a < n)[:, None]).clamp(min=0)
    w = torch.where(rest.sum(-1, keepdim=True) > 0, rest, target)
    cum = w.cumsum(-1)
    pick = (cum <= u[:, T:].double() * cum[:, -1:]).sum(-1)
    pick = torch.minimum(pick, V - 1 - (w > 0).flip(-1).long().argmax(-1)).int()
    tokens = torch.cat([torch.where(t < a[:, None], drafts, torch.full_like(drafts, -1)),
                        torch.full((B, 1), -1, device=p.device, dtype=torch.int32)], 1)
    tokens[b, a] = pick
    return (a + 1).int(), tokens


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        from paper_2605_19660_amd import binding as ob
        c = s["case"]
        if kind == "rope":
            return ob.rope(s["q"], s["k"], s["pos"], s["inv_freq"], axes=s["axes"], adjacent=c["adjacent"], inverse=c["inverse"])
        if kind == "read":
            return ob.cache_read(s["cache"], s["starts"], k=s["k"], v=s["v"])
        if kind == "draft":
            return ob.draft_attn(s["cache"], s["q"], s["k_new"], s["v_new"], new_lens=s["new_lens"],
                                 max_seq_len_hint=c["context"])
        return ob.verify_drafts(s["p"], s["q"], s["drafts"], s["u"], draft_lens=s["lens"])
    return {"rope": _plain_rope, "read": _plain_read, "draft": _plain_draft, "verify": _plain_verify}[kind](s)


# ---- what a pass cannot do without -------------------------------------------------------------

def _page_bytes(c):
    m = 4 if c["meta"] == "f32" else 2
    return 2 * R * D * c["bits"] // 8 + 2 * (R // c["k_group"]) * D * m + R * m + 2 * (D // c["v_group"]) * R * m


def work(case):
    c, kind = case, case["kind"]
    if kind == "rope":
        n, h, e = c["tokens"], c["q_heads"] + c["kv_heads"], 4 if c["io"] == "f32" else 2
        return {"bytes": 2 * n * h * D * e + 4 * n * c["axes"] + 2 * c["rotary"], "flops": 3 * n * h * c["rotary"]}
    if kind == "verify":
        # one row of the target and one of the draft a sequence decide its token
        B, T, V, e = c["batch"], c["drafts"], c["vocab"], 4 if c["io"] == "f32" else 2
        return {"bytes": 2 * B * V * e + B * (2 * T * e + 4 * T + 4 * (T + 1) + 4 * (T + 2)), "flops": 3 * B * V}
    share = 0.75 if c["ragged"] else 1.0                      # lengths are spread over context / 2 .. context
    B, T, hq, hk = c["batch"], c["tokens"], c["q_heads"], c["kv_heads"]
    if kind == "read":
        n = B * min(T, c["context"] * share) * hk
        e = 4 if c["out"] == "f32" else 2
        return {"bytes": int(n * (_page_bytes(c) / R + 2 * D * e)), "flops": int(n * (7 * D + 4 * D))}
    rows = B * T * hq * (0.5 if c["ragged"] else 1.0)
    cached = B * c["context"] * share * hk * _page_bytes(c) / R
    return {"bytes": int(cached + 2 * (2 * rows * D + 2 * B * T * hk * D)),
            "flops": int(4 * D * rows * (c["context"] * share + (T + 1) / 2))}


# ---- the same in 64 bits, from the numbers before they are packed --------------------------------

def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None
    if kind == "rope":
        return _exact_rope(case, seed)
    h = _history(case, seed)
    if case["batch"] * case["kv_heads"] * h["pages"] > 16384 and kind == "draft" and case["tokens"] > 64:
        return None
    return _exact_read(case, seed, h) if kind == "read" else _exact_draft(case, seed, h)


def _exact_rope(case, seed):
    q, k, pos, inv = _rope_inputs(case, seed)
    r, half = case["rotary"], case["rotary"] // 2
    axis = _axis_of_pair(case)
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                       (-1 if case["inverse"] else 1) * pos.double()[torch.from_numpy(axis).cuda()].t() * inv.double())
    first = torch.arange(0, r, 2) if case["adjacent"] else torch.arange(half)
    second = first + (1 if case["adjacent"] else half)
    out = []
    for x in (q, k):
        y = x.double().clone()
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _tokens_64(case, h, b):
    """Keys (rotated basis, with norms) and values of sequence b, [kv head, token, channel], 64 bits."""
    n = int(h["lens"][b] - h["res"][b]) // R
    kg, vg = case["k_group"], case["v_group"]
    kc, vc = h["k_codes"][b, :n].double(), h["v_codes"][b, :n].double()
    kc, vc = kc.unflatten(2, (-1, kg)), vc.unflatten(3, (-1, vg))
    ks, kz = h["k_step"][b, :n].double()[:, :, :, None], h["k_zero"][b, :n].double()[:, :, :, None]
    vs, vz = h["v_step"][b, :n].double()[..., None], h["v_zero"][b, :n].double()[..., None]
    k = (ks * kc + kz if case["zp_min"] else ks * (kc - kz)).flatten(2, 3) * h["k_norm"][b, :n].double()[..., None]
    v = (vs * vc + vz if case["zp_min"] else vs * (vc - vz)).flatten(3, 4)
    r = int(h["res"][b])
    k, v = (x.transpose(0, 1).flatten(1, 2) for x in (k, v))
    return (torch.cat([k, (h["res_k"][b].double() * h["res_norm"][b].double()[..., None])[:, :r]], 1),
            torch.cat([v, h["res_v"][b, :, :r].double()], 1))


def _exact_read(case, seed, h):
    B, T, H = case["batch"], case["tokens"], case["kv_heads"]
    starts = _starts(case, seed)
    ko = torch.zeros(B, T, H, D, device="cuda", dtype=torch.float64)
    vo = torch.zeros_like(ko)
    had = _hadamard(torch.float64)
    for b in range(B):
        k, v = (x[:, starts[b]:starts[b] + T].transpose(0, 1) for x in _tokens_64(case, h, b))
        ko[b, :k.shape[0]], vo[b, :v.shape[0]] = torch.matmul(k, had), v
    return ko, vo


def _exact_draft(case, seed, h):
    d = _draft_inputs(case, seed)
    B, T, hq, hk = case["batch"], case["tokens"], case["q_heads"], case["kv_heads"]
    g = hq // hk
    out = torch.zeros(B, T, hq, D, device="cuda", dtype=torch.float64)
    had = _hadamard(torch.float64)
    behind = torch.ones(T, T, device="cuda", dtype=torch.bool).triu(1).repeat_interleave(g, 0)
    for b in range(B):
        n = T if d["new_lens"] is None else int(d["new_lens"][b])
        k, v = _tokens_64(case, h, b)
        for kv in range(hk):
            q = d["q"][b].double()[:, kv * g:(kv + 1) * g].reshape(T * g, D)
            own_logits = (q @ d["k_new"][b, :, kv].double().t()).masked_fill(behind, -math.inf)
            logits = torch.cat([(q @ had) @ k[kv].t(), own_logits], 1) / math.sqrt(D)
            e = torch.exp(logits - logits.amax(1, keepdim=True))
            o = e @ torch.cat([v[kv], d["v_new"][b, :, kv].double()]) / e.sum(1, keepdim=True)
            out[b, :n, kv * g:(kv + 1) * g] = o.view(T, g, D)[:n]
    return out
