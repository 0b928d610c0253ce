"""oscar_draft_attn held to what two-limb operands give: against attention in 64 bits over the cache's numbers, with
tolerances in which a single lost token shows, on caches whose values, steps and queries are far from 1."""
import numpy as np
import pytest

from cache_numbers import DT, filled_cache, hadamard, numbers, torch_type

pytestmark = pytest.mark.gpu

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# Relative to the sum of a product's absolute terms: every operand that is not exact is held to 2^-22 (two limbs of 11
# bits), a product of two of them is another 2^-21 off (its low limb rounds, low x low is left out), sums are 32 bits
# wide: 4 2^-22 and a dozen additions of 2^-24.
SUM = 2.0 ** -20
# A matrix instruction adds 32 products after cutting each at 2^-24 of the largest one, where a code's operand counts as
# 2^-14 whatever its bits: 2^6 above the code 1 at the lowest bit offset, 2^-20.  So each of the 32 is off by 2^-18 of
# the largest product of the instruction with a code of 1 (steps times 1 is at most what code and zero term together are).
CUT = 32 * 2.0 ** -18


def k_step_of_channel(bits):
    u = np.arange(128) % 32
    return 2 * (u // 16) + u % 8 // 4 if bits == 2 else u // 8


def largest_by_group(x, group):
    """x [.., n] added up over groups (numbers 0 .. of the n places), of each group its largest."""
    order = np.argsort(group, kind="stable")
    first = np.flatnonzero(np.diff(group[order], prepend=-1))
    return np.maximum.reduceat(x[..., order], first, axis=-1).sum(-1)


def attention(c, q, k_new, v_new, new_lens, io, leave_out=None):
    """The output in 64 bits and a bound of the kernel's distance per element.  leave_out: a token of every sequence
    that is not counted (a mistake on purpose)."""
    H = hadamard()
    scale = 1 / np.sqrt(128.0)
    B, T, hq, _ = q.shape
    g = hq // k_new.shape[2]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b, s in enumerate(numbers(c)):
        for h in range(hq):
            kv = h // g
            qr = q[b, :, h] @ H if c.cfg.rotation == 0 else q[b, :, h]
            n = s["n"][kv] * scale
            old = (qr @ (s["kc"][kv] + s["kb"][kv]).T) * n
            # (the rotation's own sum: 2^-22 of its absolute terms, handed on by every channel)
            k_size = np.abs(s["kc"][kv]) + np.abs(s["kb"][kv])
            e_old = (SUM * np.abs(qr) @ k_size.T +
                     CUT * largest_by_group(np.abs(qr)[:, None, :] * k_size, k_step_of_channel(c.cfg.bits)) +
                     2.0 ** -22 * np.outer(np.abs(q[b, :, h]).sum(1) / np.sqrt(128), np.abs(s["kc"][kv] + s["kb"][kv]).sum(1))) * n
            for t in range(T if new_lens is None else max(0, min(int(new_lens[b]), T))):
                new = (q[b, t, h] @ k_new[b, :t + 1, kv].T) * scale
                e_new = SUM * (np.abs(q[b, t, h]) @ np.abs(k_new[b, :t + 1, kv]).T) * scale
                lg = np.concatenate([old[t], new])
                e = np.concatenate([e_old[t], e_new]) + 2.0 ** -21 * (1 + np.abs(lg))   # fp32 logits and exponentials
                keep = np.ones(len(lg), bool)
                if leave_out is not None:
                    keep[leave_out] = False
                p = np.exp(lg - lg[keep].max()) * keep
                p /= p.sum()
                v = np.concatenate([s["vc"][kv] + s["vb"][kv], v_new[b, :t + 1, kv]])
                size = np.concatenate([np.abs(s["vc"][kv]) + np.abs(s["vb"][kv]), np.abs(v_new[b, :t + 1, kv])])
                o = p @ v
                # (values: 32 tokens an instruction, in a page those of one token / 4 % 4)
                i = np.arange(len(p))
                groups = i // 128 * 4 + np.where(i < (~s["window"]).sum(), i // 4 % 4, i // 32 % 4)
                d = (p * np.expm1(2 * e)) @ np.abs(v - o) + SUM * (p @ size)
                d += CUT * largest_by_group((p[:, None] * size).T, groups)
                out[b, t, h] = o
                tol[b, t, h] = d + (np.abs(o) + d) * HALF_STEP[io] + (2.0 ** -25 if io == "f16" else 0)
    return out, tol


def run(c, q, k, v, new_lens=None, splits=0, hint=None):
    import torch
    from paper_2605_19660_amd import binding as ob
    lens = None if new_lens is None else torch.tensor(new_lens, dtype=torch.int32, device="cuda")
    hint = int(c.seq_lens.max()) if hint is None else hint
    return ob.draft_attn(c, q, k, v, new_lens=lens, max_seq_len_hint=hint, num_splits=splits).double().cpu().numpy()


def check(c, q, k, v, io, new_lens=None, splits=(0,)):
    want, tol = attention(c, *(x.double().cpu().numpy() for x in (q, k, v)), new_lens, io)
    for s in splits:
        err = np.abs(run(c, q, k, v, new_lens, s) - want)
        far = (err / np.maximum(tol, 1e-300)).max()
        # A rounding is evenly spread over half a step: its square is a third of that one's square, or less, on
        # average, and within 15 % of that over ten thousand elements (0.62^2 = 1.15 / 3); the rest is below 2^-15.
        norm = np.linalg.norm(err) / np.linalg.norm(want)
        print("splits", s, "err / tol %.3f" % far, "rel %.2e" % norm, flush=True)
        assert np.isfinite(err).all() and far <= 1, (s, far, norm)
        assert norm <= 0.62 * HALF_STEP[io] + 2.0 ** -15, (s, far, norm)
    return want, tol


def new_tokens(c, T, io, seed=1, qmul=1.0, vmul=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    mk = lambda h, m: (torch.randn(c.batch, T, h, 128, generator=g) * m).to(torch_type(io)).cuda()
    return mk(c.cfg.n_q_heads, qmul), mk(c.cfg.n_kv_heads, 1.0), mk(c.cfg.n_kv_heads, vmul)


FORMATS = [(2, 128, 32, "f16", "f16", False), (4, 128, 32, "f16", "f16", False), (2, 32, 64, "f16", "f16", True),
           (4, 64, 128, "f16", "f16", True), (2, 64, 32, "bf16", "f16", False)]


@pytest.mark.parametrize("bits,kg,vg,io,meta,zp_min", FORMATS)
@pytest.mark.parametrize("T", [2, 5, 9])
def test_two_limbs(bits, kg, vg, io, meta, zp_min, T):
    c = filled_cache([700, 128, 1, 0, 383], hk=2, hq=8, bits=bits, kg=kg, vg=vg, io=io, meta=meta, zp_min=zp_min,
                     scattered=True, seed=bits * kg + vg)
    check(c, *new_tokens(c, T, io), io, splits=(1, 3))


@pytest.mark.parametrize("qmul", [0.01, 6.0])
def test_two_limbs_flat_and_sharp(qmul):
    c = filled_cache([900, 2500], hk=1, hq=4, io="f16")
    check(c, *new_tokens(c, 5, "f16", qmul=qmul), "f16", splits=(1, 4))


@pytest.mark.parametrize("n,at", [(130, 7), (700, 500), (1290, 1285)])
def test_a_lost_token_shows(n, at):
    """The tolerance is one in which leaving a single cached token out is seen, in pages and in the window: against an
    oracle that has lost it, some element is outside.  (The softmax is flat, so that every token has weight; beside one
    that takes nearly all, no 16-bit output shows another's loss.)"""
    c = filled_cache([n], hk=2, hq=4, io="bf16")
    check(c, *new_tokens(c, 3, "bf16"), "bf16")
    x = new_tokens(c, 3, "bf16", qmul=0.3)
    check(c, *x, "bf16")
    lost, tol = attention(c, *(y.double().cpu().numpy() for y in x), None, "bf16", leave_out=at)
    assert (np.abs(run(c, *x) - lost) > tol).any()


def appended(k, v, cfg, eager=True):
    """A cache holding k and v [batch, tokens, kv heads, 128] after one prompt."""
    import torch
    from paper_2605_19660_amd import binding as ob
    c = ob.Cache(cfg, k.shape[0], k.shape[1] // 128 + 1)
    dt = torch_type({v: n for n, v in DT.items()}[cfg.io_dtype])
    ob.quantize_append(c, *(torch.from_numpy(x.astype(np.float32)).to(dt).cuda() for x in (k, v)), eager=eager, max_seq_len_hint=0)
    return c


@pytest.mark.parametrize("gain", [1e-2, 1e-3, 3e-4])
@pytest.mark.parametrize("sharp", [12.0, 15.0])
@pytest.mark.parametrize("bits,vg", [(2, 32), (4, 128)])
def test_small_values_beside_a_token_that_takes_the_softmax(bits, vg, sharp, gain):
    """What the other tokens have left of the softmax keeps its bits, though their products with small value steps lie
    2^15 and more below the dominant token's probability; values of pages, window and new tokens."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(int(sharp))
    n, T = 1700, 2
    k, v = (rng.standard_normal((1, n, 2, 128)) for _ in range(2))
    d = rng.standard_normal((2, 128))
    d /= np.linalg.norm(d, axis=-1, keepdims=True)
    k[0, 5] = sharp * d
    v *= gain
    v[0, 5] *= 1e-3
    c = appended(k, v, ob.Config(2, 2, bits=bits, v_group=vg))
    q = np.sqrt(128) * d + 0.1 * rng.standard_normal((1, T, 2, 128))
    dev = lambda x: torch.from_numpy(x.astype(np.float32)).bfloat16().cuda()
    kn, vn = rng.standard_normal((1, T, 2, 128)), gain * rng.standard_normal((1, T, 2, 128))
    check(c, dev(q), dev(kn), dev(vn), "bf16", splits=(1, 2))


@pytest.mark.parametrize("growth", [3.0, 1 / 3.0])
@pytest.mark.parametrize("io,vg", [("bf16", 32), ("f16", 64)])
def test_values_that_grow_and_shrink_along_the_sequence(io, vg, growth):
    """Each page's values are three times (a third of) the page's before, and the groups' sizes differ by 2^9: what is
    summed is rescaled on the way, group by group."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(7)
    n, T = 1500, 3
    k, v = (rng.standard_normal((1, n, 1, 128)) for _ in range(2))
    v *= (growth ** (np.arange(n) // 128 - 6.0))[None, :, None, None] * (2.0 ** (-3 * (np.arange(128) // vg)))
    c = appended(k, v, ob.Config(4, 1, v_group=vg, io_dtype=DT[io]))
    x = new_tokens(c, T, io, vmul=0.1)
    check(c, *x, io, splits=(1, 3))


@pytest.mark.parametrize("kmul", [1e-3, 200.0])
@pytest.mark.parametrize("bits", [2, 4])
def test_keys_and_queries_of_opposite_sizes(bits, kmul):
    """Keys without a norm (their steps are their own size), and queries that bring the logits back to 1."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(9)
    k, v = rng.standard_normal((2, 400, 2, 128)) * kmul, rng.standard_normal((2, 400, 2, 128))
    c = appended(k, v, ob.Config(4, 2, bits=bits, io_dtype=ob.F16, scale_mode=ob.SCALE_NONE))
    q, kn, vn = new_tokens(c, 3, "f16", qmul=1 / kmul)
    check(c, q, kn, vn, "f16")


def test_large_new_and_window_values_in_bf16():
    """bf16 values beyond fp16's range are what they are."""
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([40, 300], hq=4, hk=2, gain=3e5, meta="f32")
    q, k, v = new_tokens(c, 5, "bf16", vmul=1e7)
    check(c, q, k, v, "bf16", splits=(1, 2))


@pytest.mark.parametrize("bits,kg,vg,zp_min", [(2, 128, 32, False), (4, 64, 128, True), (2, 32, 64, True), (4, 128, 32, False)])
@pytest.mark.parametrize("T", [2, 9])
def test_fp32_metadata_is_not_narrowed(bits, kg, vg, zp_min, T):
    c = filled_cache([700, 128, 0, 383], hk=2, hq=8, bits=bits, kg=kg, vg=vg, io="f16", meta="f32", zp_min=zp_min, seed=bits + kg)
    check(c, *new_tokens(c, T, "f16"), "f16", splits=(1, 3))


@pytest.mark.parametrize("gain", [1e-6, 1e-10, 1e6, 1e15])
@pytest.mark.parametrize("bits,vg", [(2, 32), (4, 128)])
def test_fp32_metadata_of_any_size(bits, vg, gain):
    """Steps below fp16's smallest number and above its largest."""
    c = filled_cache([520, 300], hk=2, hq=4, bits=bits, vg=vg, meta="f32", gain=gain)
    check(c, *new_tokens(c, 3, "bf16", vmul=gain), "bf16", splits=(1, 2))


@pytest.mark.parametrize("splits", [17, 52, 65, 512])
@pytest.mark.parametrize("hq,new_lens", [(4, [4, 2]), (14, [4, 3])])
def test_many_splits(splits, hq, new_lens):
    """Records of 17 .. 64 and of more splits, most of them of waves without a page; blocks of rows of one and two tiles."""
    c = filled_cache([1290, 300], hk=2, hq=hq, scattered=True)
    check(c, *new_tokens(c, 4, "bf16"), "bf16", new_lens=new_lens, splits=(splits,))


@pytest.mark.parametrize("hq,T", [(4, 3), (7, 5)])
def test_a_long_context_with_the_split_count_of_the_library(hq, T):
    from paper_2605_19660_amd import binding as ob
    c = filled_cache([33000], hk=1, hq=hq, io="f16")
    assert ob.draft_auto_splits(c.cfg, 1, T, 33000) > 16
    check(c, *new_tokens(c, T, "f16"), "f16")


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 1e38])
@pytest.mark.parametrize("T,splits", [(3, 1), (9, 2)])
def test_a_query_that_is_no_number_spoils_its_own_row_only(bad, T, splits):
    c = filled_cache([300, 140], hk=2, hq=8)
    q, k, v = new_tokens(c, T, "bf16")
    want, tol = attention(c, *(x.double().cpu().numpy() for x in (q, k, v)), None, "bf16")
    q[0, 1, 2, 5] = bad
    err = np.abs(run(c, q, k, v, None, splits) - want)
    err[0, 1, 2] = 0
    assert np.isfinite(err).all() and (err <= tol).all()
