"""What a cache holds, as 64-bit numbers by kv head and token, read through oscar_debug_dump (the layout-free
copy): for the tests of the calls that read the packed pages."""
import numpy as np

DT = {"f32": 0, "bf16": 1, "f16": 2}


def torch_type(io):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[io]


def hadamard():
    i = np.arange(128)
    odd = np.array([bin(x).count("1") % 2 for x in range(128)])
    return (1.0 - 2.0 * odd[i[:, None] & i[None, :]]) / np.sqrt(128.0)


def filled_cache(lens, steps=(), hq=4, hk=2, bits=2, kg=128, vg=32, io="bf16", meta="f16", zp_min=False, scattered=False,
                 pages=None, seed=0, gain=1.0, poison=True, rotation=True, scale=0, norm_scope=0):
    """A cache after a ragged prompt of `lens` tokens and one decoding append per entry of `steps` (tokens a
    sequence).  poison: what no token owns is NaN (fp16 / bf16 / fp32 pattern 0x7fff... / codes all set)."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    B = len(lens)
    pages = pages or int(lens.max() + sum(max(s) for s in steps)) // 128 + 1
    cfg = ob.Config(hq, hk, bits=bits, k_group=kg, v_group=vg, io_dtype=DT[io], meta_dtype=DT[meta],
                    zp_mode=ob.ZP_MIN if zp_min else ob.ZP_INT, rotation=ob.ROTATION_ON if rotation else ob.ROTATION_OFF,
                    scale_mode=scale, norm_scope=norm_scope)
    perm = rng.permutation(B * pages) if scattered else None
    c = ob.Cache(cfg, B, pages, page_perm=perm)
    if poison:
        for name in ("k_codes", "k_meta", "k_norms", "v_codes", "v_meta", "res_k", "res_v", "res_norm"):
            getattr(c, name).view(torch.int16).fill_(0x7fff)

    def new(T):
        m = np.exp(0.5 * rng.standard_normal((B, T, 1, 1)))
        return [torch.from_numpy((rng.standard_normal((B, T, hk, 128)) * m * g).astype(np.float32)).to(torch_type(io)).cuda()
                for g in (1.0, gain)]
    if lens.max() > 0:
        k, v = new(int(lens.max()))
        ob.quantize_append(c, k, v, new_lens=torch.from_numpy(lens).cuda(), eager=True, max_seq_len_hint=0)
    for s in steps:
        s = np.asarray(s, np.int32)
        k, v = new(int(s.max()))
        ob.quantize_append(c, k, v, new_lens=torch.from_numpy(s).cuda())
    return c


def numbers(c):
    """Per sequence: keys = n (kc + kb) in the cache's own basis, values = vc + vb, [kv head, token, channel];
    kc, vc are what the codes carry (the 16-bit number itself in the window), kb, vb the zero terms; `window` marks
    the window's tokens."""
    from paper_2605_19660_amd import binding as ob
    cfg, out = c.cfg, []
    for b in range(c.batch):
        heads = []
        for h in range(cfg.n_kv_heads):
            d = {k: x.astype(np.float64) for k, x in ob.debug_dump(c, b, h).items()}
            total, res = int(d["lens"][0]), int(d["lens"][1])
            n = total - res
            kd, kz = (np.repeat(d[x], cfg.k_group, 0)[:n] for x in ("k_delta", "k_zero"))
            vd, vz = (np.repeat(d[x], cfg.v_group, 1)[:n] for x in ("v_delta", "v_zero"))
            ints = cfg.zp_mode == ob.ZP_INT
            cat = lambda a, w: np.concatenate([a, w[:res]])
            heads.append({"kc": cat(d["k_codes"][:n] * kd, d["res_k"]), "kb": cat(-kd * kz if ints else kz, 0 * d["res_k"]),
                          "n": cat(d["k_norm"][:n], d["res_norm"]), "vc": cat(d["v_codes"][:n] * vd, d["res_v"]),
                          "vb": cat(-vd * vz if ints else vz, 0 * d["res_v"])})
        seq = {k: np.stack([x[k] for x in heads]) for k in heads[0]}
        seq["window"] = np.arange(total) >= n
        out.append(seq)
    return out
