"""The 8-bit cache in 64 bits on the CPU: what its definition says it holds, for the tests of its calls."""
import numpy as np

D = 128


def torch_type(io):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[io]


def counted(x, io):
    """Numbers as the cache takes them: NaN as 0, large ones as the largest."""
    most = 65504.0 if io == "f16" else 2.0 ** 60
    return np.clip(np.nan_to_num(x, nan=0.0, posinf=np.inf, neginf=-np.inf), -most, most)


def e4m3(r):
    """The nearest number of four significant bits, exponents -6 .. 8, ties to even (|r| <= 448)."""
    _, e = np.frexp(np.abs(r))                      # |r| = m 2^e, 1/2 <= m < 1
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(r / step) * step


def stands_for(x, block, io):
    """[tokens, channels] of one kv head -> what its whole blocks and its other tokens count as, and the scales."""
    y = counted(x.astype(np.float64), io)
    scales = []
    for t in range(0, len(y) // block * block, block):
        a = np.abs(y[t:t + block]).max()
        m, e = np.frexp(a)
        e = max(e - 9 + (m > 0.875), -100) if a > 0 else 0
        scales.append(2.0 ** e)
        y[t:t + block] = e4m3(y[t:t + block] / 2.0 ** e) * 2.0 ** e
    return y, np.array(scales)


def tokens(rng, B, S, H, io, wild=False):
    """[B, S, H, 128] in 64 bits, values that the io type holds."""
    import torch
    x = rng.standard_normal((B, S, H, D)) * np.exp(0.5 * rng.standard_normal((B, S, 1, 1)))
    x[..., ::37] *= 8.0
    if wild:
        # blocks of zeros, of tiny and of huge numbers, ties and the edges of the format
        x[:, 32:64] = 0.0
        x[:, 64:96] *= 2.0 ** -20
        x[:, 96:128] *= 2.0 ** (9 if io == "f16" else 40)
        x[:, 128:160] = rng.integers(-64, 65, size=x[:, 128:160].shape) * 7.0
        x[:, 160:192] = rng.choice([0.0, -0.0, 448.0, -448.0, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 449.0, 1.0625, 1.1875],
                                   size=x[:, 160:192].shape)
    return torch.from_numpy(x).to(torch_type(io)).double().numpy()


def dev(x, io):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch_type(io)).cuda()


def ints(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def scattered_cache(ob, H, B, pages, block, io, rng, poison=True):
    """A cache whose pages lie in any order; what no token owns is no number."""
    import torch
    perm = rng.permutation(B * pages + 3)[:B * pages].reshape(B, pages)
    c = ob.Q8Cache(H, B, pages, block=block, io_dtype={"bf16": ob.BF16, "f16": ob.F16}[io], num_pages=B * pages + 3,
                   block_table=ints(perm))
    if poison:
        c.k_codes.fill_(0x7f), c.v_codes.fill_(0x7f)
        for x in (c.k_scales, c.v_scales):
            x.fill_(float("nan"))
        for x in (c.win_k, c.win_v):
            x.view(torch.int16).fill_(0x7fff)
    return c


def packed_rows(x, old, new, spare=0):
    """[B, S, H, 128] -> the new tokens of every sequence one behind the other, and their first rows."""
    rows = [x[b, old[b]:old[b] + n] for b, n in enumerate(new)]
    starts = np.concatenate([[0], np.cumsum(new)])
    rows.append(np.zeros((spare,) + x.shape[2:]))
    return np.concatenate(rows), starts


def padded_rows(x, old, new, T):
    out = np.zeros((len(new), T) + x.shape[2:])
    for b, n in enumerate(new):
        out[b, :n] = x[b, old[b]:old[b] + n]
    return out
