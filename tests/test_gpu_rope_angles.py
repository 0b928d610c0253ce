"""oscar_rope's angles: the product of position and frequency counts exactly, however far the position."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def cos_and_sin(pos, inv):
    """In 80-bit arithmetic, whose 64 bits hold the product of a 32-bit and a 24-bit number: after the reduction the
    angle is off by 2^31 2^-64 at most."""
    a = pos[:, None].astype(np.longdouble) * inv.astype(np.longdouble)
    a = np.remainder(a, 2 * np.longdouble("3.14159265358979323846264338327950288"))
    return np.cos(a), np.sin(a)


@pytest.mark.parametrize("first", [0, 1 << 20, 2 ** 31 - 60000, -2 ** 31])
@pytest.mark.parametrize("inverse", [False, True])
def test_angles_are_exact(first, inverse):
    """A pair (1, 0) turns into (cos a, sin a).  Each is rounded once to fp32, half a step: 2^-24 of itself; the product
    with 1 and the sum with 0 are exact.  What is left of the angle's error, 2^-33 of the oracle, counts for values
    near 0."""
    import torch
    from paper_2605_19660_amd import binding as ob
    rng = np.random.default_rng(abs(first) % 1000)
    n = 4000
    pos = (first + rng.integers(0, 60000, size=n)).astype(np.int32)
    inv = np.concatenate([1e4 ** (-np.arange(0, 64) / 64), rng.random(64)]).astype(np.float32)
    for part in (inv[:64], inv[64:]):
        x = torch.zeros(n, 1, 128, device="cuda")
        x[:, :, :64] = 1.0
        y = ob.rope(x, None, torch.from_numpy(pos).cuda(), torch.from_numpy(part).cuda(), inverse=inverse)[0]
        y = y[:, 0].double().cpu().numpy()
        c, s = cos_and_sin(pos, part)
        for got, want in ((y[:, :64], c), (y[:, 64:], -s if inverse else s)):
            err = np.abs(got - want)
            assert (err <= np.abs(want) * 2.0 ** -24 * (1 + 1e-6) + 2.0 ** -32).all(), float((err - np.abs(want) * 2.0 ** -24).max())


def test_turns_are_as_near_as_64_bit_angles_give():
    """A turn in fp32: sine and cosine half a step each, two products and their difference half a step each."""
    import torch
    from paper_2605_19660_amd import binding as ob
    g = torch.Generator().manual_seed(4)
    n = 500
    x = torch.randn(n, 2, 128, generator=g)
    pos = torch.randint(0, 2 ** 31 - 1, (n,), generator=g).int()
    inv = (1e4 ** (-np.arange(0, 128, 2) / 128)).astype(np.float32)
    y = ob.rope(x.cuda(), None, pos.cuda(), torch.from_numpy(inv).cuda())[0].double().cpu().numpy()
    c, s = (t.astype(np.float64)[:, None] for t in cos_and_sin(pos.numpy(), inv))
    a, b = x[..., :64].double().numpy(), x[..., 64:].double().numpy()
    for got, (u, v) in ((y[..., :64], (a * c, -b * s)), (y[..., 64:], (b * c, a * s))):
        bound = 2.0 ** -24 * (2 * np.abs(u) + 2 * np.abs(v) + np.abs(u + v)) * (1 + 1e-6) + 2.0 ** -31
        assert (np.abs(got - (u + v)) <= bound).all()


def test_frequencies_of_any_size():
    """Against 60-digit arithmetic where the product has 51 bits before the point and more than the fraction's left;
    beyond that a turn stays a turn."""
    import torch
    from decimal import Decimal, getcontext
    from paper_2605_19660_amd import binding as ob
    getcontext().prec = 60
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    inv = np.array([3e5, 1e6, 1.7e7, 1e-30, 0.0, 3e38] + [1e12] * 58, np.float32)
    pos = np.array([2 ** 31 - 1, -2 ** 31, 1999999999, -3, 0, 77], np.int32)
    x = torch.zeros(len(pos), 1, 128, device="cuda")
    x[:, :, :64] = 1.0
    y = ob.rope(x, None, torch.from_numpy(pos).cuda(), torch.from_numpy(inv).cuda())[0][:, 0].double().cpu().numpy()
    for i, p in enumerate(pos):
        for j in range(5):
            a = float(Decimal(int(p)) * Decimal(float(inv[j])) % two_pi)
            for got, want in ((y[i, j], np.cos(a)), (y[i, 64 + j], np.sin(a))):
                assert abs(got - want) <= abs(want) * 2.0 ** -24 * (1 + 1e-6) + 2.0 ** -40, (p, inv[j])
    assert (np.abs(y[:, :64] ** 2 + y[:, 64:] ** 2 - 1) <= 4 * 2.0 ** -24).all()
