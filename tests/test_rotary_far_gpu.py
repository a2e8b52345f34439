"""The rotation's angles for any position and any frequency, against angles formed in whole numbers (1 / (2 pi) to 2400 bits).

Bound, with u = 2^-24: an angle is formed to 2^-30 of a turn (6e-9, a tenth of u) and rounded as an fp32 argument of half turns below 1
(pi u / 2); sincospif is within 2 units in the last place (4 u); amplitude, products and sum 4 roundings: below 10 u (|a| + |b|), and the
rounding to the type, u of the value."""
import math

import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BITS = 2400


def inverse_of_a_turn():
    """2^BITS / (2 pi), by Machin's formula."""
    one = 1 << (BITS + 64)

    def arctan_of_inverse(n):
        t = total = one // n
        k, sign = 1, -1
        while t:
            t //= n * n
            k += 2
            total += sign * (t // k)
            sign = -sign
        return total

    return (one * one // (8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239)))) >> 64


def angle(position, frequency, inverse):
    """position * frequency mod a turn, in radians from -pi to pi."""
    a, b = float(frequency).as_integer_ratio()
    den = b << BITS
    num = position * a * inverse % den
    return ((num << 80) // den) / 2.0 ** 80 * 2 * math.pi if 2 * num < den else -((((den - num) << 80) // den) / 2.0 ** 80 * 2 * math.pi)


POSITIONS = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31, -2 ** 31 - 1, 2 ** 32 + 7, 2 ** 40 + 3, 2 ** 52 + 1, -2 ** 57 - 99, 2 ** 63 - 1, -2 ** 63, 30011]
FREQS = [1.0, 0.5403, 1e-4, 1.99999, 2.0, 7.0, 1e3, 1e6, -1e6, 123456789.25, 2.0 ** 63, 2.0 ** 64, 1e40, -3e200, 1.7976931348623157e308, 1e-30,
         2.0 ** -70, -2.0 ** -1000, 5e-324, 0.0]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_any_position_and_frequency(interleaved, index):
    inverse = inverse_of_a_turn()
    assert abs(inverse / 2 ** BITS * 2 * math.pi - 1) < 1e-15
    positions = [p for p in POSITIONS if index is torch.int64 or -2 ** 31 <= p < 2 ** 31]
    n, part = len(positions), 2 * len(FREQS)
    x = torch.randn(n, 2, part, generator=torch.Generator().manual_seed(1))
    at, freqs = torch.tensor(positions, dtype=index), torch.tensor(FREQS, dtype=torch.float64)
    theta = torch.tensor([[angle(p, f, inverse) for f in FREQS] for p in positions], dtype=torch.float64)[:, None]
    half = len(FREQS)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    a, b = a.double(), b.double()
    for inverse_call, sign in ((ops.rotary, 1), (ops.rotary_bwd, -1)):
        got = inverse_call(x.cuda(), None, at.cuda(), freqs.cuda(), interleaved=interleaved).double().cpu()
        ga, gb = (got[..., 0::2], got[..., 1::2]) if interleaved else (got[..., :half], got[..., half:])
        c, s = theta.cos(), sign * theta.sin()
        for name, y, ref in (("first", ga, a * c - b * s), ("second", gb, a * s + b * c)):
            err = (y - ref).abs() / (10 * U * (a.abs() + b.abs()) + U * ref.abs())
            i = int(err.amax((1,)).argmax())
            assert float(err.max()) <= 1, f"{name} of position {positions[i // half]}, frequency {FREQS[i % half]}: {float(err.max()):.3g} of the bound"
    ccq.device_status()


def test_random_far_positions():
    """Positions and frequencies of every magnitude, in one call of many tokens."""
    inverse = inverse_of_a_turn()
    g = torch.Generator().manual_seed(2)
    n, half = 64, 32
    positions = [int(m * 2 ** (e - 20)) for m, e in zip(torch.randint(-2 ** 20, 2 ** 20, (n,), generator=g).tolist(), torch.randint(20, 63, (n,), generator=g).tolist())]
    freqs = (torch.rand(half, dtype=torch.float64, generator=g) + 1) * torch.exp2(torch.randint(-30, 40, (half,), generator=g).double())
    x = torch.randn(n, 1, 2 * half, generator=g)
    theta = torch.tensor([[angle(p, f, inverse) for f in freqs.tolist()] for p in positions], dtype=torch.float64)[:, None]
    a, b = x.double().split(half, -1)
    got = ops.rotary(x.cuda(), None, torch.tensor(positions).cuda(), freqs.cuda()).double().cpu()
    ref = torch.cat([a * theta.cos() - b * theta.sin(), a * theta.sin() + b * theta.cos()], -1)
    room = 10 * U * (a.abs() + b.abs()).repeat(1, 1, 2) + U * ref.abs()
    assert ((got - ref).abs() <= room).all(), float(((got - ref).abs() / room).max())
