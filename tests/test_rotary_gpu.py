"""GPU checks of the rotation of queries and keys by their positions (ccq_rotary) against 64 bits.

Bound, set before the first run, with u = 2^-24: y = m (a cos - b sin).  The argument of sincospif, |x| <= 1, is rounded to
half a step (pi u / 2 of the angle) and cut at 2^-31 (nothing beside it); sincospif is within 2 units in the last place (4 u);
the amplitude, the product and the sum are rounded once each (3 u), the second product is fused or rounded (1 u): together below
10 u m (|a| + |b|).  Then one rounding to the type, half a step: r = 2^-8 of the value in bf16, u in fp32.
"""
import math

import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
R = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status():
    yield
    ccq.device_status()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def reference(x, positions, freqs, interleaved, amplitude, sign=1.0):
    """The rotation in 64 bits, and the bound."""
    x = x.double()
    part = 2 * freqs.numel()
    theta = sign * positions.double()[..., None] * freqs
    c, s = amplitude * theta.cos()[..., None, :], amplitude * theta.sin()[..., None, :]
    index = torch.arange(part // 2, device=x.device)
    ia, ib = (2 * index, 2 * index + 1) if interleaved else (index, index + part // 2)
    y, bound = x.clone(), torch.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    bound[..., ia] = bound[..., ib] = 10 * U * abs(amplitude) * (a.abs() + b.abs())
    return y, bound


def check(got, x, positions, freqs, interleaved, amplitude, sign=1.0):
    ref, bound = reference(x, positions, freqs, interleaved, amplitude, sign)
    bound = bound + R[x.dtype] * ref.abs()
    part = 2 * freqs.numel()
    assert torch.equal(got[..., part:], x[..., part:])
    bad = ~((got.double() - ref).abs() <= bound)[..., :part]
    assert not bad.any(), float(((got.double() - ref).abs() / bound)[..., :part].max())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,heads,kv,width,part", [(1, 1, 1, 1, 2, 2), (2, 33, 16, 4, 128, 128), (1, 77, 3, 1, 128, 64),
                                                     (3, 5, 2, 2, 96, 96), (1, 300, 2, 1, 80, 20), (2, 9, 1, 1, 66, 66),
                                                     (1, 3, 1, 3, 7, 6), (1, 2, 40, 8, 256, 256), (256, 1, 16, 16, 128, 128),
                                                     (1, 4, 2, 2, 4096, 4096)])
def test_rotary(dtype, interleaved, B, T, heads, kv, width, part):
    g = gen(B * T + width)
    q = torch.randn(B, T, heads, width, device="cuda", generator=g).to(dtype)
    k = torch.randn(B, T, kv, width, device="cuda", generator=g).to(dtype)
    positions = torch.randint(0, 40000, (B, T), device="cuda", generator=g)
    freqs, amplitude = ops.rotary_frequencies(part, scaling="yarn", factor=4.0)
    for pos in (positions, positions.int()):
        a, b = ops.rotary(q, k, pos, freqs, interleaved=interleaved, amplitude=amplitude)
        check(a, q, pos, freqs, interleaved, amplitude)
        check(b, k, pos, freqs, interleaved, amplitude)
    assert torch.equal(ops.rotary(q, None, positions, freqs, interleaved=interleaved, amplitude=amplitude), a)
    a, b = ops.rotary_bwd(q, k, positions, freqs, interleaved=interleaved, amplitude=amplitude)
    check(a, q, positions, freqs, interleaved, amplitude, -1.0)
    check(b, k, positions, freqs, interleaved, amplitude, -1.0)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("offset", [0, 1, 2, 4, 8])
def test_slices_transposes_and_offsets(dtype, offset):
    """Any strides and any alignment of the type, in and out."""
    g = gen(offset)
    B, T, heads, width = 2, 19, 4, 64
    freqs, _ = ops.rotary_frequencies(48)
    positions = torch.arange(T, device="cuda").expand(B, T).contiguous()
    fused = torch.randn(B, T, 3 * heads * width + offset, device="cuda", generator=g).to(dtype)
    q = fused[..., offset:offset + heads * width].unflatten(-1, (heads, width))
    k = fused[..., offset + heads * width:offset + 2 * heads * width].unflatten(-1, (heads, width))
    out_k = torch.full((B, heads, T, width + offset), 7.0, device="cuda", dtype=dtype)[..., :width].transpose(1, 2)
    a, b = ops.rotary(q, k, positions, freqs, out=(None, out_k))
    assert b is out_k and a.is_contiguous()
    check(a, q, positions, freqs, False, 1.0)
    check(b, k, positions, freqs, False, 1.0)
    # heads and tokens the other way round, and one head's values read by all
    t = torch.randn(B, heads, T, width, device="cuda", generator=g).to(dtype).transpose(1, 2)
    shared = t[:, :, :1].expand(B, T, heads, width)
    a, b = ops.rotary(t, shared, positions, freqs, interleaved=True)
    check(a, t, positions, freqs, True, 1.0)
    check(b, shared, positions, freqs, True, 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(interleaved):
    g = gen(5)
    qkv = torch.randn(2, 50, 3 * 4 * 128, device="cuda", generator=g).to(BF16)
    before = qkv.clone()
    q, k, v = (t.unflatten(-1, (4, 128)) for t in qkv.split(512, -1))
    freqs, _ = ops.rotary_frequencies(64)
    positions = torch.arange(100, device="cuda").view(2, 50)
    a, b = ops.rotary(q, k, positions, freqs, interleaved=interleaved, out=(q, k))
    assert a is q and b is k
    was = [t.unflatten(-1, (4, 128)) for t in before.split(512, -1)]
    check(q, was[0], positions, freqs, interleaved, 1.0)
    check(k, was[1], positions, freqs, interleaved, 1.0)
    assert torch.equal(v, was[2])


def test_far_and_negative_positions():
    """Angles do not lose the position: far beyond 2^24, where an fp32 product would be off by many turns."""
    freqs, _ = ops.rotary_frequencies(64)
    positions = torch.tensor([0, -1, 2 ** 24 + 1, 2 ** 30 + 12345, -2 ** 31, 2 ** 40 + 3], device="cuda")
    x = torch.randn(6, 2, 64, device="cuda", generator=gen(3))
    got = ops.rotary(x, None, positions, freqs)
    # in 64 bits the product is exact to 2^-53 of the angle: 1e-4 radians at 2^40, so that one is held to less
    ref, bound = reference(x, positions, freqs, False, 1.0)
    angle = (positions.double().abs()[:, None] * freqs)[:, None].repeat(1, 1, 2)
    bound = bound + U * ref.abs() + (angle * 2.0 ** -52 + 2 * math.pi * 2.0 ** -31) * 2 * x.double().abs().amax(-1, keepdim=True)
    assert ((got.double() - ref).abs() <= bound).all()


def test_frequencies_that_are_not_ordinary():
    x = torch.randn(4, 1, 12, device="cuda", generator=gen(4))
    freqs = torch.tensor([0.0, 7.0, -0.5, 1e-300, 1e-20, float("inf")], dtype=torch.float64, device="cuda")
    positions = torch.tensor([0, 1, 2, 1000], device="cuda")
    got = ops.rotary(x, None, positions, freqs)
    ref, bound = reference(x[..., [0, 1, 2, 3, 4, 6, 7, 8, 9, 10]], positions, freqs[:5], False, 1.0)
    finite = got[..., [0, 1, 2, 3, 4, 6, 7, 8, 9, 10]]
    assert ((finite.double() - ref).abs() <= bound + U * ref.abs()).all()
    assert got[..., [5, 11]].isnan().all()


def test_gradient_against_differences():
    """The rotation is linear: <rotary(x + e) - rotary(x), g> = <e, rotary_bwd(g)>."""
    g = gen(6)
    freqs, amplitude = ops.rotary_frequencies(32, scaling="yarn", factor=8.0)
    positions = torch.arange(40, device="cuda")
    x, e, dy = (torch.randn(40, 3, 64, device="cuda", generator=g) for _ in range(3))
    for interleaved in (False, True):
        how = dict(interleaved=interleaved, amplitude=amplitude)
        step = ops.rotary(x + e, None, positions, freqs, **how).double() - ops.rotary(x, None, positions, freqs, **how).double()
        along = (step * dy).sum()
        by_gradient = (ops.rotary_bwd(dy, None, positions, freqs, **how).double() * e).sum()
        # each product's error: 12 u of |x| + |e| (two rotations and the sum x + e), times |dy|
        room = 24 * U * amplitude * ((x.abs() + e.abs()).double() * 2 * dy.abs()).sum()
        assert abs(along - by_gradient) <= room


def test_offsets_past_32_bits():
    tokens, heads, width = 1_100_000, 16, 128  # 2.25e9 elements
    x = torch.zeros(tokens, heads, width, dtype=BF16, device="cuda")
    at = torch.tensor([tokens - 1, 1_048_577, 5], device="cuda")
    x[at] = torch.randn(3, heads, width, device="cuda", generator=gen(7)).to(BF16)
    was = x[at].clone()
    positions = torch.arange(tokens, device="cuda")
    freqs, _ = ops.rotary_frequencies(width)
    assert ops.rotary(x, None, positions, freqs, out=(x, None)) is x
    check(x[at], was, at, freqs, False, 1.0)
    assert int((x.view(tokens, -1) != 0).any(1).sum()) == 3


def test_empty():
    freqs, _ = ops.rotary_frequencies(64)
    for shape in ((0, 2, 64), (0, 5, 2, 64), (3, 0, 2, 64)):
        x = torch.empty(shape, device="cuda")
        a, b = ops.rotary(x, x, torch.empty(shape[:-2], dtype=torch.int64, device="cuda"), freqs)
        assert a.shape == x.shape and b.shape == x.shape
