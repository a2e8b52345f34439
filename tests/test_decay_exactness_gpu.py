"""What linear attention with a decay for each head keeps of a state over many tokens, and the 24 bits of a state that is handed out.

With u = 2^-24.  A state that nothing is added to is g^n S0.  Each product with the factor rounds an entry by up to u of itself; the
roundings of different entries are independent of each other (their bits are random) and take no side, so their mean over N
entries after m products is near 0: its standard deviation is below u sqrt(m / 3) / sqrt(N), and 8 of these are allowed.  An error of the factor
itself has the same sign in every entry and at every product and adds up to m times that error, which the mean shows.  The factor as two
floats is off by 2^-47 of itself (half a unit of the second): m 2^-47 is allowed too.
"""
import math

import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status():
    yield
    ccq.device_status()


def slow_decays(H, tokens):
    """Memories of an eighth of the tokens (so that what is left of a state is an ordinary number) to 8192."""
    least = math.log2(tokens / 8)
    bits = least + (13 - least) * torch.arange(H, dtype=torch.float64) / max(1, H - 1)
    return torch.log1p(-torch.exp2(-bits)).float().cuda()


def check_kept(state, start, log_decay, tokens, products, what):
    """state = g^tokens start in every entry within m u, and the mean of the relative errors within its own bound."""
    d = start.shape[-1]
    ref = start.double() * torch.exp(log_decay.double() * tokens)[:, None, None]
    err = state.double() / ref - 1
    assert float(err.abs().max()) <= 1.01 * products * U + products * 2.0 ** -47, what
    mean = err.mean((-1, -2)).abs().max()
    assert float(mean) <= 8 * U * math.sqrt(products / 3) / d + products * 2.0 ** -47, f"{what}: mean {float(mean):.3g}"


@pytest.mark.parametrize("d", [64, 128])
def test_a_state_decoded_token_by_token(d):
    """4000 steps with a state that nothing is added to, against the recurrence in 64 bits with its state rounded to fp32 once a step.
    (Against the exact power the mean is no measure here: a product with a factor this near 1 sends neighbouring numbers to the same one,
    half of all pairs each time the state halves, so that the entries' roundings are not independent.  In numpy, with factors in
    64 bits, the exact recurrence itself has a mean of 3e-7.)  A step's factor is off by at most 1.3 2^-24 x^2 < 2^-41 (x = log g > -1/500), 2^-17 of
    a unit in the last place: n 2^-41 in n steps, and at most a fraction n 2^-16 = 1/16 of the entries have a rounding that falls the other way, by a
    unit (2 u) to either side, 8 standard deviations of their mean 16 u sqrt(1/16) / 64: below 2^-29 + 2^-28 = 6e-9 together."""
    H, steps = 8, 4000
    ld = slow_decays(H, steps)
    start = torch.randn(2, H, d, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(d))
    state = start.clone()
    x = torch.randn(2, H, d, device="cuda")
    zero = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    ops.decay_attention_step(x, zero, x, ld, start.clone())
    with torch.cuda.graph(graph):
        for _ in range(100):
            ops.decay_attention_step(x, zero, x, ld, state)
    for _ in range(steps // 100):
        graph.replay()
    rounded, gamma = start.clone(), ld.double().exp()[:, None, None]
    for _ in range(steps):
        rounded = (rounded * gamma).float()
    err = state.double() / rounded.double() - 1
    assert float(err.abs().max()) <= 2 * steps * U
    mean = float(err.mean((-1, -2)).abs().max())
    assert mean <= 2.0 ** -29 + 2.0 ** -28, mean


def test_steps_and_a_prompt_keep_the_same():
    """2000 tokens one by one, on a state, against the recurrence in 64 bits: within the roundings of each step (u of the new entry, u of
    k v, which is at most the new one and the old one together: 3 u of the largest), added up over what the state remembers, at most
    1 / (1 - g) tokens."""
    B, H, d, T = 1, 4, 64, 2000
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(T, B, H, d, device="cuda", generator=g) for _ in range(3))
    ld = slow_decays(H, T)
    state = torch.randn(B, H, d, d, device="cuda", generator=g)
    exact, gamma = state.double(), ld.double().exp()[:, None, None]
    largest = exact.abs()
    for t in range(T):
        ops.decay_attention_step(q[t], k[t], v[t], ld, state)
        exact = gamma * exact + k[t].double()[..., None] * v[t].double()[:, :, None]
        largest = torch.maximum(largest, exact.abs())
    memory = (1 / (1 - gamma)).clamp(max=T)
    err = (state.double() - exact).abs()
    assert (err <= 3 * U * memory * largest.amax((-1, -2), keepdim=True)).all()
    # roundings that take no side: the mean error along the state itself (a wrong factor shrinks or grows it as a whole)
    along = ((state.double() - exact) * exact).sum((-1, -2)) / (exact * exact).sum((-1, -2))
    room = 8 * 3 * U * (memory[..., 0, 0] / 3).sqrt() / d * largest.amax((-1, -2)) / exact.pow(2).mean((-1, -2)).sqrt()
    assert (along.abs() <= room).all(), (along / room).tolist()


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,T,H", [(1, 20480, 1), (1, 20480, 8), (1, 3001, 2), (8, 4096, 16)])
def test_a_state_kept_through_a_prompt(dtype, d, B, T, H):
    """Keys of zero: the state handed out is g^T of the one before, by a product for each chunk (128 tokens in bf16, 32 in fp32) and for
    each segment of a sequence that is cut; so is the gradient of the state before, of the one behind."""
    if dtype == FP32 and B == 8:
        B = 2
    ld = slow_decays(H, T)
    start = torch.randn(B, H, d, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(T + d))
    x = torch.randn(B, T, H, d, device="cuda").to(dtype)
    zero = torch.zeros_like(x)
    products = -(-T // (32 if dtype == FP32 else 128)) + 65
    _, state = ops.decay_attention(x, zero, x, ld, state=start)
    check_kept(state, start, ld, T, products, "state")
    g = ops.decay_attention_bwd(zero, x, x, ld, x, dfinal_state=start)
    check_kept(g["dstate"], start, ld, T, products, "dstate")


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [2, 33, 128, 300])
def test_a_state_handed_out_has_24_bits(dtype, d, T):
    """One token with a value, the rest zeros: each entry of the state is one product, g^n k v.  The power is within 2^-22 of itself,
    its product with k is rounded to 24 bits (u), the sum of the three terms' products is cut at most by a unit (2 u), each product with
    a block's factor is rounded once (u; blocks of 32 tokens in fp32, of 128 in bf16): 2^-22 + (4 + blocks) u.  (Two bf16 terms would be
    off by up to 2^-18, 64 u.)"""
    H = 4
    g = torch.Generator(device="cuda").manual_seed(T)
    ld = torch.tensor([-0.0003, -0.01, -0.02, -0.037], device="cuda")
    bound = 2.0 ** -22 + (4 + -(-T // (32 if dtype == FP32 else 128))) * U
    for at in {0, T // 2, T - 2}:
        k, v = (torch.zeros(1, T, H, d, device="cuda").to(dtype) for _ in range(2))
        k[:, at], v[:, at] = (torch.randn(1, H, d, device="cuda", generator=g).to(dtype) for _ in range(2))
        _, state = ops.decay_attention(k, k, v, ld)
        exact = lambda n: (torch.exp(ld.double() * n)[:, None, None] * k[0, at].double()[..., None] * v[0, at].double()[:, None])[None]  # noqa: E731
        ref = exact(T - 1 - at)
        assert ((state.double() - ref).abs() <= bound * ref.abs()).all(), at
        # the gradient of the state before: scale g^(n + 1) q dout
        grads = ops.decay_attention_bwd(k, k, k, ld, v, dfinal_state=torch.zeros_like(state), scale=0.5)
        ref = 0.5 * exact(at + 1)
        assert ((grads["dstate"].double() - ref).abs() <= bound * ref.abs()).all(), at


@pytest.mark.parametrize("Hk", [128, 64])
def test_gradients_of_offsets_past_32_bits(Hk):
    """The last of many rows, 2^31 elements and more in, of heads of their own and of shared ones; the rows before have no gradient."""
    B, T, H, d = 9000, 16, 128, 128  # 2.36e9 elements
    g = torch.Generator(device="cuda").manual_seed(Hk)
    n = lambda h: torch.randn(1, T, h, d, device="cuda", generator=g).to(BF16)  # noqa: E731
    q, k, v, dout = (torch.zeros(B, T, h, d, dtype=BF16, device="cuda") for h in (H, Hk, Hk, H))
    for x in (q, k, v, dout):
        x[-1:] = n(x.shape[2])
    ld = torch.linspace(-0.3, -0.01, H, device="cuda")
    grads = ops.decay_attention_bwd(q, k, v, ld, dout)
    alone = ops.decay_attention_bwd(q[-1:], k[-1:], v[-1:], ld, dout[-1:])
    for name, x in grads.items():
        assert torch.equal(x[-1], alone[name][0]) and not x[0].any() and not x[-2].any() and alone[name].any(), name


def test_states_past_32_bits():
    """States of 2^31 elements and more, as a pool for steps and before and after many short prompts: the last rows as by themselves."""
    rows, H, d = 9000, 16, 128  # 2.36e9 elements
    g = torch.Generator(device="cuda").manual_seed(6)
    pool = torch.zeros(rows, H, d, d, device="cuda")
    pool[-2:] = torch.randn(2, H, d, d, device="cuda", generator=g)
    before = pool[-2:].clone()
    ld = torch.linspace(-0.3, -0.01, H, device="cuda")
    q, k, v = (torch.randn(2, H, d, device="cuda", generator=g).to(BF16) for _ in range(3))
    alone = before.clone()
    expect = ops.decay_attention_step(q, k, v, ld, alone)
    o = ops.decay_attention_step(q, k, v, ld, pool, slots=torch.tensor([rows - 2, rows - 1], device="cuda"))
    assert torch.equal(o, expect) and torch.equal(pool[-2:], alone) and not pool[:-2].any()
    for dtype in (BF16, FP32):
        x = torch.zeros(rows, 3, H, d, device="cuda", dtype=dtype)
        x[-2:] = torch.randn(2, 3, H, d, device="cuda", generator=g).to(dtype)
        expect, state = ops.decay_attention(x[-2:], x[-2:], x[-2:], ld, state=pool[-2:])
        o, states = ops.decay_attention(x, x, x, ld, state=pool)
        assert torch.equal(o[-2:], expect) and torch.equal(states[-2:], state) and not states[:-2].any() and not o[:-2].any()
        expect = ops.decay_attention_bwd(x[-2:], x[-2:], x[-2:], ld, x[-2:], state=pool[-2:], dfinal_state=state)
        grads = ops.decay_attention_bwd(x, x, x, ld, x, state=pool, dfinal_state=states)
        for n in expect:
            assert torch.equal(grads[n][-2:], expect[n]) and not grads[n][:-2].any(), n
        del x, o, states, grads
