"""GPU checks of linear attention with a decay for each head (ccq_decay_attention and its gradients and step).

The reference is the sum over all pairs of tokens in 64 bits, and its gradients by reverse mode.  Bounds, set before
the first run, with u = 2^-24, A = the same sums of the magnitudes of all terms (an output is a sum of products of three
inputs and a power of the decay), and r = half a step of the output's type (2^-8 of its value in bf16, u in fp32):
  fp32 arithmetic: a term passes a dot product over d (d u), a sum over a block (32 u) and, within the state, a product and a
    sum for each block of 32 tokens (2 u each); the powers, off by 2^-22 and u |log2| each, and the products with them: 12 u
    and 3 u a block.  (d + 44 + 5 blocks) u A, + r |ref|.
  tensor cores: the scores and the state are rounded to bf16 where they enter their second product, half a step of each
    term: 2^-8 A; the state is carried to two bf16 halves of a scaled key (2^-17) and fp32 sums of chunks of 128:
    (2^-17 + (d + 140 + 5 chunks) u) A for it.
  shared heads' gradients: one more fp32 sum.
"""
import math

import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
R = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF16, FP32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(autouse=True)
def _status():
    yield
    ccq.device_status()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def decays(H):
    """From no decay at all to none kept."""
    return torch.tensor([-0.01, 0.0, -0.3, -3.0, -1e-4, -50.0, -INF, -0.1] * (H // 8 + 1), device="cuda")[:H].contiguous()


def make(B, T, H, Hq, Hk, Hv, d, dtype, seed, state=True):
    g = gen(seed)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v = (n(B, T, h, d).to(dtype) for h in (Hq, Hk, Hv))
    return q, k, v, decays(H), n(B, H, d, d) if state else None


def all_pairs(q, k, v, log_decay, S0, scale):
    """o and the final state by sums over all pairs; 64-bit [B, T, heads, d]."""
    B, T, _, d = q.shape
    H = log_decay.shape[0]
    q, k, v = (x.repeat_interleave(H // x.shape[2], 2).transpose(1, 2) for x in (q, k, v))
    t = torch.arange(T, device=q.device)
    gap = (t[:, None] - t).clamp(min=0)
    power = lambda n: torch.where(n == 0, 1.0, torch.exp(n.double() * log_decay.double().view(-1, *[1] * n.dim())))  # noqa: E731
    D = power(gap) * (t[:, None] >= t)
    o = ((q @ k.transpose(-1, -2)) * D) @ v
    ST = (k * power(T - 1 - t)[..., None]).transpose(-1, -2) @ v
    if S0 is not None:
        o = o + (q * power(t + 1)[..., None]) @ S0
        ST = ST + power(torch.tensor(T, device=q.device)).view(-1, 1, 1) * S0
    return (o * scale).transpose(1, 2), ST


def with_gradients(q, k, v, log_decay, S0, scale, dout, dST):
    leaves = [x.double().requires_grad_() for x in (q, k, v)] + ([S0.double().requires_grad_()] if S0 is not None else [])
    o, ST = all_pairs(*leaves[:3], log_decay, leaves[3] if S0 is not None else None, scale)
    L = (o * dout.double()).sum() + (0 if dST is None else (ST * dST.double()).sum())
    return torch.autograd.grad(L, leaves)


def eps_of(dtype, d, T, tensor_cores):
    """(of an output, of a state), relative to A."""
    if not tensor_cores:
        e = (d + 44 + 5 * (T // 32 + 1)) * U
        return e, e
    e = 2.0 ** -17 + (d + 140 + 5 * (T // 128 + 1)) * U
    return 2.0 ** -8 + e, e


def close(x, ref, bound, what):
    err = (x.double() - ref).abs()
    bad = ~(err <= bound + 1e-35)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst {float((err / (bound + 1e-35)).nan_to_num(1e9).max()):.3g} of the bound"


def check_forward(o, ST, q, k, v, ld, S0, scale, cores):
    d, T = q.shape[3], q.shape[1]
    d64 = lambda x: None if x is None else x.double()  # noqa: E731
    mag = lambda x: None if x is None else x.double().abs()  # noqa: E731
    ref, refS = all_pairs(d64(q), d64(k), d64(v), ld, d64(S0), scale)
    A, AS = all_pairs(mag(q), mag(k), mag(v), ld, mag(S0), abs(scale))
    e, eS = eps_of(q.dtype, d, T, cores)
    close(o, ref, e * A + R[q.dtype] * ref.abs(), "o")
    if ST is not None:
        close(ST, refS, eS * AS + U * refS.abs(), "state")


def check_backward(g, q, k, v, ld, S0, scale, dout, dST, cores):
    ref = with_gradients(q, k, v, ld, S0, scale, dout, dST)
    mag = lambda x: None if x is None else x.double().abs()  # noqa: E731
    A = with_gradients(mag(q), mag(k), mag(v), ld, mag(S0), abs(scale), mag(dout), mag(dST))
    e, eS = eps_of(q.dtype, q.shape[3], q.shape[1], cores)
    for i, name in enumerate(("dq", "dk", "dv")):
        close(g[name], ref[i], (e + U * 16) * A[i] + R[q.dtype] * ref[i].abs(), name)
    if S0 is not None:
        close(g["dstate"], ref[3], eS * A[3] + U * ref[3].abs(), "dstate")


LENGTHS = [1, 2, 31, 32, 33, 64, 127, 128, 129, 255, 300, 515]


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", LENGTHS)
def test_forward(dtype, d, T):
    B, H = 2, 8
    for state in (False, True):
        q, k, v, ld, S0 = make(B, T, H, H, H, H, d, dtype, T + d, state)
        o, ST = ops.decay_attention(q, k, v, ld, state=S0)
        check_forward(o, ST, q, k, v, ld, S0, d ** -0.5, dtype == BF16)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", LENGTHS)
def test_backward(dtype, d, T):
    B, H = 2, 8
    for state in (False, True):
        q, k, v, ld, S0 = make(B, T, H, H, H, H, d, dtype, T + d + 1, state)
        dout = torch.randn(B, T, H, d, device="cuda", generator=gen(T)).to(dtype)
        dST = torch.randn(B, H, d, d, device="cuda", generator=gen(T + 1)) if state else None
        g = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST)
        check_backward(g, q, k, v, ld, S0, d ** -0.5, dout, dST, dtype == BF16)
        assert set(g) == {"dq", "dk", "dv"} | ({"dstate"} if state else set())


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("H,Hq,Hk,Hv", [(4, 4, 1, 1), (6, 6, 2, 3), (8, 2, 2, 8), (4, 1, 1, 1)])
def test_shared_heads(dtype, H, Hq, Hk, Hv):
    B, T, d = 2, 150, 64
    q, k, v, ld, S0 = make(B, T, H, Hq, Hk, Hv, d, dtype, H + Hv)
    o, ST = ops.decay_attention(q, k, v, ld, state=S0, scale=0.3)
    scale = float(torch.tensor(0.3))
    check_forward(o, ST, q, k, v, ld, S0, scale, dtype == BF16)
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(9)).to(dtype)
    dST = torch.randn(B, H, d, d, device="cuda", generator=gen(10))
    g = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST, scale=0.3)
    check_backward(g, q, k, v, ld, S0, scale, dout, dST, dtype == BF16)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("layout", ["fused", "heads_first", "odd", "expanded"])
def test_layouts(dtype, layout):
    B, T, H, d = 2, 141, 4, 128
    g = gen(21)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g).to(dtype)  # noqa: E731
    if layout == "fused":
        q, k, v = (t.unflatten(-1, (H, d)) for t in n(B, T, 3 * H * d).split(H * d, -1))
    elif layout == "heads_first":
        q, k, v = (n(B, H, T, d).transpose(1, 2) for _ in range(3))
    elif layout == "odd":
        q, k, v = (n(B, T, H, d + 1)[..., 1:] for _ in range(3))
    else:
        q, k, v = (n(B, T, 1, d).expand(B, T, H, d) for _ in range(3))
    ld = decays(H)
    cores = dtype == BF16 and layout != "odd"
    out = {"heads_first": lambda: torch.empty(B, H, T, d, dtype=dtype, device="cuda").transpose(1, 2),
           "odd": lambda: torch.full((B, T, H, d + 3), 5.0, dtype=dtype, device="cuda")[..., :d]}.get(layout, lambda: None)
    o_buf = out()
    o, ST = ops.decay_attention(q, k, v, ld, out=o_buf)
    assert o_buf is None or o is o_buf
    check_forward(o, ST, q, k, v, ld, None, d ** -0.5, cores)
    dout = (n(B, T, H, d + 1)[..., 1:] if layout == "odd" else n(B, H, T, d).transpose(1, 2))
    given = {"dq": out(), "dv": out()} if out() is not None else None
    grads = ops.decay_attention_bwd(q, k, v, ld, dout, out=given)
    assert given is None or (grads["dq"] is given["dq"] and grads["dv"] is given["dv"])
    check_backward(grads, q, k, v, ld, None, d ** -0.5, dout, None, cores)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths", [[5, 0, 1, 128, 33, 200, 0], [300], [0, 0], [127, 129, 1, 1, 256]])
def test_packed(dtype, d, lengths):
    """Each sequence as by itself; rows of no sequence, before the first and after the last, are left as they are."""
    H, before, after = 4, 3, 70
    total = sum(lengths)
    q, k, v, ld, _ = make(1, before + total + after, H, H, 2, 2, d, dtype, total + d, False)
    # what no sequence has is not read into any
    for x in (q, k, v):
        x[:, :before] = INF
        x[:, before + total:] = float("nan")
    n = len(lengths)
    cu = (torch.tensor([0] + lengths, device="cuda").cumsum(0) + before)
    S0 = torch.randn(n, H, d, d, device="cuda", generator=gen(1))
    dST = torch.randn(n, H, d, d, device="cuda", generator=gen(2))
    dout = torch.randn(1, before + total + after, H, d, device="cuda", generator=gen(3)).to(dtype)
    dout[:, before + total:] = float("nan")
    o = torch.full_like(q, 7.0)
    ops.decay_attention(q, k, v, ld, state=S0, cu_seqlens=cu.int(), out=o)
    o, ST = ops.decay_attention(q, k, v, ld, state=S0, cu_seqlens=cu, out=o)
    grads = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST, cu_seqlens=cu)
    assert (o[:, :before] == 7).all() and (o[:, before + total:] == 7).all()
    at = before
    for s, m in enumerate(lengths):
        cut = slice(at, at + m)
        at += m
        if m == 0:
            assert torch.equal(ST[s], S0[s]) and torch.equal(grads["dstate"][s], dST[s])
            continue
        args = q[:, cut], k[:, cut], v[:, cut], ld, S0[s:s + 1], d ** -0.5
        check_forward(o[:, cut], ST[s:s + 1], *args, dtype == BF16)
        mine = {x: grads[x][:, cut] for x in ("dq", "dk", "dv")} | {"dstate": grads["dstate"][s:s + 1]}
        check_backward(mine, *args, dout[:, cut], dST[s:s + 1], dtype == BF16)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("n", [200, 256, 257, 700])
def test_many_packed_sequences(dtype, n):
    """Up to 256 run by their lengths, more as they lie: a token's result is that of its sequence by itself either way."""
    H, d = 2, 64
    lengths = torch.randint(0, 60, (n,), device="cuda", generator=gen(n))
    lengths[n // 2] = 300
    cu = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    total = int(cu[-1])
    q, k, v, ld, _ = make(1, total, H, H, H, H, d, dtype, n, False)
    S0 = torch.randn(n, H, d, d, device="cuda", generator=gen(n + 1))
    o, ST = ops.decay_attention(q, k, v, ld, state=S0, cu_seqlens=cu)
    g = ops.decay_attention_bwd(q, k, v, ld, v, state=S0, dfinal_state=S0, cu_seqlens=cu)
    # in a batch of rows of the longest's length, with zeros past each end: they add nothing to o; one sequence at a time for states
    at = torch.arange(300, device="cuda")
    held = at < lengths[:, None]
    rows = torch.where(held, cu[:-1, None] + at, 0)
    pad = lambda x: x[0][rows] * held[..., None, None]  # noqa: E731
    padded, _ = ops.decay_attention(pad(q), pad(k), pad(v), ld, state=S0)
    assert torch.equal(o[0], padded[held])
    for s in (0, n // 2, n - 1):
        cut = slice(int(cu[s]), int(cu[s + 1]))
        if cut.start == cut.stop:
            assert torch.equal(ST[s], S0[s])
            continue
        args = q[:, cut], k[:, cut], v[:, cut], ld, S0[s:s + 1], d ** -0.5
        check_forward(o[:, cut], ST[s:s + 1], *args, dtype == BF16)
        mine = {x: g[x][:, cut] for x in ("dq", "dk", "dv")} | {"dstate": g["dstate"][s:s + 1]}
        check_backward(mine, *args, v[:, cut], S0[s:s + 1], dtype == BF16)


def test_offsets_that_go_back():
    """An offset below the one before it makes an empty sequence, and is reported; nothing is read or written out of range."""
    q, k, v, ld, _ = make(1, 300, 2, 2, 2, 2, 64, BF16, 8, False)
    cu = torch.tensor([0, 200, 100, 300], device="cuda")
    o, ST = ops.decay_attention(q, k, v, ld, cu_seqlens=cu)
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6 and not ST[1].any()
    check_forward(o[:, :100], None, q[:, :200][:, :100], k[:, :100], v[:, :100], ld, None, 64 ** -0.5, True)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("given", ["state", "gradient"])
@pytest.mark.parametrize("T", [100, 1600])
def test_backward_with_one_state(dtype, given, T):
    """A state before without a gradient behind, and the other way round: the missing one is zero."""
    B, H, d = 1, 2, 64
    q, k, v, _, S = make(B, T, H, H, H, H, d, dtype, T + 3)
    ld = torch.tensor([-0.01, -0.2], device="cuda")
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(T)).to(dtype)
    zero = torch.zeros_like(S)
    S0, dST = (S, None) if given == "state" else (None, S)
    g = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST)
    check_backward(g, q, k, v, ld, zero if S0 is None else S0, d ** -0.5, dout, zero if dST is None else dST, dtype == BF16)
    both = ops.decay_attention_bwd(q, k, v, ld, dout, state=zero if S0 is None else S0, dfinal_state=zero if dST is None else dST)
    assert all(torch.equal(g[x], both[x]) for x in both)


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,T,H", [(1, 3000, 2), (1, 1537, 1), (3, 1025, 1)])
def test_long_sequences_in_segments(dtype, d, B, T, H):
    """Few heads and many tokens: a sequence is cut into segments that run at once."""
    q, k, v, ld, S0 = make(B, T, H, H, H, H, d, dtype, T)
    ld = torch.tensor([-0.002, -0.05], device="cuda")[:H]
    kept = S0.clone()
    o, ST = ops.decay_attention(q, k, v, ld, state=S0)
    assert torch.equal(S0, kept)
    check_forward(o, ST, q, k, v, ld, S0, d ** -0.5, dtype == BF16)
    o2, again = ops.decay_attention(q, k, v, ld, state=S0, final_state=S0)  # in place
    assert again is S0 and torch.equal(again, ST) and torch.equal(o2, o)
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(8)).to(dtype)
    dST = torch.randn(B, H, d, d, device="cuda", generator=gen(9))
    g = ops.decay_attention_bwd(q, k, v, ld, dout, state=kept, dfinal_state=dST)
    check_backward(g, q, k, v, ld, kept, d ** -0.5, dout, dST, dtype == BF16)


# (on a GPU of 152 SMs, in bf16) 160 heads: a full round and 8 heads in segments; 192 passes of the gradients: 40 in segments
@pytest.mark.parametrize("d,B,T,aligned", [(128, 10, 700, True), (64, 10, 513, True), (128, 10, 600, False), (128, 10, 511, True)])
def test_more_heads_than_a_round(d, B, T, aligned):
    """The sequences that full rounds leave over run in segments beside whole ones, in place as well."""
    H = 16
    q, k, v, ld, S0 = make(B, T, H, H, H, H, d, BF16, T)
    if not aligned:  # (the fp32 kernel, which cuts all sequences or none)
        q = torch.nn.functional.pad(q, (1, 1))[..., 1:-1]
    kept = S0.clone()
    o, ST = ops.decay_attention(q, k, v, ld, state=S0)
    assert torch.equal(S0, kept)
    check_forward(o, ST, q, k, v, ld, S0, d ** -0.5, aligned)
    o2, again = ops.decay_attention(q, k, v, ld, state=S0, final_state=S0)
    assert again is S0 and torch.equal(again, ST) and torch.equal(o2, o)


def test_one_packed_sequence_of_more_heads_than_a_round():
    q, k, v, ld, S0 = make(1, 700, 160, 160, 160, 160, 64, BF16, 5)
    cu = torch.tensor([3, 680], device="cuda")
    out = torch.full_like(q, 7.0)
    o, ST = ops.decay_attention(q, k, v, ld, state=S0, cu_seqlens=cu, out=out)
    check_forward(o[:, 3:680], ST, q[:, 3:680], k[:, 3:680], v[:, 3:680], ld, S0, 64 ** -0.5, True)
    assert (o[:, :3] == 7).all() and (o[:, 680:] == 7).all()
    dout, dST = torch.randn_like(q), torch.randn_like(S0)
    g = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST, cu_seqlens=cu)
    part = {n: x[:, 3:680] if n != "dstate" else x for n, x in g.items()}
    check_backward(part, q[:, 3:680], k[:, 3:680], v[:, 3:680], ld, S0, 64 ** -0.5, dout[:, 3:680], dST, True)


@pytest.mark.parametrize("d,B,T,Hk,given", [(128, 4, 513, 16, True), (64, 4, 700, 4, True), (64, 4, 640, 16, False)])
def test_gradients_of_more_passes_than_a_round(d, B, T, Hk, given):
    H = 16
    q, k, v, ld, S0 = make(B, T, H, H, Hk, Hk, d, BF16, T, given)
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(8)).to(BF16)
    dST = torch.randn(B, H, d, d, device="cuda", generator=gen(9)) if given else None
    call = lambda: ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST)  # noqa: E731
    g = call()
    check_backward(g, q, k, v, ld, S0, d ** -0.5, dout, dST, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call()
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(captured[n], g[n]) for n in g)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    again = [ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST, stream=s) for s in (None, other)]
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(r[n], g[n]) for r in again for n in g)


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_resumed_calls_and_steps(dtype):
    """A prompt in two calls, then tokens one by one, as the whole prompt in one call."""
    B, T, H, d = 2, 260, 4, 128
    q, k, v, ld, S0 = make(B, T, H, H, 2, 2, d, dtype, 4)
    _, state = ops.decay_attention(q[:, :150], k[:, :150], v[:, :150], ld, state=S0)
    o1, state = ops.decay_attention(q[:, 150:250], k[:, 150:250], v[:, 150:250], ld, state=state, final_state=state)
    outs = [o1] + [ops.decay_attention_step(q[:, t], k[:, t], v[:, t], ld, state)[:, None] for t in range(250, 260)]
    o = torch.cat(outs, 1)
    d64 = lambda x: x.double()  # noqa: E731
    ref, refS = all_pairs(d64(q), d64(k), d64(v), ld, d64(S0), d ** -0.5)
    A, AS = all_pairs(*(x.double().abs() for x in (q, k, v)), ld, S0.double().abs(), d ** -0.5)
    e, eS = eps_of(dtype, d, 2 * T, dtype == BF16)
    close(o, ref[:, 150:], (e * A + R[dtype] * ref.abs())[:, 150:], "o")
    close(state, refS, eS * AS + U * refS.abs(), "state")


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,Hq,Hk,Hv,rows", [(1, 1, 1, 1, 1, 0), (3, 8, 8, 2, 4, 0), (5, 4, 4, 4, 4, 9), (300, 2, 1, 1, 2, 301)])
def test_step(dtype, d, B, H, Hq, Hk, Hv, rows):
    """o: a dot product over d of sums of two (d + 6) u A; a state: three roundings and the power's."""
    g = gen(B + H)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v = n(B, Hq + 1, d + 8).to(dtype)[:, 1:, :d], n(B, Hk, d).to(dtype), n(B, Hv, d + 1).to(dtype)[..., 1:]
    state, ld = n(rows or B, H, d, d), decays(H)
    slots = torch.randperm(rows, device="cuda", generator=g)[:B] if rows else None
    if rows and B > 2:
        slots[1] = -1
    for s in ([None] if slots is None else [slots, slots.int()]):
        before = state.double()
        o = ops.decay_attention_step(q, k, v, ld, state, slots=s, scale=0.25)
        at = torch.arange(B, device="cuda") if s is None else s.long()
        live = at >= 0
        gamma = ld.double().exp()[:, None, None]
        Q, K, V = (x.double().repeat_interleave(H // x.shape[1], 1)[live] for x in (q, k, v))
        kept, new = gamma * before[at[live]], K[..., None] * V[:, :, None]
        ref, mag = kept + new, kept.abs() + new.abs()
        close(state[at[live]], ref, 8 * U * mag, "state")
        rest = torch.ones(state.shape[0], dtype=torch.bool, device="cuda")
        rest[at[live]] = False
        assert torch.equal(state[rest], before[rest].float())
        r = 0.25 * (Q[..., None] * ref).sum(2)
        close(o[live], r, (d + 12) * U * 0.25 * (Q.abs()[..., None] * mag).sum(2) + R[dtype] * r.abs(), "o")
        assert (o[~live] == 0).all()


def test_step_slots_that_are_refused():
    """A slot outside the states, or that an earlier row has, changes nothing."""
    d, H = 64, 2
    q, k, v = (torch.randn(4, H, d, device="cuda", generator=gen(i)) for i in range(3))
    state = torch.randn(3, H, d, d, device="cuda", generator=gen(3))
    alone = state.clone()
    ld = decays(H)
    expect = ops.decay_attention_step(q[:1], k[:1], v[:1], ld, alone, slots=torch.tensor([2], device="cuda"))
    o = ops.decay_attention_step(q, k, v, ld, state, slots=torch.tensor([2, 2, 3, 2 ** 40], device="cuda"))
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6
    assert torch.equal(o[:1], expect) and (o[1:] == 0).all() and torch.equal(state, alone)


def test_offsets_outside_the_tokens_are_held():
    q, k, v, ld, _ = make(1, 40, 2, 2, 2, 2, 64, FP32, 6, False)
    o, _ = ops.decay_attention(q, k, v, ld, cu_seqlens=torch.tensor([-5, 10, 10 ** 12], device="cuda"))
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6
    ref, _ = ops.decay_attention(q, k, v, ld, cu_seqlens=torch.tensor([0, 10, 40], device="cuda"))
    assert torch.equal(o, ref)


def test_gradients_against_differences():
    """<o, dout> + <state, dstate> is linear in each of q, k, v and the state: a difference is the gradient's product.  fp32:
    each of the two calls is off by e A, e and A as in the module's bound (sums of magnitudes, here of the whole scalar)."""
    B, T, H, d = 1, 200, 4, 64
    q, k, v, ld, S0 = make(B, T, H, H, 2, 2, d, FP32, 12)
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(13))
    dST = torch.randn(B, H, d, d, device="cuda", generator=gen(14))
    g = ops.decay_attention_bwd(q, k, v, ld, dout, state=S0, dfinal_state=dST)
    e, _ = eps_of(FP32, d, T, False)

    def scalar(*x):
        o, ST = ops.decay_attention(*x[:3], ld, state=x[3])
        return (o.double() * dout).sum() + (ST.double() * dST).sum()

    x = [q, k, v, S0]
    base = scalar(*x)
    for i, name in enumerate(("dq", "dk", "dv", "dstate")):
        step = torch.randn(x[i].shape, device="cuda", generator=gen(20 + i))
        moved = x[:i] + [x[i] + step] + x[i + 1:]
        A, AS = all_pairs(*(t.double().abs() for t in moved[:3]), ld, moved[3].double().abs(), d ** -0.5)
        room = 4 * e * ((A * dout.abs()).sum() + (AS * dST.abs()).sum())
        # (the step that was made: x + step, rounded, less x)
        made = (moved[i].double() - x[i].double())
        assert abs((scalar(*moved) - base) - (g[name].double() * made).sum()) <= room, name


def test_values_that_are_not_finite_stay_in_later_tokens():
    """fp32 arithmetic: a NaN reaches no output before its own."""
    q, k, v, ld, _ = make(1, 100, 2, 2, 2, 2, 64, FP32, 15, False)
    ref, _ = ops.decay_attention(q, k, v, ld)
    for x in (q, k, v):
        y = x.clone()
        y[:, 45] = float("nan")
        args = [y if t is x else t for t in (q, k, v)]
        o, _ = ops.decay_attention(*args, ld)
        assert torch.equal(o[:, :45], ref[:, :45]) and o[:, 45].isnan().all()


def test_empty():
    ld = decays(2)
    for B, T in ((0, 5), (2, 0)):
        q = torch.empty(B, T, 2, 64, device="cuda")
        S0 = torch.randn(B, 2, 64, 64, device="cuda")
        o, ST = ops.decay_attention(q, q, q, ld, state=S0)
        assert o.shape == q.shape and torch.equal(ST, S0)
        g = ops.decay_attention_bwd(q, q, q, ld, q, state=S0, dfinal_state=S0)
        assert g["dq"].shape == q.shape and torch.equal(g["dstate"], S0)
        _, none = ops.decay_attention(q, q, q, ld, return_state=False)
        assert none is None
    q = torch.empty(0, 2, 64, device="cuda")
    assert ops.decay_attention_step(q, q, q, ld, torch.empty(0, 2, 64, 64, device="cuda")).shape == q.shape


def test_a_layer_end_to_end():
    """As a layer uses them: positions, a prompt, the gated norm, its gradients, then tokens on a pool of states."""
    B, T, H, d = 2, 90, 4, 64
    g = gen(30)
    qkv = torch.randn(B, T, 3 * H * d, device="cuda", generator=g).to(BF16)
    q, k, v = (t.unflatten(-1, (H, d)) for t in qkv.split(H * d, -1))
    gate = torch.randn(B, T, H * d, device="cuda", generator=g).to(BF16)
    positions = torch.arange(T, device="cuda").expand(B, T).contiguous()
    freqs, amplitude = ops.rotary_frequencies(d, scaling="yarn", factor=2.0)
    ld = decays(H)
    qr, kr = ops.rotary(q, k, positions, freqs, amplitude=amplitude)
    pool = torch.zeros(5, H, d, d, device="cuda")
    slots = torch.tensor([3, 1], device="cuda")
    n = T - 1
    o, state = ops.decay_attention(qr[:, :n], kr[:, :n], v[:, :n], ld)
    pool[slots] = state
    last = ops.decay_attention_step(qr[:, n], kr[:, n], v[:, n], ld, pool, slots=slots)
    whole, final = ops.decay_attention(qr, kr, v, ld)
    check_forward(torch.cat([o, last[:, None]], 1), pool[slots], qr, kr, v, ld, None, d ** -0.5, True)
    y = ops.group_norm(whole.flatten(2), None, None, gate, groups=H)
    dnorm = ops.group_norm_bwd(whole.flatten(2), None, None, gate, torch.ones_like(y), groups=H)
    dout = dnorm["dx"].unflatten(-1, (H, d))
    grads = ops.decay_attention_bwd(qr, kr, v, ld, dout)
    check_backward(grads, qr, kr, v, ld, None, d ** -0.5, dout, None, True)
    dq, dk = ops.rotary_bwd(grads["dq"], grads["dk"], positions, freqs, amplitude=amplitude)
    assert dq.shape == q.shape and dk.shape == k.shape and dq.isfinite().all() and dk.isfinite().all()


def _calls(g):
    B, T, H, d = 2, 1500, 2, 128
    q, k, v, ld, S0 = make(B, T, H, H, 1, 1, d, BF16, g)
    dout = torch.randn(B, T, H, d, device="cuda", generator=gen(g + 1)).to(BF16)
    positions = torch.arange(T, device="cuda").expand(B, T).contiguous()
    freqs, _ = ops.rotary_frequencies(d)
    pool = torch.randn(B, H, d, d, device="cuda", generator=gen(g + 2))

    def run(stream=None):
        qr, kr = ops.rotary(q, k, positions, freqs, stream=stream)
        o, ST = ops.decay_attention(qr, kr, v, ld, state=S0, stream=stream)
        gr = ops.decay_attention_bwd(qr, kr, v, ld, dout, state=S0, dfinal_state=S0, stream=stream)
        step = ops.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], ld, pool, stream=stream)
        back = ops.rotary_bwd(gr["dq"], gr["dk"], positions, freqs, stream=stream)
        return [qr, kr, o, ST, *[gr[n] for n in sorted(gr)], step, *back]

    return run, pool, (q, k, v, dout, S0)


def test_streams_and_graphs():
    """On another stream, with stream=, and captured and replayed on other inputs: the same bits."""
    run, pool, inputs = _calls(40)
    start = pool.clone()
    expect = run()
    after = pool.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pool.copy_(start)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = run(side)
    noise = [torch.full_like(x, 3.0) for x in expect]  # (nothing of the call's memory is given out meanwhile)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, expect):
        assert torch.equal(a, b)
    assert torch.equal(pool, after) and len(noise)
    pool.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    other = _calls(50)
    for x, y in zip(inputs, other[2]):
        x.copy_(y)
    pool.copy_(other[1])
    graph.replay()
    expect = other[0]()
    for a, b in zip(got, expect):
        assert torch.equal(a, b)
    assert torch.equal(pool, other[1])


def test_two_graphs_do_not_share_a_workspace():
    runs = [_calls(s) for s in (60, 70)]
    graphs, outs = [], []
    for run, pool, _ in runs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(run())
    starts = [pool.clone() for _, pool, _ in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, gr in zip(streams, graphs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            gr.replay()
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for (run, pool, _), start, out in zip(runs, starts, outs):
        pool.copy_(start)
        for a, b in zip(out, run()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("cores", [False, True])
def test_offsets_past_32_bits(cores):
    """The last of many rows, 2^31 elements and more in.  (Rows of q that are one row again and again are no tiles: that call
    is computed in fp32, and held to its bound.)"""
    B, T, H, d = 9000, 16, 128, 128  # 2.36e9 elements
    v = torch.zeros(B, T, H, d, dtype=BF16, device="cuda")
    q = torch.randn(1, T, 1, d, device="cuda", generator=gen(1)).to(BF16).expand(B, T, H, d)
    if cores:
        q = q.contiguous()
    ld = torch.full((H,), -0.1, device="cuda")
    v[-1, :, -1] = 1.0
    o, _ = ops.decay_attention(q, q, v, ld, return_state=False)
    check_forward(o[-1:], None, q[-1:], q[-1:], v[-1:], ld, None, d ** -0.5, cores)
    assert not o[0].any() and not o[-2].any() and o[-1, :, -1].any()
