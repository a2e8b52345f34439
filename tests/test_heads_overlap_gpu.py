"""Outputs that share elements with inputs are refused through the binding too, nothing is written, and slices that interleave are computed as
tensors of their own are."""
import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu


def make(dtype, seed=1):
    B, T, H, d = 2, 40, 4, 64
    x = torch.randn(B, T + 1, 4 * H * d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)
    return x, [t.unflatten(-1, (H, d)) for t in x[:, :T].split(H * d, -1)], torch.linspace(-0.3, -0.01, H, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_refused_and_nothing_written(dtype):
    x, (q, k, v, o), ld = make(dtype)
    before = x.clone()
    H, d = q.shape[2:]
    later = x[:, 1:].split(H * d, -1)[0].unflatten(-1, (H, d))  # one token into q
    freqs, _ = ops.rotary_frequencies(d)
    positions = torch.arange(40, device="cuda").expand(2, 40).contiguous()
    pool = torch.zeros(2, H, d, d, device="cuda")
    step = torch.randn(3, 2, H, d, device="cuda").to(dtype)
    for call in (lambda: ops.decay_attention(q, k, v, ld, out=later), lambda: ops.decay_attention_bwd(q, k, v, ld, o, out={"dv": later}),
                 lambda: ops.decay_attention_bwd(q.clone(), k, v, ld, o, out={"dq": q, "dk": later}), lambda: ops.rotary(q, k, positions, freqs, out=(later, None)),
                 lambda: ops.rotary(q, k, positions, freqs, out=(None, later)),
                 lambda: ops.decay_attention_step(step[0], step[1], step[2], ld, pool, out=step.flatten(0, 1)[1:3])):
        with pytest.raises((ccq.CCQError, ValueError), match="overlaps"):
            call()
    torch.cuda.synchronize()
    assert torch.equal(x, before) and not pool.any()
    ccq.device_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_slices_that_interleave(dtype):
    x, (q, k, v, o), ld = make(dtype)
    copies = [t.clone() for t in (q, k, v)]
    ref, state = ops.decay_attention(*copies, ld)
    got, again = ops.decay_attention(q, k, v, ld, out=o)
    assert got is o and torch.equal(o, ref) and torch.equal(state, again) and all(torch.equal(a, b) for a, b in zip(copies, (q, k, v)))
    dout = torch.randn_like(ref)
    ref = ops.decay_attention_bwd(*copies, ld, dout)
    grads = torch.empty_like(x)
    out = dict(zip(("dq", "dk", "dv"), (t.unflatten(-1, q.shape[2:]) for t in grads[:, 1:].split(q.shape[2] * q.shape[3], -1))))
    ops.decay_attention_bwd(q, k, v, ld, dout, out=out)
    assert all(torch.equal(out[n], ref[n]) for n in ("dq", "dk", "dv"))
    ccq.device_status()
