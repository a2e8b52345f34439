"""Packed linear attention with a decay for each head: tokens that no sequence holds (padding before the first offset and behind
the last, gaps that offsets going back leave).  Their gradients are zero, whatever the tensors and the workspace held; a new
output is zero there, a given one is left as it was.  All of it is exact: no tolerance."""
import pytest
import torch

from paper_2606_01294_gb300 import ccq, ops

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
NAN = float("nan")
CASES = [  # offsets, tokens; the rows that a sequence holds follow from them
    ([3, 8, 8, 9, 137, 200], 270), ([0, 300], 300), ([40, 300], 300), ([0, 60], 300), ([0], 70), ([9], 70), ([5, 5], 130), ([0, 0, 64], 64)]
BACK = [([50, 10, 20], 300), ([0, 200, 100, 300], 310), ([-5, 10, 10 ** 12], 40), ([90, 20], 100)]


def held_by(cu, T):
    return times_held(cu, T) > 0


def times_held(cu, T):
    """(Offsets that go back may give rows to two sequences: they hold what either writes.)"""
    held = torch.zeros(T, dtype=torch.int32)
    for a, b in zip(cu, cu[1:]):
        begin = min(max(a, 0), T)
        held[begin:min(max(b, begin), T)] += 1
    return held.cuda()


def make(T, H, Hk, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v, dout = (torch.randn(1, T, h, d, device="cuda", generator=g).to(dtype) for h in (H, Hk, Hk, H))
    return q, k, v, dout, torch.linspace(-0.5, -0.001, H, device="cuda")


def poisoned_memory(*shapes_and_types):
    """Blocks of the allocator that a call's new tensors are likely to get, full of NaN."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.full(s, NAN, dtype=t, device="cuda") for s, t in shapes_and_types for _ in range(3)]
    del blocks


def status(expected):
    if not expected:
        ccq.device_status()
        return
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6  # an index outside its range


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("H,Hk", [(4, 4), (4, 2), (6, 1)])
@pytest.mark.parametrize("cu,T", CASES + BACK)
def test_gradients_of_tokens_outside_are_zero(dtype, H, Hk, cu, T):
    d = 64
    q, k, v, dout, ld = make(T, H, Hk, d, dtype, T + H)
    held = held_by(cu, T)
    offsets = torch.tensor(cu, device="cuda")
    for x in (q, k, v, dout):
        x[:, ~held] = NAN  # (what no sequence holds reaches nothing)
    n = len(cu) - 1
    need = ops._size("ccq_decay_attention_bwd_workspace_size", 0, 1, T, H, H, Hk, Hk, d, n, ops._CODE[dtype])
    workspace = torch.full((max(need // 4, 4),), NAN, device="cuda").view(torch.uint8)
    given = {"dq": torch.full_like(q, NAN), "dk": torch.full_like(k, NAN), "dv": torch.full_like(v, NAN)}
    g = ops.decay_attention_bwd(q, k, v, ld, dout, cu_seqlens=offsets, out=given, workspace=workspace)
    poisoned_memory((q.shape, dtype), (k.shape, dtype), ((max(need, 16),), torch.float16))
    new = ops.decay_attention_bwd(q, k, v, ld, dout, cu_seqlens=offsets)
    status((cu, T) in BACK)
    for name in ("dq", "dk", "dv"):
        assert g[name] is given[name]
        assert (g[name][:, ~held] == 0).all(), name
        assert (new[name][:, ~held] == 0).all(), name
        once = times_held(cu, T) == 1
        assert g[name][:, held].isfinite().all() and torch.equal(g[name][:, once], new[name][:, once]), name


@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("cu,T", CASES + BACK)
def test_a_new_output_is_zero_outside(dtype, cu, T):
    """... and one that is given keeps what it held."""
    q, k, v, _, ld = make(T, 4, 4, 128, dtype, T)
    held = held_by(cu, T)
    offsets = torch.tensor(cu, device="cuda").long()
    for x in (q, k, v):
        x[:, ~held] = NAN
    poisoned_memory((q.shape, dtype))
    calls = [ops.decay_attention(q, k, v, ld, cu_seqlens=offsets)[0],
             ops.decay_attention(q, k, v, ld, cu_seqlens=offsets.clamp(-2 ** 31, 2 ** 31 - 1).int(), return_state=False)[0]]
    given = torch.full_like(q, 7.0)
    ops.decay_attention(q, k, v, ld, cu_seqlens=offsets, out=given)
    status((cu, T) in BACK)
    for o in calls:
        assert (o[:, ~held] == 0).all() and o.isfinite().all()
    once = times_held(cu, T) == 1
    assert torch.equal(calls[0][:, once], given[:, once])  # (in bf16 the second call's state has fewer bits: none is handed out)
    assert (given[:, ~held] == 7).all()


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_what_lies_between_the_rows_is_kept(dtype):
    """Gradients in slices of wider tensors, at addresses that no wide access fits: zeros go to the rows' own elements alone."""
    T, H, Hk, d = 150, 4, 2, 64
    q, k, v, dout, ld = make(T, H, Hk, d, dtype, 3)
    wide = {n: torch.full((1, T + 2, h + 1, d + 3), 7.0, dtype=dtype, device="cuda") for n, h in (("dq", H), ("dk", Hk), ("dv", Hk))}
    out = {n: x[:, 1:-1, 1:, 1:d + 1] for n, x in wide.items()}
    ops.decay_attention_bwd(q, k, v, ld, dout, cu_seqlens=torch.tensor([20, 20, 90], device="cuda"), out=out)
    ccq.device_status()
    for n, x in out.items():
        assert (x[:, :20] == 0).all() and (x[:, 90:] == 0).all() and (x[:, 20:90] != 0).any(), n
        x.fill_(7.0)
        assert (wide[n] == 7).all(), n


@pytest.mark.parametrize("n", [300, 2000])
def test_many_sequences_and_much_padding(n):
    """More words of rows than CTAs that zero them, more sequences than threads."""
    H, d = 2, 64
    lengths = torch.randint(0, 9, (n,), generator=torch.Generator().manual_seed(n))
    before, after = 5000, 33333
    T = before + int(lengths.sum()) + after
    cu = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)]).cuda() + before
    q, k, v, dout, ld = make(T, H, 1, d, BF16, n)
    out = {"dq": torch.full_like(q, NAN), "dk": torch.full_like(k, NAN), "dv": torch.full_like(v, NAN)}
    ops.decay_attention_bwd(q, k, v, ld, dout, cu_seqlens=cu, out=out)
    poisoned_memory((q.shape, BF16))
    out["o"] = ops.decay_attention(q, k, v, ld, cu_seqlens=cu)[0]
    ccq.device_status()
    for x in out.values():
        assert not x[:, :before].any() and not x[:, T - after:].any() and x.isfinite().all()
        assert x[:, before:T - after].any(-1).any(-1).all()


def test_captured_and_replayed_on_other_offsets():
    T, H, d = 400, 4, 64
    q, k, v, dout, ld = make(T, H, 2, d, BF16, 9)
    cu = torch.tensor([10, 100, 390], device="cuda")
    out = {"dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v)}
    call = lambda: (ops.decay_attention_bwd(q, k, v, ld, dout, cu_seqlens=cu, out=out), ops.decay_attention(q, k, v, ld, cu_seqlens=cu)[0])  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g, o = call()
    for offsets in ([10, 100, 390], [200, 300, 301], [0, 0, 0], [0, 5, 400]):
        cu.copy_(torch.tensor(offsets))
        for x in (*out.values(), o):
            x.fill_(NAN)
        graph.replay()
        held = held_by(offsets, T)
        for x in (*out.values(), o):
            assert (x[:, ~held] == 0).all() and x.isfinite().all()
    ccq.device_status()
