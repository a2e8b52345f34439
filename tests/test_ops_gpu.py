"""GPU checks of the operators around the token mixer (ccq_ops.h) against plain implementations in 64 bits.

Bounds, set before the first run.  u = 2^-24 is fp32's half step; an output is rounded once, by half a step of
its type: r = 2^-8 of its value in bf16 (8 significant bits), u in fp32.
  embed        one product: (u + r) |ref|.
  embed_grad   a sum of k terms and a product: (k + 2) u sum|term| + r |ref|.
  group_norm   about 40 operations and sums of at most 24 levels: ARITH = 1e-5 of the largest output (40 u = 2.4e-6, and
               exponentials within 2^-21), + r |ref|; the mean's own rounding is amplified by |mean| / std.
  gradients of weight and bias: sums over n tokens, (n u + ARITH) of the sum of magnitudes, + r.
  policy loss  log-probabilities: (|z| + |log Z|) 8 u, sums of V terms in trees; gradients ARITH of the row's largest, + r.
  AdamW        8 operations: 1e-6 of each term's magnitude; 8-bit codes are equal to the fp32 operations' codes.
"""
import ctypes
import math
import threading

import pytest
import torch

from paper_2606_01294_gb300 import ccq, inputs, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ARITH = 1e-5
R = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(autouse=True)
def _status():
    yield
    ccq.device_status()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


def close(x, ref, bound, what=""):
    err = (x.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst {float((err / bound).max()):.3g} of the bound"


def strided(t, pad=0, offset=0):
    """t's values in a buffer with `pad` elements between rows, starting `offset` elements in."""
    rows, width = t.shape
    buf = torch.full((rows * (width + pad) + offset + 8,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(t)
    return view


# ---------------------------------------------------------------- embedding


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,width,pad,offset", [(1, 1, 1, 0, 0), (1, 10, 2048, 0, 0), (7, 33, 64, 8, 8), (300, 50, 500, 0, 0),
                                                     (129, 1000, 1001, 0, 0), (64, 20, 256, 1, 1), (1000, 999, 4096, 0, 0),
                                                     (5, 9, 6, 2, 2)])
def test_embed(dtype, n, rows, width, pad, offset):
    g = gen(n + width)
    table = strided(randn(g, rows, width, dtype=dtype), pad, offset)
    ids = torch.randint(0, rows, (n,), device="cuda", generator=g)
    for i in (ids, ids.int()):
        y = ops.embed(table, i, scale=1.7)
        ref = table.double()[ids] * float(torch.tensor(1.7, dtype=torch.float32))
        close(y, ref, (U + R[dtype]) * ref.abs() + 1e-38)
    out = strided(torch.zeros(n, width, device="cuda", dtype=dtype), 3, 1)
    assert torch.equal(ops.embed(table, ids, scale=1.7, out=out), y)


def test_embed_shapes_and_empty():
    table = randn(gen(1), 12, 64, dtype=torch.bfloat16)
    ids = torch.arange(12, device="cuda").view(3, 4)
    assert torch.equal(ops.embed(table, ids), table.view(3, 4, 64))
    assert ops.embed(table, ids[:0]).shape == (0, 4, 64)


def test_embed_reports_ids_outside_the_table():
    table = randn(gen(2), 10, 64)
    ids = torch.tensor([3, 10, -1, 2 ** 40, 9], device="cuda")
    y = ops.embed(table, ids)
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6
    assert torch.equal(y[0], table[3]) and torch.equal(y[4], table[9]) and not y[1:4].any()
    d = ops.embed_grad(torch.ones(5, 64, device="cuda"), ids, 10)
    with pytest.raises(ccq.CCQError):
        ccq.device_status()
    assert torch.equal(d.sum(1).nonzero()[:, 0], torch.tensor([3, 9], device="cuda"))


@pytest.mark.parametrize("first", ["index", "timeout"])
def test_an_index_does_not_hide_a_timeout(first):
    """One word reports for all kernels: outputs that are not valid come before an id that made a zero row."""
    lib = ccq.load_library()
    lib.ccq_diag_wait_timeout.argtypes = [ctypes.c_void_p]
    lib.ccq_diag_wait_timeout.restype = ctypes.c_int
    steps = [lambda: ops.embed(torch.ones(4, 64, device="cuda"), torch.tensor([0, 9], device="cuda")),
             lambda: lib.ccq_diag_wait_timeout(torch.cuda.current_stream().cuda_stream)]
    for step in steps if first == "index" else steps[::-1]:
        step()
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == ccq.CCQ_ERR_TIMEOUT


def test_embed_offsets_past_32_bits():
    rows, width = 1_100_000, 2048  # 2.25e9 elements
    table = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([rows - 1, 1_048_577, 0, 5], device="cuda")
    table[ids] = torch.arange(1, 5, device="cuda", dtype=torch.bfloat16)[:, None]
    assert torch.equal(ops.embed(table, ids)[:, -1].float(), torch.arange(1, 5, device="cuda").float())
    out = ops.embed_grad(torch.ones(4, width, dtype=torch.bfloat16, device="cuda"), ids, rows, out=table)
    assert out is table
    assert torch.equal(torch.nonzero(table[:, -1])[:, 0], ids.sort().values)
    assert int((table[:, 0] != 0).sum()) == 4


def _ids(kind, n, rows, g):
    if kind == "same":
        return torch.full((n,), rows - 1, device="cuda")
    if kind == "zipf":
        return (torch.exp(torch.rand(n, device="cuda", generator=g) * math.log(rows)).long() - 1).clamp_(0, rows - 1)
    if kind == "half":  # half of the tokens are one id in the middle
        ids = torch.randint(0, rows, (n,), device="cuda", generator=g)
        return torch.where(torch.rand(n, device="cuda", generator=g) < 0.5, rows // 2, ids)
    return torch.randint(0, rows, (n,), device="cuda", generator=g)


def _embed_grad_ref(dout, ids, rows, scale, padding=None):
    d = dout.double() * scale
    if padding is not None:
        d = torch.where((ids == padding)[:, None], 0.0, d)
    ref = torch.zeros(rows, d.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids, d)
    mass = torch.zeros_like(ref).index_add_(0, ids, d.abs())
    count = torch.bincount(ids, minlength=rows).double()[:, None]
    return ref, mass, count


@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in DTYPES for b in DTYPES])
@pytest.mark.parametrize("n,rows,width,kind", [(1, 1, 64, "same"), (1, 3000, 256, "even"), (31, 7, 33, "even"), (33, 32, 8, "same"),
                                               (500, 1000, 500, "zipf"), (4097, 513, 264, "half"), (9000, 300, 64, "same"),
                                               (20000, 40000, 72, "zipf"), (3000, 1, 130, "same"), (2500, 1200000, 8, "even")])
def test_embed_grad(dtype, out_dtype, n, rows, width, kind):
    g = gen(n + rows)
    ids = _ids(kind, n, rows, g)
    dout = randn(g, n, width, dtype=dtype)
    d = ops.embed_grad(dout, ids, rows, scale=3.0, dtype=out_dtype)
    ref, mass, count = _embed_grad_ref(dout, ids, rows, 3.0)
    close(d, ref, (count + 2) * U * mass + R[out_dtype] * ref.abs() + 1e-38)
    assert not d[count[:, 0] == 0].any()
    assert torch.equal(d, ops.embed_grad(dout, ids.int(), rows, scale=3.0, dtype=out_dtype))  # same bits again


@pytest.mark.parametrize("n,rows,width,kind", [(256, 40, 2048, "zipf"), (257, 40, 2048, "zipf"), (200, 20000, 1030, "even"), (256, 3, 40, "same"),
                                               (64, 5000, 4100, "half"), (2, 70000, 7, "even")])
@pytest.mark.parametrize("dtype,out_dtype", [(a, b) for a in DTYPES for b in DTYPES])
def test_embed_grad_few_ids(dtype, out_dtype, n, rows, width, kind):
    """On both sides of the count up to which no sort is made; some ids are padding."""
    g = gen(n + width)
    ids = _ids(kind, n, rows, g)
    dout = randn(g, n, width, dtype=dtype)
    pad = int(ids[n // 2]) if kind != "same" else 0
    d = ops.embed_grad(dout, ids, rows, scale=0.5, padding_id=pad, dtype=out_dtype)
    ref, mass, count = _embed_grad_ref(dout, ids, rows, 0.5, padding=pad)
    close(d, ref, (count + 2) * U * mass + R[out_dtype] * ref.abs() + 1e-38)
    assert not d[pad].any()


@pytest.mark.parametrize("n,rows,width,kind", [(131072, 5000, 16, "zipf"), (200001, 3000, 8, "half"), (300000, 400000, 8, "zipf"),
                                               (150000, 100, 24, "same"), (3000, 300000, 64, "zipf"), (40000, 513, 40, "even")])
def test_embed_grad_long_lists_and_large_tables(n, rows, width, kind):
    """Lists that the sort exchanges through global memory, runs of thousands of pieces, and every cluster size."""
    g = gen(n)
    ids = _ids(kind, n, rows, g)
    dout = randn(g, n, width)
    d = ops.embed_grad(dout, ids, rows)
    ref, mass, count = _embed_grad_ref(dout, ids, rows, 1.0)
    close(d, ref, (count + 2) * U * mass + U * ref.abs() + 1e-38)
    assert torch.equal(d, ops.embed_grad(dout, ids, rows))


@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (1, 0), (0, 1), (4, 2)])
def test_embed_grad_strides_and_padding(pad, offset):
    g = gen(5)
    n, rows, width = 700, 90, 96
    ids = _ids("zipf", n, rows, g)
    values = randn(g, n, width, dtype=torch.bfloat16)
    values[ids == 1] = float("nan")  # the padding rows are not read
    out = strided(torch.full((rows, width), 7.0, device="cuda"), pad, offset)
    d = ops.embed_grad(strided(values, pad, offset), ids, rows, padding_id=1, out=out)
    ref, mass, count = _embed_grad_ref(torch.nan_to_num(values), ids, rows, 1.0, padding=1)
    close(d, ref, (count + 2) * U * mass + U * ref.abs() + 1e-38)
    assert not d[1].any()


def test_embed_grad_of_nothing():
    d = ops.embed_grad(torch.empty(0, 40, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), 21)
    assert d.shape == (21, 40) and not d.any()


def test_embed_grad_by_differences():
    g = gen(6)
    ids = _ids("zipf", 200, 50, g)
    table, dout, step = randn(g, 50, 24), randn(g, 200, 24), randn(g, 50, 24)
    f = lambda t: float((ops.embed(t, ids, scale=2.0).double() * dout.double()).sum())  # noqa: E731
    slope = float((ops.embed_grad(dout, ids, 50, scale=2.0).double() * step.double()).sum())
    # linear in the table: the difference has only rounding, 4800 products of size ~2 to 2^-24
    assert abs((f(table + step) - f(table - step)) / 2 - slope) < 4800 * 8 * 4 * U


# ---------------------------------------------------------------- group norm


def _act(name, u):
    return u if name == "none" else torch.sigmoid(u) * (u if name == "silu" else 1)


def _norm64(x, w, b, gate, groups, act, centered, eps):
    X = x.double().view(x.shape[0], groups, -1).requires_grad_()
    W = torch.ones(x.shape[1], dtype=torch.float64, device="cuda") if w is None else w.double()
    B = torch.zeros(x.shape[1], dtype=torch.float64, device="cuda") if b is None else b.double()
    W, B = W.view(groups, -1).requires_grad_(), B.view(groups, -1).requires_grad_()
    G = None if gate is None else gate.double().view_as(X).requires_grad_()
    dev = X - X.mean(-1, keepdim=True) if centered else X
    u = dev / (dev.square().mean(-1, keepdim=True) + eps).sqrt() * W + B
    y = _act(act, u) if G is None else u * _act(act, G)
    return y, (X, W, B, G)


NORM_SIZES = [(1, 1, 1), (1, 128, 1), (3, 256, 2), (257, 2048, 16), (100, 1024, 16), (33, 1152, 12), (17, 165, 5), (50, 2000, 4),
              (40, 2048, 1), (9, 4096, 1), (7, 9000, 2), (5, 5000, 1), (1000, 64, 64), (70, 48, 3), (6, 600, 1), (130, 320, 5)]
# every width of access, accesses a thread and team
NORM_SIZES += [(9, 130, 1), (5, 402, 1), (4, 1030, 1), (7, 301, 1), (3, 1001, 1), (11, 135, 3), (13, 62, 2), (21, 24, 3), (6, 32, 1), (8, 18, 1),
               (900, 256, 16)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,channels,groups", NORM_SIZES)
@pytest.mark.parametrize("act,gated,centered", [("silu", True, True), ("silu", False, False), ("sigmoid", True, False), ("none", False, True)])
def test_group_norm_and_gradients(dtype, tokens, channels, groups, act, gated, centered):
    g = gen(tokens + channels)
    x = randn(g, tokens, channels) * 0.7 + 0.3
    x, dy = x.to(dtype), randn(g, tokens, channels, dtype=dtype)
    w, b = (1 + 0.2 * randn(g, channels)).to(dtype), (0.3 * randn(g, channels)).to(dtype)
    gate = randn(g, tokens, channels, dtype=dtype) if gated else None
    how = dict(groups=groups, activation=act, centered=centered, eps=1e-3)
    out, leaves = _norm64(x, w, b, gate, groups, act, centered, 1e-3)
    ref = out.detach()
    y = ops.group_norm(x, w, b, gate, **how)
    r = R[dtype]
    # with one channel a group, or a small deviation, the mean's rounding counts 1 / std times
    amp = 1 if not centered else float((x.double().abs().max() / math.sqrt(1e-3)))
    tol = ARITH * (amp if channels // groups < 8 else 1)
    close(y, ref.view_as(y), r * ref.abs().view_as(y) + tol * max(1.0, float(ref.abs().max())), "y")
    got = ops.group_norm_bwd(x, w, b, gate, dy, **how)
    grads = torch.autograd.grad(out, [t for t in leaves if t is not None], dy.double().view_as(out))
    names = ["dx", "dweight", "dbias"] + (["dgate"] if gated else [])
    assert set(got) == set(names)
    du = dy.double().abs().view(tokens, groups, -1) * 1.2 * (1 if gate is None else gate.double().abs().view_as(ref) + 1)
    for name, e in zip(names, grads):
        e = e.reshape(got[name].shape)
        if name in ("dweight", "dbias"):
            mass = (du * (1 if name == "dbias" else math.sqrt(channels // groups))).sum(0).view(-1)
            bound = (tokens * U + tol) * mass + r * e.abs()
        else:
            bound = r * e.abs() + tol * max(1.0, float(e.abs().max()))
        close(got[name], e, bound, name)


@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (2, 2), (0, 1), (0, 4)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_group_norm_strides(dtype, pad, offset):
    g = gen(3)
    make = lambda: randn(g, 37, 512, dtype=dtype)  # noqa: E731
    x, gate, dy = make(), make(), make()
    w, b = 1 + 0.1 * randn(g, 512), 0.1 * randn(g, 512)  # fp32 parameters of a bf16 layer
    a = ops.group_norm(x, w, b, gate, groups=4)
    s = ops.group_norm(strided(x, pad, offset), w, b, strided(gate, pad, offset), groups=4, out=strided(make(), pad, offset))
    close(s, a.double(), 2 * R[dtype] * a.double().abs() + ARITH * 8, "y")
    p = ops.group_norm_bwd(x, w, b, gate, dy, groups=4)
    q = ops.group_norm_bwd(strided(x, pad, offset), w, b, strided(gate, pad, offset), strided(dy, pad, offset), groups=4,
                           out={"dx": strided(make(), pad, offset), "dgate": strided(make(), pad, offset)})
    for n in p:
        close(q[n], p[n].double(), 2 * R[p[n].dtype] * p[n].double().abs() + ARITH * float(p[n].abs().max()) * 4, n)


def test_group_norm_keeps_tokens_apart():
    g = gen(4)
    x, gate, dy = (randn(g, 300, 256, dtype=torch.bfloat16) for _ in range(3))
    w = torch.ones(256, device="cuda")
    y, d = ops.group_norm(x, w, None, gate, groups=2), ops.group_norm_bwd(x, w, None, gate, dy, groups=2)
    x2 = x.clone()
    x2[7, 3], x2[100, 200] = float("nan"), float("inf")
    y2, d2 = ops.group_norm(x2, w, None, gate, groups=2), ops.group_norm_bwd(x2, w, None, gate, dy, groups=2)
    for a, b in ((y, y2), (d["dx"], d2["dx"]), (d["dgate"], d2["dgate"])):
        same = (a == b).view(300, 2, 128).all(-1)
        assert int((~same).sum()) == 2 and not same[7, 0] and not same[100, 1]
    assert torch.isnan(y2[7, :128]).all()


def test_group_norm_large_mean_and_constant_groups():
    x = 1000 + randn(gen(5), 20, 128)
    x[3] = 1000.0  # a constant group: the output is the bias
    b = torch.linspace(-1, 1, 128, device="cuda")
    y = ops.group_norm(x, None, b, groups=1, activation="none")
    ref, _ = _norm64(x, None, b, None, 1, "none", True, 1e-5)
    # the mean of 128 values near 1000 has an error of at most 7 levels of half steps, 7 * 2^-24 * 1000
    keep = torch.arange(20, device="cuda") != 3
    close(y[keep], ref.detach().view_as(y)[keep], 8 * U * 1000 * 2 + ARITH * 5)
    close(y[3:4], b.double()[None], 8 * U * 1000 / math.sqrt(1e-5))


def test_group_norm_without_parameters_and_empty():
    x = randn(gen(6), 10, 64, dtype=torch.bfloat16)
    d = ops.group_norm_bwd(x, None, None, None, x, groups=1)
    assert set(d) == {"dx"}
    w = torch.ones(64, device="cuda")
    d = ops.group_norm_bwd(x[:0], w, None, None, x[:0], groups=1)
    assert d["dx"].shape == (0, 64) and not d["dweight"].any()
    assert ops.group_norm(x[:0], groups=2).shape == (0, 64)


def test_group_norm_gradients_into_given_tensors():
    x, dy = (randn(gen(7), 30, 96) for _ in range(2))
    w = torch.ones(96, device="cuda")
    want = ops.group_norm_bwd(x, w, None, None, dy, groups=3)
    out = {"dx": torch.empty_like(x), "dweight": torch.empty_like(w), "dbias": None}
    got = ops.group_norm_bwd(x, w, None, None, dy, groups=3, out=out)
    for name in ("dx", "dweight"):
        assert got[name] is out[name] and torch.equal(got[name], want[name])
    for name, t in (("dbias", torch.empty(1, device="cuda")), ("dgate", torch.empty(1, device="cuda"))):
        with pytest.raises(ValueError, match=name):
            ops.group_norm_bwd(x, w, None, None, dy, groups=3, out={name: t})


def test_group_norm_gradients_by_differences():
    g = gen(8)
    x, gate, dy = randn(g, 6, 96), randn(g, 6, 96), randn(g, 6, 96)
    w, b = 1 + 0.1 * randn(g, 96), 0.1 * randn(g, 96)
    steps = [randn(g, *t.shape) for t in (x, w, b, gate)]
    h = 1e-2
    f = lambda s: float((ops.group_norm(*(t + s * h * e for t, e in zip((x, w, b, gate), steps)), groups=3).double()  # noqa: E731
                         * dy.double()).sum())
    d = ops.group_norm_bwd(x, w, b, gate, dy, groups=3)
    slope = sum(float((d[n].double() * e.double()).sum()) for n, e in zip(("dx", "dweight", "dbias", "dgate"), steps))
    # h^2 third derivatives (of order one, 576 terms) and rounding 576 * 1e-6 / h
    assert abs((f(1) - f(-1)) / (2 * h) - slope) < 576 * (h * h + 1e-6 / h)


def test_group_norm_offsets_past_32_bits():
    """More than 2^31 elements, then rows that lie more than 2^31 elements apart: a token's result is that of a call on it alone."""
    tokens, channels = 1_100_000, 2048  # 2.25e9 elements
    g = gen(9)
    x = torch.zeros(tokens, channels, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1_048_575, 1_048_576, tokens - 2, tokens - 1], device="cuda")
    some, dsome = randn(g, 5, channels, dtype=torch.bfloat16), randn(g, 5, channels, dtype=torch.bfloat16)
    x[rows] = some
    w, b = 1 + 0.1 * randn(g, channels), 0.1 * randn(g, channels)
    how = dict(groups=16, activation="silu")
    y = ops.group_norm(x, w, b, x, **how)
    assert torch.equal(y[rows], ops.group_norm(some, w, b, some, **how))
    dy = y.zero_()
    dy[rows] = dsome
    got = ops.group_norm_bwd(x, w, None, None, dy, out={"dx": dy}, **how)
    want = ops.group_norm_bwd(some, w, None, None, dsome, **how)
    assert torch.equal(got["dx"][rows], want["dx"])
    # five tokens' terms in the sums, in another order, and zeros
    close(got["dweight"], want["dweight"].double(), 10 * U * (dsome.double().abs() * 1.1 * math.sqrt(128)).sum(0))
    assert int((got["dx"].view(tokens, -1) != 0).any(1).sum()) == 5
    del x, y, dy, got
    stride = 1_200_000_000
    far = torch.zeros(2 * stride + 256, dtype=torch.bfloat16, device="cuda").as_strided((3, 256), (stride, 1))
    far.copy_(some[:3, :256])
    assert torch.equal(ops.group_norm(far, groups=2), ops.group_norm(some[:3, :256], groups=2))
    p = ops.group_norm_bwd(far, None, None, None, far, groups=2)["dx"]
    assert torch.equal(p, ops.group_norm_bwd(far.contiguous(), None, None, None, far.contiguous(), groups=2)["dx"])


# ---------------------------------------------------------------- policy loss


def _policy_inputs(n, vocab, dtype, seed, masked=0, spread=2.0):
    g = gen(seed)
    logits = (spread * randn(g, n, vocab)).to(dtype)
    actions = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    logp = torch.log_softmax(logits.double(), -1).gather(1, actions[:, None])[:, 0]
    old = (logp + 0.3 * torch.randn(n, device="cuda", generator=g)).float()
    ref = (logp + 0.3 * torch.randn(n, device="cuda", generator=g)).float()
    adv, w = randn(g, n), torch.rand(n, device="cuda", generator=g) + 0.1
    w[torch.randperm(n, device="cuda", generator=g)[:masked]] = 0
    return logits, actions, old, ref, adv, w


def _policy64(logits, actions, old, ref, adv, w, clip, kl, temperature):
    z = (logits.double() / temperature).requires_grad_()
    logp = torch.log_softmax(z, -1).gather(1, actions[:, None])[:, 0]
    ratio = (logp - old.double()).exp()
    a = adv.double()
    each = -torch.minimum(ratio * a, ratio.clamp(1 - clip[0], 1 + clip[1]) * a)
    if ref is not None:
        d = ref.double() - logp
        each = each + kl * (d.exp() - d - 1)
    live = w != 0
    loss = (w.double() * each)[live].sum()
    grad = torch.autograd.grad(loss, z)[0] / temperature if live.any() else torch.zeros_like(z)
    edge = ((ratio - (1 - clip[0])).abs() < 1e-4) | ((ratio - (1 + clip[1])).abs() < 1e-4)  # either slope is right there
    return loss.detach(), torch.where(live, logp.detach(), 0), grad, edge, (w.double() * each.detach()).abs()[live].sum()


POLICY_SIZES = [(1, 1), (1, 2), (3, 17), (5, 1000), (64, 4096), (130, 32000), (9, 50001), (4, 128001), (3, 300007), (2, 1000003), (300, 64)]


def _logp_bound(logits, temperature):
    z = logits.double().abs().amax(-1) / temperature
    return 8 * U * (2 * z + math.log(logits.shape[-1]) + 1) + 1e-6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab", POLICY_SIZES)
def test_policy_loss(dtype, n, vocab):
    x = _policy_inputs(n, vocab, dtype, n + vocab, masked=n // 3)
    logits, actions, old, ref, adv, w = x
    clip, kl, temperature = (0.2, 0.3), 0.1, 0.8
    loss, logp, grad, edge, mass = _policy64(*x, clip, kl, temperature)
    got = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, clip=clip, kl_coef=kl, temperature=temperature)
    tol = _logp_bound(logits, temperature)
    close(got["logp"], logp, tol + U * logp.abs(), "logp")
    worst = float(tol.max()) * 4 + ARITH
    close(got["loss"], loss, worst * mass + 1e-30, "loss")
    keep = ~edge
    top = grad.abs().amax(1, keepdim=True)
    close(got["dlogits"][keep], grad[keep], (R[dtype] * grad.abs() + (worst + ARITH) * 4 * top + 1e-38)[keep], "dlogits")
    assert not got["dlogits"][w == 0].any()
    # without the gradient, and in place of the logits
    alone = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, clip=clip, kl_coef=kl, temperature=temperature, grad=False)
    assert torch.equal(alone["loss"], got["loss"]) and torch.equal(alone["logp"], got["logp"])
    over = logits.clone()
    again = ops.policy_loss(over, actions.int(), old, adv, ref_logp=ref, weights=w, clip=clip, kl_coef=kl, temperature=temperature, dlogits=over)
    assert again["dlogits"] is over and torch.equal(over, got["dlogits"]) and torch.equal(again["loss"], got["loss"])
    score = ops.token_logp(logits, actions, temperature=temperature)
    live = w != 0
    assert torch.equal(score[live], got["logp"][live])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab", [(1000, 30000), (16500, 16400), (170000, 7), (3000, 500), (700, 9001)])
def test_policy_loss_many_rows(dtype, n, vocab):
    """Many rows for a CTA (dealt out by rank, strided, and in several batches).  The slope's error is its derivative by
    logp, w (|r A| where that counts + kl exp(d)), times logp's: it can be far above its value's rounding, as where a clipped
    token's KL term is near zero."""
    x = _policy_inputs(n, vocab, dtype, n + vocab, masked=n // 3)
    logits, actions, old, ref, adv, w = x
    clip, kl, temperature = (0.2, 0.3), 0.1, 0.8
    loss, logp, grad, edge, mass = _policy64(*x, clip, kl, temperature)
    got = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, clip=clip, kl_coef=kl, temperature=temperature)
    tol = _logp_bound(logits, temperature)
    close(got["logp"], logp, tol + U * logp.abs(), "logp")
    close(got["loss"], loss, (float(tol.max()) * 4 + ARITH) * mass + 1e-30, "loss")
    live = w != 0
    lp = torch.log_softmax(logits.double() / temperature, -1).gather(1, actions[:, None])[:, 0]
    moved = w.double() * ((lp - old.double()).exp() * adv.double().abs() + kl * (ref.double() - lp).exp()) / temperature
    slope = (tol + U * logp.abs() + 8 * U) * moved
    top = grad.abs().amax(1, keepdim=True)
    bound = R[dtype] * grad.abs() + slope[:, None] + 4 * (ARITH + tol.max()) * top + 1e-38
    keep = ~edge & live
    close(got["dlogits"][keep], grad[keep], bound[keep], "dlogits")
    assert not got["dlogits"][~live].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab", [(9000, 1003), (5000, 8197), (2500, 33001), (700, 70001)])
def test_token_logp_many_odd_rows(dtype, n, vocab):
    """Rows of every alignment in turn through each buffer, without a gradient: a buffer's cells are written by bulk copies
    in one row and by ordinary stores (a row's first and last elements) in another."""
    g = gen(n)
    logits, actions = randn(g, n, vocab).mul_(2).to(dtype), torch.randint(0, vocab, (n,), device="cuda", generator=g)
    # half of the actions on a row's first and last elements
    actions[::4], actions[1::4] = 0, vocab - 1
    logp = torch.cat([torch.log_softmax(x.double() / 0.8, -1).gather(1, a[:, None])[:, 0]
                      for x, a in zip(logits.split(500), actions.split(500))])
    bound = _logp_bound(logits, 0.8) + U * logp.abs()
    for _ in range(3):
        close(ops.token_logp(logits, actions, temperature=0.8), logp, bound, "logp")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 8), (3, 5), (2, 4), (16, 0)])
@pytest.mark.parametrize("vocab", [3000, 40008, 70001])
def test_policy_loss_strides(dtype, pad, offset, vocab):
    logits, actions, old, ref, adv, w = _policy_inputs(11, vocab, dtype, 77)
    how = dict(ref_logp=ref, kl_coef=0.1, grad_scale=512.0)
    a = ops.policy_loss(logits, actions, old, adv, **how)
    for out_offset in (offset, offset + 1):
        out = strided(torch.zeros_like(logits), pad, out_offset)
        b = ops.policy_loss(strided(logits, pad, offset), actions, old, adv, dlogits=out, **how)
        close(b["loss"], a["loss"].double(), 1e-5 * float(a["loss"].abs()) + 1e-6)
        close(b["logp"], a["logp"].double(), _logp_bound(logits, 1.0))
        top = a["dlogits"].double().abs().amax(1, keepdim=True)
        close(b["dlogits"], a["dlogits"].double(), 2 * R[dtype] * a["dlogits"].double().abs() + 4 * ARITH * top)


def test_policy_loss_masked_tokens_are_not_read():
    logits, actions, old, ref, adv, w = _policy_inputs(40, 900, torch.bfloat16, 9, masked=15)
    clean = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, kl_coef=0.1)
    dead = w == 0
    logits, actions, old, ref, adv = (t.clone() for t in (logits, actions, old, ref, adv))
    logits[dead], old[dead], ref[dead], adv[dead] = float("nan"), float("nan"), float("inf"), float("nan")
    actions[dead] = -7
    got = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, kl_coef=0.1)
    for n in clean:
        assert torch.equal(got[n], clean[n]), n
    none = ops.policy_loss(logits, actions, old, adv, weights=torch.zeros_like(w))
    assert float(none["loss"]) == 0 and not none["dlogits"].any() and not none["logp"].any()


def test_policy_loss_infinite_logits_and_bad_actions():
    logits, actions, old, ref, adv, w = _policy_inputs(6, 5000, torch.float32, 10)
    banned = torch.rand(6, 5000, device="cuda", generator=gen(1)) < 0.5
    banned.scatter_(1, actions[:, None], False)
    banned[0] = True
    banned[0, actions[0]] = False  # one token left: certain
    logits = logits.masked_fill(banned, float("-inf"))
    logits[1] = torch.where(banned[1], logits[1], torch.finfo(torch.float32).min)  # the lowest finite value
    old = torch.log_softmax(logits.double(), -1).gather(1, actions[:, None])[:, 0].float() + 0.1
    got = ops.policy_loss(logits, actions, old, adv, weights=w, clip=(10.0, 10.0))
    loss, logp, grad, _, mass = _policy64(logits, actions, old, None, adv, w, (10.0, 10.0), 0, 1.0)
    close(got["logp"], logp, torch.full_like(logp, 1e-5))
    close(got["dlogits"], grad, 1e-5 * grad.abs() + 1e-5 * grad.abs().amax(1, keepdim=True) + 1e-7)
    assert not got["dlogits"][banned].any() and float(got["logp"][0]) == 0
    bad = actions.clone()
    bad[2], bad[4] = 5000, -1
    part = ops.policy_loss(logits, bad, old, adv, weights=w, clip=(10.0, 10.0))
    with pytest.raises(ccq.CCQError) as e:
        ccq.device_status()
    assert e.value.status == 6
    for i in (0, 1, 3, 5):
        assert torch.equal(part["dlogits"][i], got["dlogits"][i])
    assert not part["dlogits"][[2, 4]].any() and float(part["logp"][2]) == 0
    score = ops.token_logp(logits, bad)
    with pytest.raises(ccq.CCQError):
        ccq.device_status()
    assert torch.isnan(score[[2, 4]]).all() and torch.isfinite(score[[0, 1, 3, 5]]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [5000, 1000003])  # staged rows, and rows that are read twice
@pytest.mark.parametrize("temperature", [0.8, 1.0, 1.5])
def test_policy_loss_of_an_action_at_the_lowest_value(dtype, vocab, temperature):
    """A mask of the type's lowest value on the action itself: divided by a temperature below 1 it is below every fp32
    number, so its log-probability is -inf; the ratio is 0, the loss finite, and nothing of the row moves."""
    logits, actions, old, ref, adv, w = _policy_inputs(6, vocab, dtype, 11)
    masked = torch.tensor([0, 3, 4], device="cuda")
    adv[0], adv[3] = 1.5, -0.7  # both sides of the smaller term
    logits[masked, actions[masked]] = torch.finfo(dtype).min
    clip = (0.2, 0.3)
    loss, logp, grad, edge, mass = _policy64(logits, actions, old, None, adv, w, clip, 0, float(torch.tensor(temperature)))
    got = ops.policy_loss(logits, actions, old, adv, weights=w, clip=clip, temperature=temperature)
    live = torch.tensor([1, 2, 5], device="cuda")
    live = live[~edge[live]]
    # masked: lowest / temperature, a quotient, a sum and its rounding: 4 u of it, or beyond fp32: -inf
    low = torch.where(logp.float().isinf(), float("-inf"), logp)[masked]
    if temperature < 1:
        assert torch.isneginf(low).all() and torch.equal(got["logp"][masked].double(), low)
    else:
        close(got["logp"][masked], low, 4 * U * low.abs(), "masked logp")
    tol = 8 * U * (2 * 20 / temperature + math.log(vocab) + 1) + 1e-6  # |logits| below 20
    close(got["logp"][live], logp[live], tol + U * logp[live].abs(), "logp")
    close(got["loss"], loss, (4 * tol + ARITH) * mass + 1e-30, "loss")
    assert not got["dlogits"][masked].any()
    top = grad.abs().amax(1, keepdim=True)
    close(got["dlogits"][live], grad[live], (R[dtype] * grad.abs() + (4 * tol + 2 * ARITH) * 4 * top + 1e-38)[live], "dlogits")
    assert torch.equal(ops.token_logp(logits, actions, temperature=temperature), got["logp"])


@pytest.mark.parametrize("vocab", [5000, 300008])  # staged rows, and rows that are read twice
def test_policy_loss_kl_term_of_a_masked_action(vocab):
    """exp(d) - d - 1 for d = ref - logp without bounds (an action whose logit is -inf) is infinite, and not NaN."""
    logits, actions, old, ref, adv, w = _policy_inputs(5, vocab, torch.float32, 13)
    logits[2, actions[2]] = float("-inf")
    got = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, kl_coef=0.1)
    assert torch.isneginf(got["logp"][2]) and float(got["loss"]) == math.inf
    ref[2] = float("-inf")  # d the other way: exp(d) = 0, -d infinite
    logits[2, actions[2]] = 0.0
    assert float(ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, kl_coef=0.1)["loss"]) == math.inf
    w[2] = 0
    assert math.isfinite(float(ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=w, kl_coef=0.1)["loss"]))


def test_policy_loss_nan_stays_in_its_row_and_empty():
    logits, actions, old, ref, adv, w = _policy_inputs(8, 40000, torch.bfloat16, 12)
    clean = ops.policy_loss(logits, actions, old, adv)
    logits[3, 39999] = float("nan")
    got = ops.policy_loss(logits, actions, old, adv)
    keep = torch.arange(8, device="cuda") != 3
    assert torch.equal(got["dlogits"][keep], clean["dlogits"][keep]) and torch.isnan(got["dlogits"][3]).all()
    assert torch.isnan(got["loss"]) and torch.isnan(got["logp"][3])
    none = ops.policy_loss(logits[:0], actions[:0], old[:0], adv[:0])
    assert float(none["loss"]) == 0 and none["dlogits"].shape == (0, 40000)


def test_policy_loss_offsets_past_32_bits():
    n, vocab = 17, 140_000_000  # 2.4e9 elements
    logits = torch.zeros(n, vocab, dtype=torch.bfloat16, device="cuda")
    logits[:, 5] = 18.0
    logits[n - 1, vocab - 1] = 20.0
    actions = torch.full((n,), 5, device="cuda")
    actions[n - 1] = vocab - 1
    want = torch.tensor([18 - math.log(vocab - 1 + math.exp(18.0))] * (n - 1)
                        + [20 - math.log(vocab - 2 + math.exp(18.0) + math.exp(20.0))], device="cuda", dtype=torch.float64)
    got = ops.policy_loss(logits, actions, want.float(), torch.ones(n, device="cuda"), dlogits=logits)
    # sums of up to 1e5 terms a thread
    close(got["logp"], want, torch.full_like(want, 1e5 * U))
    p = want[-1].exp()
    assert abs(float(got["dlogits"][n - 1, vocab - 1]) * n + float(1 - p)) < 0.02


@pytest.mark.parametrize("n,vocab", [(4096, 4096), (64, 300000)])  # staged rows, and rows that are read twice
@pytest.mark.parametrize("temperature", [1.0, 0.9, 0.8, 1.3])
@pytest.mark.parametrize("reach", [10.0, 90.0])
def test_policy_loss_near_the_reference(n, vocab, temperature, reach):
    """KL term alone, |ref - logp| about 1e-3: the gradient follows logp's error 1000-fold, and logp in one float would have
    half steps of up to 2^-18 (64 u) at logp = -100.  Rows of zeros but for the action at -c: the exponentials are 1 (exactly)
    and e^(-c/T), so Z is off by half a step a level of its sum at most, and relative to Z by 4 u (the e^(-c/T) counts in
    a few partial sums that double from one to the next).  logp: those, log f (|log f| < 0.41: one step and its sum, 1 u), the low
    parts' own roundings (1 u); d = ref - logp: u |d|.  The slope -expm1(d) / T (1 - p): 8 u of itself."""
    g = gen(51)
    actions = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    c = reach * (0.5 + torch.rand(n, device="cuda", generator=g))
    logits = torch.zeros(n, vocab, device="cuda").scatter_(1, actions[:, None], -c[:, None])
    T = float(torch.tensor(temperature, dtype=torch.float32))
    z = -c.double() / T
    logp = z - torch.log(vocab - 1 + z.exp())
    ref = (logp + 1e-3 * torch.randn(n, device="cuda", generator=g)).float()
    zeros = torch.zeros(n, device="cuda")
    got = ops.policy_loss(logits, actions, logp.float(), zeros, ref_logp=ref, weights=torch.ones_like(zeros), kl_coef=1.0,
                          temperature=temperature)
    d = ref.double() - logp
    slope = -torch.expm1(d) / T * (1 - logp.exp())
    close(got["dlogits"].gather(1, actions[:, None])[:, 0], slope, 6 * U * d.exp() / T + 8 * U * slope.abs(), "dlogits")
    # the loss: expm1(d) - d, each rounded (2 u |d|), its slope by logp, and the rows' sum
    each = torch.expm1(d) - d
    close(got["loss"], each.sum(), (6 * U * torch.expm1(d).abs() + 4 * U * d.abs()).sum() + 12 * U * each.sum(), "loss")


def test_policy_gradient_by_differences():
    logits, actions, old, ref, adv, w = _policy_inputs(12, 50, torch.float32, 14)
    how = dict(ref_logp=ref, weights=w, clip=(5.0, 5.0), kl_coef=0.3, temperature=1.3)
    d = ops.policy_loss(logits, actions, old, adv, **how)["dlogits"]
    step, h = randn(gen(15), 12, 50), 1e-2
    f = lambda s: float(ops.policy_loss(logits + s * h * step, actions, old, adv, grad=False, **how)["loss"])  # noqa: E731
    # the loss is a sum of 12 terms of order one: third derivatives times h^2, and rounding over h
    assert abs((f(1) - f(-1)) / (2 * h) - float((d.double() * step.double()).sum())) < 12 * (4 * h * h + 4 * U / h)


# ---------------------------------------------------------------- AdamW


def _encode32(x, scale, turn):
    y = x / scale
    bits = (((y.view(torch.int32) + turn) >> 20) - 960).clamp(max=127)
    small = ((y * 512 * 1048576).int() + turn) >> 20
    return torch.where(y < 2.0 ** -6, small, bits)


def _scale32(x):
    top = torch.where(torch.isfinite(x), x, 0).amax(1, keepdim=True).view(torch.int32)
    return ((((top + 0x1FFFFF) >> 23) - 8).clamp(min=27) << 23).view(torch.float32)


def _adamw32(p, grad, m, v, scale, step, lr, betas, eps, decay, clip):
    """The update's fp32 operations one by one (the moments), and its formula in 64 bits (the parameter)."""
    n = p.numel()
    g = grad.float().view(-1) * clip
    m, v = m.view(-1).float(), v.view(-1).float()
    if scale is not None:
        per = scale.repeat_interleave(256, 0)[:n]
        m, v = m * per[:, 0], (v * per[:, 1]).square()
    m = m * betas[0] + g * (1 - betas[0])
    v = v * betas[1] + g * g * (1 - betas[1])
    p64 = p.double().view(-1) * (1 - lr * decay)
    move = lr / (1 - betas[0] ** step) * m.double() / (v.double().sqrt() / math.sqrt(1 - betas[1] ** step) + eps)
    if scale is None:
        return p64 - move, move, m, v, None
    root = torch.sqrt(v)
    blocks = lambda x: torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)  # noqa: E731
    i = torch.arange(n, device="cuda")
    turn = blocks((((i * 0x6A09E667 + step * 0x9E3779B1) & 0xFFFFFFFF) >> 12)).int()
    sm, sv = _scale32(blocks(m.abs())), _scale32(blocks(root))
    cm = _encode32(blocks(m.abs()), sm, 0xFFFFF - turn) + 128 * (blocks(m) < 0)
    cv = torch.where(blocks(root) == 0, 0, _encode32(blocks(root), sv, turn).clamp(min=1))
    code = lambda c: c.view(-1)[:n].to(torch.uint8)  # noqa: E731
    return p64 - move, move, code(cm), code(cv), torch.cat([sm, sv], 1)


def _tensors(shapes, dtype, grad_dtype, seed, offset=0):
    g = gen(seed)

    def make(shape, dt, size):
        n = math.prod(shape)
        buf = torch.zeros(n + offset, dtype=dt, device="cuda")
        buf[offset:] = (size * randn(g, n)).to(dt)
        return buf[offset:].view(shape)

    return [make(s, dtype, 0.1) for s in shapes], [make(s, grad_dtype, 0.02 * (1 + i % 3)) for i, s in enumerate(shapes)]


SHAPES = [(1,), (3, 5), (256,), (257,), (2048,), (2049,), (64, 100), (0,), (5000,), (255,)]


@pytest.mark.parametrize("dtype,grad_dtype,bits,master", [(torch.float32, torch.float32, 32, False), (torch.float32, torch.bfloat16, 32, False),
                                                          (torch.bfloat16, torch.bfloat16, 32, True), (torch.bfloat16, torch.float32, 32, False),
                                                          (torch.float32, torch.float32, 8, False), (torch.float32, torch.bfloat16, 8, False),
                                                          (torch.bfloat16, torch.bfloat16, 8, True), (torch.bfloat16, torch.bfloat16, 8, False),
                                                          (torch.bfloat16, torch.float32, 8, True), (torch.bfloat16, torch.float32, 8, False),
                                                          (torch.bfloat16, torch.bfloat16, 32, False), (torch.bfloat16, torch.float32, 32, True)])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_adamw(dtype, grad_dtype, bits, master, offset):
    params, grads = _tensors(SHAPES, dtype, grad_dtype, 21, offset)
    state = ops.adamw_state(params, bits=bits, master=master)
    if offset:  # moments off their 16-byte boundaries too
        for name in ("m", "v") + (("master",) if master else ()):
            ts = getattr(state, name)
            for k, t in enumerate(ts):
                raw = t.view(torch.uint8) if bits == 8 and name != "master" else t
                buf = torch.zeros(t.numel() + offset, dtype=raw.dtype, device="cuda")
                buf[offset:] = raw.view(-1)
                ts[k] = buf[offset:].view(t.dtype).view(t.shape) if bits == 8 and name != "master" else buf[offset:].view(t.shape)
    clip = torch.tensor(0.5, device="cuda")
    how = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    for step in (1, 2, 3):
        want = []
        for k, p in enumerate(params):
            if not p.numel():
                want.append(None)
                continue
            start = state.master[k] if master else p
            want.append(_adamw32(start.clone(), grads[k], state.m[k].clone(), state.v[k].clone(),
                                 state.scale[k].clone() if bits == 8 else None, step, 1e-2, (0.9, 0.99), 1e-8, 0.1, clip))
        ops.adamw_step(params, grads, state, step, grad_scale=clip, **how)
        for k, expected in enumerate(want):
            if expected is None:
                continue
            p, move, m, v, scale = expected
            tol = 4 * U * p.abs() + 16 * U * move.abs() + 1e-30
            if master:
                close(state.master[k].view(-1), p, tol, f"master {k}")
                assert torch.equal(params[k], state.master[k].bfloat16())
            else:
                close(params[k].view(-1), p, tol + R[dtype] * p.abs(), f"param {k}")
            raw = (lambda t: t.view(torch.uint8).view(-1)) if bits == 8 else (lambda t: t.view(-1))
            assert torch.equal(raw(state.m[k]), m) and torch.equal(raw(state.v[k]), v), f"moments {k}"
            if bits == 8:
                assert torch.equal(state.scale[k], scale)


def test_adamw_many_tensors():
    shapes = [(1 + 37 * i % 700,) for i in range(1100)]
    params, grads = _tensors(shapes, torch.float32, torch.float32, 22)
    state = ops.adamw_state(params)
    want = [_adamw32(p.clone(), g, m, v, None, 1, 1e-3, (0.9, 0.999), 1e-8, 0.01, 1.0)[0]
            for p, g, m, v in zip(params, grads, state.m, state.v)]
    ops.adamw_step(params, grads, state, 1, lr=1e-3)
    for p, w in zip(params, want):
        close(p, w, 4 * U * w.abs() + 1e-3 * 16 * U)


def test_adamw_8bit_moments_follow_slow_changes():
    """Zero gradients: v falls by a thousandth a step where its e4m3 neighbours are an eighth apart."""
    n, steps, beta2 = 4096, 600, 0.999
    p = [torch.zeros(n, device="cuda")]
    state = ops.adamw_state(p, bits=8)
    ops.adamw_step(p, [torch.rand(n, device="cuda", generator=gen(3)) + 0.5], state, 1, lr=0.0, betas=(0.9, beta2))
    value = lambda: (state.v[0].float().view(-1, 256) * state.scale[0][:, 1:]).double().mean().item()  # noqa: E731
    start, zero = value(), [torch.zeros(n, device="cuda")]
    for step in range(2, steps + 2):
        ops.adamw_step(p, zero, state, step, lr=0.0, betas=(0.9, beta2))
    # each element is within one neighbour (1 / 8) of its moment, their mean over 4096 thresholds far closer
    assert abs(value() / start - beta2 ** (steps / 2)) < 0.02
    assert state.m[0].float().abs().max() * state.scale[0][:, 0].max() < 1e-6


def test_adamw_8bit_non_finite_gradient_stays_in_its_element():
    params, grads = _tensors([(1000,)], torch.bfloat16, torch.bfloat16, 30)
    state = ops.adamw_state(params, bits=8, master=True)
    grads[0][300], grads[0][700] = float("nan"), float("inf")
    ops.adamw_step(params, grads, state, 1, lr=1e-3)
    bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
    bad[[300, 700]] = True
    assert torch.isfinite(state.scale[0]).all()
    assert torch.equal(torch.isnan(state.m[0].float()), bad) and torch.equal(torch.isnan(state.v[0].float()), bad)
    assert torch.equal(torch.isnan(state.master[0]), bad)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_smallest_eps(bits):
    """No gradient so far and the smallest eps: 0 / eps is 0, and the parameters decay alone."""
    params, _ = _tensors([(1000,)], torch.float32, torch.float32, 31)
    start, state = params[0].double(), ops.adamw_state(params, bits=bits)
    ops.adamw_step(params, [torch.zeros(1000, device="cuda")], state, 1, lr=1e-2, eps=2.0 ** -126, weight_decay=0.1)
    close(params[0], start * (1 - 1e-3), 2 * U * start.abs())
    with pytest.raises(ccq.CCQError, match="eps"):
        ops.adamw_step(params, [torch.zeros(1000, device="cuda")], state, 2, lr=1e-2, eps=1e-39)


def test_adamw_tensor_past_32_bits():
    n = 2 ** 31 + 4097
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    grad[[0, 2 ** 31 - 1, 2 ** 31, n - 1]] = 1.0
    state = ops.adamw_state([p], bits=8)
    ops.adamw_step([p], [grad], state, 1, lr=0.5, weight_decay=0.0)
    assert torch.equal(torch.nonzero(p)[:, 0], torch.tensor([0, 2 ** 31 - 1, 2 ** 31, n - 1], device="cuda"))
    assert torch.equal(p[[0, n - 1]].float(), torch.tensor([-0.5, -0.5], device="cuda"))
    assert int((state.m[0].view(torch.uint8) != 0).sum()) == 4


# ---------------------------------------------------------------- streams


def test_operators_run_on_the_current_stream():
    g = gen(40)
    table, ids = randn(g, 500, 256, dtype=torch.bfloat16), torch.randint(0, 500, (300,), device="cuda", generator=g)
    w = torch.ones(256, device="cuda")
    logits, actions, old, ref, adv, weights = _policy_inputs(300, 700, torch.bfloat16, 41)

    def all_of():
        e = ops.embed(table, ids)
        y = ops.group_norm(e, w, None, e, groups=2)
        d = ops.group_norm_bwd(e, w, None, e, y, groups=2)
        t = ops.embed_grad(d["dx"], ids, 500)
        p, state = [table.clone()], ops.adamw_state([table], bits=8)
        ops.adamw_step(p, [t], state, 1, lr=1e-2)
        loss = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights)
        return [y, d["dx"], d["dweight"], t, p[0], loss["loss"], loss["dlogits"]]

    want = all_of()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # a call on another stream would be done long before
        got = all_of()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # and in a graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_of()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, held):
        assert torch.equal(a, b)


def test_stream_argument(monkeypatch):
    """A call with stream= behind a long wait on that stream: its workspace is not given to the current stream's next
    tensors, and results are those of the current stream."""
    g = gen(42)
    n = 3000
    ids = torch.randint(0, 500, (n,), device="cuda", generator=g)
    x, gate, dy = (randn(g, n, 256, dtype=torch.bfloat16) for _ in range(3))
    w, b = 1 + 0.1 * randn(g, 256), 0.1 * randn(g, 256)
    table = randn(g, 500, 256)
    logits, actions, old, ref, adv, weights = _policy_inputs(n, 700, torch.bfloat16, 43)

    def all_of(**how):
        d = ops.group_norm_bwd(x, w, b, gate, dy, groups=2, **how)
        p = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, kl_coef=0.1, **how)
        return [ops.embed(table, ids, **how), ops.group_norm(x, w, b, gate, groups=2, **how), ops.token_logp(logits, actions, **how),
                ops.embed_grad(dy, ids, 500, **how)] + [d[k] for k in sorted(d)] + [p[k] for k in sorted(p)]

    want = all_of()
    side, spaces, keep = torch.cuda.Stream(), [], ops._workspace

    def workspace(*args):
        made = keep(*args)
        if made[0] is not None:
            spaces.append((made[0].data_ptr(), made[1]))
        return made

    monkeypatch.setattr(ops, "_workspace", workspace)
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    got = all_of(stream=side)
    assert len(spaces) == 3
    # tensors of those sizes on the current stream, written while the other has yet to begin
    fills = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _, size in spaces for _ in range(8)]
    assert not side.query()
    for at, size in spaces:
        assert all(f.data_ptr() + f.numel() <= at or at + size <= f.data_ptr() for f in fills)
    torch.cuda.current_stream().wait_stream(side)
    for a, c in zip(want, got):
        assert torch.equal(a, c)


@pytest.mark.parametrize("backbone", [ccq.GLA, ccq.GDN])
def test_stream_argument_of_the_mixer(backbone):
    """As above, for the mixer's forward (split sequences, which need a workspace) and the decode step."""
    P = inputs.make_inputs(backbone, 1, 4096, 2, 128, 128, dtype=torch.bfloat16, seed=5)
    D = {n: (None if x is None else x.cuda()) for n, x in P.items()}
    token = {n: (None if x is None else x[:, -1].clone()) for n, x in D.items()}
    gates = (D["gate"],) if backbone == ccq.GLA else (D["gate"], D["beta"])
    fwd = ccq.gla_fwd if backbone == ccq.GLA else ccq.gdn_fwd
    made = (ccq.gla_workspace if backbone == ccq.GLA else ccq.gdn_workspace)(1, 4096, 2, 128, 128, "cuda")
    assert made is not None
    size = made.numel()
    del made

    def both(**how):
        o, state = fwd(D["q"], D["k"], D["v"], *gates, D["lam"], **how)
        y = ccq.decode_step(backbone, token["q"], token["k"], token["v"], token["gate"], token["lam"], state, token["beta"], **how)
        return [o, y, state.S, state.C, state.m, state.t]

    want, side = both(), torch.cuda.Stream()
    torch.cuda.synchronize()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    got = both(stream=side)
    fills = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert not side.query()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert all(bool((f == 255).all()) for f in fills)


def test_tensors_of_a_device_that_is_not_current_are_refused(monkeypatch):
    """(The other device is the host's fiction: nothing is launched, and no workspace's size is asked for.)"""
    x, ids = torch.ones(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    monkeypatch.setattr(ccq, "_current_device", lambda: 1)
    sizes = ops._size.cache_info().currsize
    for call in (lambda: ops.embed(x, ids), lambda: ops.group_norm(x, groups=1), lambda: ops.token_logp(x, ids),
                 lambda: ops.group_norm_bwd(x, x[0], None, None, x, groups=1), lambda: ops.embed_grad(x, ids, 5),
                 lambda: ops.policy_loss(x, ids, x[:, 0].contiguous(), x[:, 0].contiguous()),
                 lambda: ops.adamw_step([x], [x], ops.adamw_state([x]), 1, lr=1e-3), lambda: ccq.device_status(device=x.device)):
        with pytest.raises(ValueError, match="current device is cuda:1"):
            call()
    # (those of the embedding's gradient and of the policy loss are the same on every device)
    assert ops._size.cache_info().currsize <= sizes + 2
    monkeypatch.undo()
    assert torch.equal(ops.embed(x, ids), x[ids])


def test_two_threads_at_once():
    """Each thread has its own plan, argument block and stream; what they share is the library's memory of the device."""
    g = gen(44)
    jobs = []
    for vocab, tokens in ((700, 2000), (4096, 900)):
        x = _policy_inputs(tokens, vocab, torch.bfloat16, vocab)
        params, grads = _tensors([(300,), (64, 100), (5000,)], torch.float32, torch.float32, vocab)
        ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=g)
        rows, w = randn(g, tokens, 256), 1 + 0.1 * randn(g, 256)

        def job(x=x, params=params, grads=grads, ids=ids, rows=rows, w=w, vocab=vocab):
            logits, actions, old, ref, adv, weights = x
            p = [t.clone() for t in params]
            ops.adamw_step(p, grads, ops.adamw_state(p, bits=8), 1, lr=1e-2)
            loss = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, kl_coef=0.1)
            d = ops.group_norm_bwd(rows, w, None, None, rows, groups=2)
            return p + [loss["loss"], loss["dlogits"], d["dx"], d["dweight"], ops.embed_grad(rows, ids, vocab), ops.embed(rows, ids % 100)]

        jobs.append(job)
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(2)

    def run(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait()
                for _ in range(20):
                    got = jobs[k]()
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(want[k], got)):
                        wrong.append(k)
        except Exception as e:  # (an error in a thread is not the test's by itself)
            wrong.append(e)

    threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_graph_replayed_on_other_inputs():
    """A captured step computes from what its inputs hold at the replay: ids, masks and values."""
    g = gen(45)
    n = 700
    ids = torch.randint(0, 90, (n,), device="cuda", generator=g)
    rows, gate, w = randn(g, n, 256), randn(g, n, 256), 1 + 0.1 * randn(g, 256)
    x = list(_policy_inputs(n, 801, torch.bfloat16, 46, masked=200))

    def step():
        logits, actions, old, ref, adv, weights = x
        d = ops.group_norm_bwd(rows, w, None, gate, rows, groups=2)
        loss = ops.policy_loss(logits, actions, old, adv, ref_logp=ref, weights=weights, kl_coef=0.1)
        few = ops.embed_grad(rows[:100], ids[:100], 90, padding_id=3)
        return [ops.embed(rows, ids), ops.group_norm(rows, w, None, gate, groups=2), d["dx"], d["dgate"], d["dweight"], loss["loss"],
                loss["logp"], loss["dlogits"], ops.embed_grad(rows, ids, 90, padding_id=3), few, ops.token_logp(logits, actions)]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (47, 48):
        h = gen(seed)
        ids.copy_(_ids("zipf", n, 90, h))
        rows.copy_(randn(h, n, 256))
        gate.copy_(randn(h, n, 256))
        for old, new in zip(x, _policy_inputs(n, 801, torch.bfloat16, seed, masked=40 * (seed - 46))):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)
