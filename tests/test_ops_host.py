"""Host-side checks of the operators around the token mixer (ccq_ops.h): every bad argument is refused with a
status before any CUDA call, sizes are answered without a GPU, and the binding refuses CPU tensors."""
import ctypes
import inspect

import pytest
import torch

from paper_2606_01294_gb300 import _build, ccq, ops

FAKE = 0x10000  # aligned, never dereferenced on these paths
INVALID, UNSUPPORTED = ccq.CCQ_ERR_INVALID_ARG, ccq.CCQ_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return ops._library()


def test_header_declares_and_library_exports(lib):
    names = set(ccq.header_symbols())
    for n in ("ccq_embed", "ccq_embed_grad", "ccq_group_norm", "ccq_group_norm_bwd", "ccq_policy_loss", "ccq_token_logp",
              "ccq_adamw_step", "ccq_default_policy_params"):
        assert n in names and hasattr(lib, n)
    assert lib.ccq_status_string(6) != lib.ccq_status_string(99)


def _call(fn, good, **changes):
    args = dict(good)
    for k, v in changes.items():
        assert k in args
        args[k] = v
    return fn(*args.values())


def _refused(lib, fn, good, status, text, **changes):
    assert _call(fn, good, **changes) == status, changes
    assert text in lib.ccq_last_error(), (changes, lib.ccq_last_error())


def test_embed_refusals(lib):
    good = dict(table=FAKE, dtype=0, ts=64, ids=FAKE, id_bytes=8, n=5, rows=10, width=64, scale=1.0, out=FAKE, os=64, stream=None)
    for text, ch in ((b"NULL", dict(table=None)), (b"NULL", dict(ids=None)), (b"NULL", dict(out=None)), (b"aligned", dict(table=FAKE + 1)),
                     (b"aligned", dict(ids=FAKE + 4)), (b"sizes", dict(n=-1)), (b"sizes", dict(rows=0)), (b"sizes", dict(width=0)),
                     (b"dtype", dict(dtype=3)), (b"id_bytes", dict(id_bytes=2)), (b"stride", dict(ts=63)), (b"stride", dict(os=10))):
        _refused(lib, lib.ccq_embed, good, INVALID, text, **ch)
    assert _call(lib.ccq_embed, good, n=0) == 0


def test_embed_grad_refusals(lib):
    good = dict(dout=FAKE, dtype=0, ds=64, ids=FAKE, id_bytes=8, n=500, rows=10, width=64, scale=1.0, padding=-1, dtable=FAKE, od=1, os=64,
                ws=FAKE, nbytes=1 << 30, stream=None)
    for text, ch in ((b"NULL", dict(dout=None)), (b"NULL", dict(dtable=None)), (b"NULL", dict(ws=None)), (b"aligned", dict(ws=FAKE + 8)),
                     (b"workspace", dict(nbytes=16)), (b"padding", dict(padding=10)), (b"stride", dict(ds=60)), (b"stride", dict(os=60)),
                     (b"dtype", dict(od=2)), (b"dtype", dict(dtype=-1)), (b"sizes", dict(n=-2))):
        _refused(lib, lib.ccq_embed_grad, good, INVALID, text, **ch)
    _refused(lib, lib.ccq_embed_grad, good, UNSUPPORTED, b"2^30", n=(1 << 30) + 1)
    n = ctypes.c_size_t()
    assert lib.ccq_embed_grad_workspace_size(1000, 500, 64, ctypes.byref(n)) == 0 and n.value >= 16 * 1000
    assert lib.ccq_embed_grad_workspace_size(1000, 500, 64, None) == INVALID
    assert lib.ccq_embed_grad_workspace_size(256, 500, 64, ctypes.byref(n)) == 0 and n.value == 0  # few ids need none
    assert lib.ccq_embed_grad_workspace_size(257, 500, 64, ctypes.byref(n)) == 0 and n.value >= 16 * 257


def test_group_norm_refusals(lib):
    good = dict(x=FAKE, xs=64, gate=FAKE, gs=64, w=FAKE, b=FAKE, dtype=0, pd=1, y=FAKE, ys=64, tokens=4, channels=64, groups=2, centered=1,
                eps=1e-5, act=1, stream=None)
    for text, ch in ((b"NULL", dict(x=None)), (b"NULL", dict(y=None)), (b"stride", dict(xs=63)), (b"stride", dict(gs=63)), (b"stride", dict(ys=0)),
                     (b"sizes", dict(groups=3)), (b"sizes", dict(groups=0)), (b"sizes", dict(tokens=-1)), (b"sizes", dict(channels=0)),
                     (b"dtype", dict(dtype=2)), (b"dtype", dict(pd=2)), (b"activation", dict(act=3)), (b"eps", dict(eps=-1.0)),
                     (b"eps", dict(eps=float("nan"))), (b"aligned", dict(w=FAKE + 2)), (b"aligned", dict(x=FAKE + 1))):
        _refused(lib, lib.ccq_group_norm, good, INVALID, text, **ch)
    assert _call(lib.ccq_group_norm, good, tokens=0) == 0
    bwd = dict(x=FAKE, xs=64, gate=FAKE, gs=64, w=FAKE, b=FAKE, dy=FAKE, ds=64, dtype=0, pd=1, dx=FAKE, dxs=64, dgate=FAKE, dgs=64, dw=FAKE,
               db=FAKE, tokens=4, channels=64, groups=2, centered=1, eps=1e-5, act=1, ws=FAKE, nbytes=1 << 28, stream=None)
    for text, ch in ((b"NULL", dict(dy=None)), (b"NULL", dict(dx=None)), (b"dgate", dict(dgate=None)), (b"dgate", dict(gate=None)),
                     (b"workspace", dict(ws=None)), (b"workspace", dict(nbytes=8)), (b"stride", dict(dgs=10)), (b"aligned", dict(dw=FAKE + 2))):
        _refused(lib, lib.ccq_group_norm_bwd, bwd, INVALID, text, **ch)


def test_policy_refusals(lib):
    p = ops._PolicyParams()
    lib.ccq_default_policy_params(ctypes.byref(p))
    assert (round(p.clip_low, 3), round(p.clip_high, 3), p.kl_coef, p.temperature, p.grad_scale) == (0.2, 0.2, 0, 1, 1)
    good = dict(x=FAKE, dtype=0, xs=100, act=FAKE, ab=8, old=FAKE, ref=FAKE, adv=FAKE, w=FAKE, n=3, vocab=100, p=ctypes.byref(p), loss=FAKE,
                logp=FAKE, dx=FAKE, dxs=100, ws=FAKE, nbytes=1 << 20, stream=None)
    for text, ch in ((b"NULL", dict(x=None)), (b"NULL", dict(act=None)), (b"NULL", dict(old=None)), (b"NULL", dict(adv=None)), (b"NULL", dict(loss=None)),
                     (b"workspace", dict(ws=None)), (b"workspace", dict(nbytes=4)), (b"stride", dict(xs=99)), (b"stride", dict(dxs=99)),
                     (b"row stride", dict(dxs=200)), (b"sizes", dict(n=-1)), (b"sizes", dict(vocab=0)), (b"dtype", dict(dtype=5)),
                     (b"id_bytes", dict(ab=1)), (b"aligned", dict(ref=FAKE + 2))):
        _refused(lib, lib.ccq_policy_loss, good, INVALID, text, **ch)
    for field, value, text in (("temperature", 0.0, b"temperature"), ("temperature", float("nan"), b"temperature"), ("temperature", float("inf"), b"temperature"),
                               ("clip_low", -0.1, b"clip"), ("clip_high", float("nan"), b"clip")):
        q = ops._PolicyParams(0.2, 0.2, 0.0, 1.0, 1.0)
        setattr(q, field, value)
        _refused(lib, lib.ccq_policy_loss, good, INVALID, text, p=ctypes.byref(q))
    assert lib.ccq_token_logp(FAKE, 0, 100, FAKE, 8, 3, 100, 0.0, FAKE, None) == INVALID
    assert lib.ccq_token_logp(FAKE, 0, 100, FAKE, 8, 0, 100, 1.0, FAKE, None) == 0


def _adamw(lib, rows, **kw):
    flat = [x or 0 for r in rows for x in r]
    table = (ctypes.c_int64 * max(1, len(flat)))(*flat)
    a = dict(count=len(rows), pd=1, gd=1, bits=32, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, step=1, clip=None)
    a.update(kw)
    p = ops._AdamWParams(a["lr"], a["b1"], a["b2"], a["eps"], a["wd"], a["step"])
    return lib.ccq_adamw_step(ctypes.addressof(table), a["count"], a["pd"], a["gd"], a["bits"], ctypes.byref(p), a["clip"], None)


def test_adamw_refusals(lib):
    row = [FAKE, FAKE, FAKE, FAKE, None, None, 10]
    change = lambda i, v: [row[:i] + [v] + row[i + 1:]]  # noqa: E731
    for text, rows, kw in ((b"param", change(0, None), {}), (b"grad", change(1, None), {}), (b"m is", change(2, None), {}), (b"v is", change(3, None), {}),
                           (b"not used", change(4, FAKE), {}), (b"master", change(5, FAKE), {}), (b"n=", change(6, -1), {}),
                           (b"scale is NULL", [row], dict(bits=8)), (b"state_bits", [row], dict(bits=16)), (b"step", [row], dict(step=0)),
                           (b"betas", [row], dict(b1=1.0)), (b"betas", [row], dict(b2=-0.1)), (b"eps", [row], dict(eps=-1.0)), (b"dtype", [row], dict(pd=4)),
                           (b"aligned", change(0, FAKE + 2), {}), (b"count", [row], dict(count=-1)), (b"grad_scale", [row], dict(clip=FAKE + 1)),
                           (b"master is NULL", [row[:5] + [FAKE, 10], row], dict(pd=0))):
        assert _adamw(lib, rows, **kw) == INVALID, (text, kw)
        assert text in lib.ccq_last_error(), (text, lib.ccq_last_error())
    assert _adamw(lib, []) == 0
    assert _adamw(lib, [[None] * 6 + [0]]) == 0


def test_binding_refuses_cpu_tensors_and_bad_shapes():
    x, ids = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.embed(x, ids), lambda: ops.embed_grad(x, ids, 4), lambda: ops.group_norm(x, groups=1),
                 lambda: ops.group_norm_bwd(x, None, None, None, x, groups=1), lambda: ops.token_logp(x, ids),
                 lambda: ops.policy_loss(x, ids, x[:, 0], x[:, 0]),
                 lambda: ops.adamw_step([x], [x], ops.adamw_state([x]), 1, lr=1e-3)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="bits"):
        ops.adamw_state([x], bits=4)


@pytest.mark.parametrize("bad", ["columns", "overlap", "two strides"])
def test_rows_refuses_what_one_stride_does_not_reach(bad, monkeypatch):
    monkeypatch.setattr(ops, "_cuda", lambda t, name, device=None: t)
    t = {"columns": torch.zeros(8, 6)[:, ::2], "overlap": torch.zeros(64).as_strided((4, 6), (3, 1)),
         "two strides": torch.zeros(4, 9, 6)[:, :3]}[bad]
    with pytest.raises(ValueError):
        ops._rows(t, "t")


def test_rows_strides(monkeypatch):
    monkeypatch.setattr(ops, "_cuda", lambda t, name, device=None: t)
    assert ops._rows(torch.zeros(3, 4, 5), "t") == 5
    assert ops._rows(torch.zeros(3, 4, 9)[..., 2:7], "t") == 9
    assert ops._rows(torch.zeros(3, 9)[1:2, :4], "t") == 4
    assert ops._rows(torch.zeros(6, 4, 9)[::2, 1:2, :5], "t") == 72


STREAMED = [ops.embed, ops.embed_grad, ops.group_norm, ops.group_norm_bwd, ops.policy_loss, ops.token_logp, ccq.gla_fwd, ccq.gla_fwd_save,
            ccq.gla_bwd, ccq.gdn_fwd, ccq.gdn_bwd, ccq.gdn_fwd_decayed, ccq.fwd_varlen, ccq.decode_step]


@pytest.mark.parametrize("call", STREAMED, ids=lambda f: f.__name__)
def test_a_given_stream_is_entered_for_the_whole_call(call, monkeypatch):
    """What a call allocates has to belong to the stream it runs on: with ``stream`` the whole call is made within it, with
    every other argument as it came."""
    seen = []
    for module in (ops, ccq):
        monkeypatch.setattr(module, "_on_stream", lambda stream, fn, *args, **kw: seen.append((stream, fn, args, kw)) or "result")
    given = {name: object() for name, p in inspect.signature(call).parameters.items() if p.kind != p.VAR_KEYWORD}
    more = {"l2norm": object(), "seq_split": object()} if len(given) < len(inspect.signature(call).parameters) else {}
    assert call(**given, **more) == "result"
    (stream, fn, args, kw), = seen
    assert stream is given.pop("stream") and fn is call
    bound = dict(inspect.signature(call).bind(*args, **kw).arguments)
    assert bound.pop("kw", {}) == more
    assert bound.keys() == given.keys() and all(bound[name] is given[name] for name in given)


def test_on_stream_enters_and_records(monkeypatch):
    """The call runs inside the stream's context and every tensor that it returns is recorded on the caller's."""
    inside, recorded = [], []

    class Context:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            inside.append(self.stream)

        def __exit__(self, *error):
            inside.pop()

    class Stream:
        device = "cuda:0"

    stream = Stream()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: ("caller", device))
    monkeypatch.setattr(torch.cuda, "stream", Context)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.append((t.numel(), s)))
    made = [torch.zeros(k) for k in range(1, 8)]
    state = ccq.CCQState(*made[3:])

    def call(a, b=None):
        assert inside == [stream] and (a, b) == (1, 2)
        return made[0], None, {"x": made[1], "y": [made[2], state]}

    result = ccq._on_stream(stream, call, 1, b=2)
    assert not inside and result[2]["y"][1] is state
    assert sorted(recorded) == [(k, ("caller", "cuda:0")) for k in range(1, 8)]


def test_tensors_of_a_device_that_is_not_current_are_refused(monkeypatch):
    monkeypatch.setattr(ccq, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(ccq, "_raw_stream", lambda index: 100 + index)
    assert ccq._stream(torch.device("cuda:0"), None) == 100
    with pytest.raises(ValueError, match="cuda:1.*current device is cuda:0"):
        ccq._stream(torch.device("cuda:1"), None)


def test_a_status_word_that_cannot_be_resolved_is_an_error(lib):
    """Kernels write to the status word, so no call passes on one that is missing, as it is without a device.  (With a device
    the same calls, on its memory, pass.)"""
    gpu = torch.cuda.is_available()
    held = [torch.zeros(1 << 16, dtype=torch.uint8, device="cuda") for _ in range(8)] if gpu else []
    at = [t.data_ptr() for t in held] or [FAKE] * 8
    p = ops._PolicyParams(0.2, 0.2, 0.0, 1.0, 1.0)
    for got in (lib.ccq_embed(at[0], 1, 8, at[1], 8, 4, 10, 8, 1.0, at[2], 8, None),
                lib.ccq_embed_grad(at[0], 1, 8, at[1], 8, 4, 10, 8, 1.0, -1, at[2], 1, 8, None, 0, None),
                lib.ccq_embed_grad(at[0], 1, 8, at[1], 8, 300, 10, 8, 1.0, -1, at[2], 1, 8, at[3], 1 << 16, None),
                lib.ccq_policy_loss(at[0], 1, 100, at[1], 8, at[2], None, at[3], None, 3, 100, ctypes.byref(p), at[4], None, at[5], 100, at[6],
                                    1 << 16, None),
                lib.ccq_token_logp(at[0], 1, 100, at[1], 8, 3, 100, 1.0, at[2], None)):
        assert got == (ccq.CCQ_OK if gpu else ccq.CCQ_ERR_CUDA)
        assert gpu or b"status word" in lib.ccq_last_error()
    if gpu:
        torch.cuda.synchronize()


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 4.2e-39])
def test_a_temperature_without_a_finite_reciprocal_is_refused(lib, temperature):
    """n = 0: a call that passes its checks launches nothing.  log2(e) / 4.3e-39 = 3.36e38 is a number in fp32, / 4.2e-39 is not."""
    n0 = (FAKE, 0, 100, FAKE, 8)
    score = lambda t: lib.ccq_token_logp(*n0, 0, 100, t, FAKE, None)  # noqa: E731
    assert score(temperature) == INVALID and b"temperature" in lib.ccq_last_error()
    assert score(4.3e-39) == 0 and score(1e30) == 0 and score(2e30) == INVALID


def test_an_eps_below_the_normal_numbers_is_refused(lib):
    for eps in (1e-60, 1e-45, 1e-39, 1.17e-38):
        assert _adamw(lib, [], eps=eps) == INVALID and b"eps" in lib.ccq_last_error(), eps
    for eps in (0.0, 1.18e-38, 1e-8):
        assert _adamw(lib, [], eps=eps) == 0, eps


@pytest.mark.parametrize("name", ["dgate", "dweight", "dbias"])
def test_group_norm_gradients_that_nothing_belongs_to_are_refused(name, monkeypatch):
    """A tensor under the name of an operand that is not there has no type or size that it could be checked for."""
    monkeypatch.setattr(ops, "_cuda", lambda t, name, device=None: t)
    x = torch.zeros(4, 64)
    operands = dict(zip(("dweight", "dbias", "dgate"), (x[0], x[0], x)))
    operands[name] = None
    with pytest.raises(ValueError, match=f"out has {name}, but there is no {name[1:]}"):
        ops.group_norm_bwd(x, operands["dweight"], operands["dbias"], operands["dgate"], x, groups=1, out={name: torch.zeros(1)})
