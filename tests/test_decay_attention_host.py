"""Host-side checks of the rotation by positions and of linear attention with a decay for each head (ccq_ops.h): every bad
argument is refused with a status before any CUDA call, sizes are answered without a GPU, and the binding refuses what
the library cannot take."""
import ctypes
import math
import struct

import pytest
import torch

from paper_2606_01294_gb300 import _build, ccq, ops

FAKE = 0x10000  # aligned, never dereferenced on these paths
INVALID, UNSUPPORTED = ccq.CCQ_ERR_INVALID_ARG, ccq.CCQ_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return ops._library()


def heads(p=FAKE, batch=1 << 14, token=512, head=128, n=4):
    return struct.pack("5q", p, batch, token, head, n)


def refused(lib, fn, good, status, text, **changes):
    args = dict(good)
    for k, v in changes.items():
        assert k in args
        args[k] = v
    assert fn(*args.values()) == status, changes
    assert text in lib.ccq_last_error(), (changes, lib.ccq_last_error())


def test_the_library_exports_them(lib):
    names = set(ccq.header_symbols())
    for n in ("ccq_rotary", "ccq_decay_attention", "ccq_decay_attention_bwd", "ccq_decay_attention_step",
              "ccq_decay_attention_workspace_size", "ccq_decay_attention_bwd_workspace_size"):
        assert n in names and hasattr(lib, n)


def test_rotary_refusals(lib):
    good = dict(x=heads() + heads(), y=heads() + heads(), count=2, dtype=0, B=2, T=32, width=128, part=64, positions=FAKE,
                pb=8, freqs=FAKE, amplitude=1.0, inter=0, inverse=0, stream=None)
    for text, ch in ((b"count", dict(count=0)), (b"count", dict(count=3)), (b"NULL", dict(x=None)), (b"dtype", dict(dtype=5)),
                     (b"sizes", dict(B=-1)), (b"sizes", dict(T=-1)), (b"even part", dict(part=63)), (b"even part", dict(part=130)),
                     (b"even part", dict(part=0)), (b"even part", dict(width=1)), (b"position_bytes", dict(pb=2)),
                     (b"NULL", dict(positions=None)), (b"aligned", dict(positions=FAKE + 4)), (b"NULL", dict(freqs=None)),
                     (b"aligned", dict(freqs=FAKE + 4)), (b"amplitude", dict(amplitude=math.inf)),
                     (b"amplitude", dict(amplitude=math.nan)), (b"x[1] is NULL", dict(x=heads() + heads(0))),
                     (b"aligned", dict(x=heads(FAKE + 1) + heads())), (b"heads", dict(x=heads(n=0) + heads())),
                     (b"differ in heads", dict(y=heads() + heads(n=2))), (b"stride", dict(x=heads(token=-4) + heads())),
                     (b"stride", dict(x=heads() + heads(batch=1 << 41))), (b"overlap", dict(y=heads(head=64) + heads())),
                     (b"overlap", dict(y=heads(token=0) + heads())), (b"overlap", dict(y=heads(batch=512) + heads()))):
        refused(lib, lib.ccq_rotary, good, INVALID, text, **ch)
    refused(lib, lib.ccq_rotary, good, UNSUPPORTED, b"2^31", B=1 << 20, T=1 << 20)
    refused(lib, lib.ccq_rotary, good, UNSUPPORTED, b"4096", width=8192, part=8192,
            y=heads(head=1 << 13, token=1 << 15, batch=1 << 21) * 2)
    assert lib.ccq_rotary(*dict(good, T=0).values()) == 0


def attention():
    return dict(q=heads(), k=heads(), v=heads(n=2), dtype=0, ld=FAKE, scale=0.1, S0=None, o=heads(FAKE * 2), ST=None, B=2, T=32, H=4, d=128,
                cu=None, cb=8, n=2, ws=None, nbytes=0, stream=None)


def test_attention_refusals(lib):
    good = attention()
    for text, ch in ((b"NULL", dict(q=None)), (b"NULL", dict(o=None)), (b"dtype", dict(dtype=7)), (b"log_decay is NULL", dict(ld=None)),
                     (b"aligned", dict(ld=FAKE + 2)), (b"scale", dict(scale=math.nan)), (b"sizes", dict(B=-1)), (b"sizes", dict(H=0)),
                     (b"no divisor", dict(k=heads(n=3))), (b"no divisor", dict(v=heads(n=8))), (b"o has", dict(o=heads(FAKE * 2, n=2))),
                     (b"overlap", dict(o=heads(FAKE * 2, head=100))), (b"k is NULL", dict(k=heads(0))), (b"aligned", dict(v=heads(FAKE + 1))),
                     (b"aligned", dict(S0=FAKE + 4)), (b"aligned", dict(ST=FAKE + 8)), (b"num_seqs", dict(n=3)), (b"B = 1", dict(cu=FAKE)),
                     (b"cu_bytes", dict(cu=FAKE, B=1, cb=3)), (b"aligned", dict(cu=FAKE + 4, B=1)), (b"stride", dict(q=heads(head=-1))),
                     (b"o is k", dict(o=heads(FAKE * 3), k=heads(FAKE * 3)))):
        refused(lib, lib.ccq_decay_attention, good, INVALID, text, **ch)
    refused(lib, lib.ccq_decay_attention, good, UNSUPPORTED, b"64 or 128", d=96)
    refused(lib, lib.ccq_decay_attention, good, UNSUPPORTED, b"2^24", cu=FAKE, B=1, n=1 << 23)
    long = dict(B=1, n=1, T=1 << 16, H=2, q=heads(n=2), k=heads(n=2), v=heads(n=2), o=heads(FAKE * 2, n=2))
    refused(lib, lib.ccq_decay_attention, good, INVALID, b"workspace", **long)
    refused(lib, lib.ccq_decay_attention, good, INVALID, b"workspace", **long, ws=FAKE, nbytes=64)
    refused(lib, lib.ccq_decay_attention, good, INVALID, b"aligned", **long, ws=FAKE + 8, nbytes=1 << 40)
    assert lib.ccq_decay_attention(*dict(good, B=0, n=0).values()) == 0


def test_attention_gradient_refusals(lib):
    a = attention()
    good = dict(q=a["q"], k=a["k"], v=a["v"], dtype=0, ld=FAKE, scale=0.1, S0=None, do=heads(), dST=FAKE * 4, dq=heads(FAKE * 2), dk=heads(FAKE * 2),
                dv=heads(FAKE * 2, n=2), dS0=FAKE, B=2, T=32, H=4, d=128, cu=None, cb=8, n=2, ws=FAKE, nbytes=1 << 30, stream=None)
    for text, ch in ((b"NULL", dict(do=None)), (b"NULL", dict(dv=None)), (b"dout has", dict(do=heads(n=2))), (b"dk has 2", dict(dk=heads(FAKE * 2, n=2))),
                     (b"overlap", dict(dq=heads(FAKE * 2, token=100))), (b"dS0 is dST", dict(dST=FAKE)), (b"aligned", dict(dST=FAKE + 4)),
                     (b"dq is dout", dict(dq=heads(FAKE * 3), do=heads(FAKE * 3))), (b"workspace", dict(ws=None)), (b"workspace", dict(nbytes=100)), (b"dtype", dict(dtype=2))):
        refused(lib, lib.ccq_decay_attention_bwd, good, INVALID, text, **ch)
    refused(lib, lib.ccq_decay_attention_bwd, good, UNSUPPORTED, b"64 or 128", d=256)


def test_step_refusals(lib):
    good = dict(q=heads(), k=heads(), v=heads(n=1), dtype=1, ld=FAKE, scale=0.1, state=FAKE, rows=9, slots=FAKE, sb=8, o=heads(), B=5, H=4, d=64,
                stream=None)
    for text, ch in ((b"NULL", dict(v=None)), (b"NULL", dict(state=None)), (b"aligned", dict(state=FAKE + 8)), (b"slot_bytes", dict(sb=1)),
                     (b"aligned", dict(slots=FAKE + 4)), (b"states for a batch", dict(slots=None, rows=4)), (b"no divisor", dict(k=heads(n=3))),
                     (b"o has", dict(o=heads(n=2))), (b"overlap", dict(o=heads(batch=0))), (b"sizes", dict(rows=-1)), (b"scale", dict(scale=math.inf)),
                     (b"log_decay", dict(ld=None)), (b"dtype", dict(dtype=-1))):
        refused(lib, lib.ccq_decay_attention_step, good, INVALID, text, **ch)
    refused(lib, lib.ccq_decay_attention_step, good, UNSUPPORTED, b"64 or 128", d=32)
    refused(lib, lib.ccq_decay_attention_step, good, UNSUPPORTED, b"2^24", B=1 << 23, rows=1 << 23)
    assert lib.ccq_decay_attention_step(*dict(good, B=0).values()) == 0


def test_workspace_sizes(lib):
    n = ctypes.c_size_t(1)
    size = lambda *a: (lib.ccq_decay_attention_workspace_size(*a, ctypes.byref(n)), n.value)[0]  # noqa: E731
    back = lambda *a: (lib.ccq_decay_attention_bwd_workspace_size(*a, ctypes.byref(n)), n.value)[0]  # noqa: E731
    for dtype in (0, 1):
        assert size(256, 4096, 16, 128, 256, dtype) == 0 and n.value == 0  # the GPU is full without segments
        assert size(1, 100000, 2, 128, 1, dtype) == 0 and n.value >= 2 * 2 * 128 * 128 * 4
        assert back(256, 100, 16, 16, 16, 16, 64, 256, dtype) == 0 and n.value == 0
        assert back(256, 100, 16, 16, 4, 4, 64, 256, dtype) == 0 and n.value == 2 * 256 * 100 * 16 * 64 * 4
    assert size(1, 10, 2, 128, 1, 3) == INVALID and size(1, 10, 2, 96, 1, 0) == UNSUPPORTED
    assert back(1, 10, 4, 3, 4, 4, 64, 1, 0) == INVALID and b"divisor" in lib.ccq_last_error()
    assert lib.ccq_decay_attention_workspace_size(1, 10, 2, 64, 1, 0, None) == INVALID
    assert lib.ccq_decay_attention_bwd_workspace_size(1, 10, 2, 2, 2, 2, 64, 1, 0, None) == INVALID


def test_status_word_is_required(lib):
    if torch.cuda.is_available():
        pytest.skip("a device resolves the status word")
    a = attention()
    assert lib.ccq_decay_attention(*a.values()) == ccq.CCQ_ERR_CUDA and b"status word" in lib.ccq_last_error()
    step = (heads(), heads(), heads(), 1, FAKE, 0.1, FAKE, 9, None, 8, heads(FAKE * 2), 5, 4, 64, None)
    assert lib.ccq_decay_attention_step(*step) == ccq.CCQ_ERR_CUDA and b"status word" in lib.ccq_last_error()


def test_the_binding_refuses_cpu_tensors():
    x, p = torch.zeros(1, 4, 2, 64), torch.zeros(1, 4, dtype=torch.int64)
    ld, f = torch.zeros(2), torch.zeros(32, dtype=torch.float64)
    for call in (lambda: ops.rotary(x, x, p, f), lambda: ops.rotary_bwd(x, None, p, f), lambda: ops.decay_attention(x, x, x, ld),
                 lambda: ops.decay_attention_bwd(x, x, x, ld, x),
                 lambda: ops.decay_attention_step(x[0], x[0], x[0], ld, torch.zeros(4, 2, 64, 64))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


class OnDevice:
    """Tensors as the binding's checks see them on a GPU."""

    @pytest.fixture(autouse=True)
    def patch(self, monkeypatch):
        monkeypatch.setattr(ops, "_cuda", lambda t, name, device=None: t)


class TestBinding(OnDevice):
    def test_shapes_and_types(self):
        x, ld = torch.zeros(2, 4, 4, 64), torch.zeros(4)
        cases = [(ValueError, "batch, tokens", lambda: ops.decay_attention(x[0], x, x, ld)),
                 (ValueError, "k has shape", lambda: ops.decay_attention(x, x[:1], x, ld)),
                 (ValueError, "v must be", lambda: ops.decay_attention(x, x, x[0], ld)),
                 (TypeError, "k must be", lambda: ops.decay_attention(x, x.double(), x, ld)),
                 (ValueError, "no divisor of 3", lambda: ops.decay_attention(x, x, x, ld[:3])),
                 (ValueError, r"\[heads\]", lambda: ops.decay_attention(x, x, x, ld.view(2, 2))),
                 (TypeError, "log_decay", lambda: ops.decay_attention(x, x, x, ld.double())),
                 (ValueError, "contiguous channels", lambda: ops.decay_attention(x.transpose(-1, -2).contiguous().transpose(-1, -2), x, x, ld)),
                 (ValueError, "cu_seqlens", lambda: ops.decay_attention(x, x, x, ld, cu_seqlens=torch.zeros(3, dtype=torch.int64))),
                 (TypeError, "cu_seqlens", lambda: ops.decay_attention(x[:1], x[:1], x[:1], ld, cu_seqlens=torch.zeros(3))),
                 (ValueError, "state has shape", lambda: ops.decay_attention(x, x, x, ld, state=torch.zeros(1, 4, 64, 64))),
                 (TypeError, "final_state", lambda: ops.decay_attention(x, x, x, ld, final_state=torch.zeros(2, 4, 64, 64).double())),
                 (ValueError, "dout has shape", lambda: ops.decay_attention_bwd(x, x, x, ld, x[:, :2])),
                 (ValueError, "dstate has shape", lambda: ops.decay_attention_bwd(x, x, x, ld, x, out={"dstate": x})),
                 (ValueError, "batch, heads, d", lambda: ops.decay_attention_step(x, x, x, ld, x)),
                 (ValueError, "state has shape", lambda: ops.decay_attention_step(x[0], x[0], x[0], ld, torch.zeros(5, 4, 64, 64))),
                 (ValueError, "slots have shape", lambda: ops.decay_attention_step(x[0], x[0], x[0], ld, torch.zeros(5, 4, 64, 64),
                                                                                   slots=torch.zeros(3, dtype=torch.int64))),
                 (TypeError, "slots must be", lambda: ops.decay_attention_step(x[0], x[0], x[0], ld, torch.zeros(5, 4, 64, 64), slots=torch.zeros(4)))]
        p, f = torch.zeros(2, 4, dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
        cases += [(ValueError, "q must be", lambda: ops.rotary(x[0, 0], None, p, f)), (ValueError, "k must be", lambda: ops.rotary(x, x[0], p, f)),
                  (ValueError, "k has shape", lambda: ops.rotary(x, x[:, :2], p, f)), (ValueError, "k has shape", lambda: ops.rotary(x, x[..., :32], p, f)),
                  (TypeError, "freqs must be", lambda: ops.rotary(x, x, p, f.float())), (TypeError, "positions must be", lambda: ops.rotary(x, x, p.float(), f)),
                  (ValueError, "positions have shape", lambda: ops.rotary(x, x, p[0], f)), (ValueError, "out has shape", lambda: ops.rotary(x, x, p, f, out=(x[0], None)))]
        for error, text, call in cases:
            with pytest.raises(error, match=text):
                call()


def test_frequencies():
    f, m = ops.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0 and f[0] == 1 and abs(f[-1] / 10000 ** (-62 / 64) - 1) < 1e-15
    g, m = ops.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert torch.equal(g, f / 4) and m == 1.0
    g, m = ops.rotary_frequencies(64, scaling="ntk", factor=4.0, device="cpu")
    assert g[0] == 1 and abs(g[-1] * 4 / f[-1] - 1) < 1e-12 and m == 1.0  # the fastest kept, the slowest stretched by the factor
    g, m = ops.rotary_frequencies(64, scaling="yarn", factor=4.0, original_length=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns > 40], f[turns > 40]) and torch.allclose(g[turns < 0.8], f[turns < 0.8] / 4, rtol=1e-14)
    assert ((g <= f) & (g >= f / 4 * (1 - 1e-14))).all() and m == 0.1 * math.log(4) + 1
    assert ops.rotary_frequencies(2, scaling="ntk", factor=4.0, device="cpu")[0].tolist() == [1.0]
    for bad in (dict(part=7), dict(part=0), dict(part=8, base=1.0), dict(part=8, factor=0.5, scaling="ntk"), dict(part=8, scaling="cubic"),
                dict(part=8, factor=2.0), dict(part=8, factor=2.0, scaling="yarn", original_length=0),
                dict(part=8, factor=2.0, scaling="yarn", fast=1.0, slow=2.0), dict(part=8, factor=math.inf, scaling="linear")):
        with pytest.raises(ValueError):
            ops.rotary_frequencies(bad.pop("part"), device="cpu", **bad)


def test_outputs_that_another_block_still_reads_are_refused(lib):
    """Outputs on top of inputs or each other, where blocks that run at the same time would read what others have written."""
    big = 2 * 4 * 128 * 128 * 4  # bytes of the states
    good = dict(attention(), S0=FAKE * 16)
    for off in (16, -16, big - 16, 16 - big):
        refused(lib, lib.ccq_decay_attention, good, INVALID, b"ST overlaps S0", ST=FAKE * 16 + off)
    a = attention()
    good = dict(q=a["q"], k=a["k"], v=a["v"], dtype=0, ld=FAKE, scale=0.1, S0=FAKE * 32, do=heads(), dST=FAKE * 64, dq=heads(FAKE * 2),
                dk=heads(FAKE * 3), dv=heads(FAKE * 4, n=2), dS0=FAKE * 128, B=2, T=32, H=4, d=128, cu=None, cb=8, n=2, ws=FAKE,
                nbytes=1 << 30, stream=None)
    for text, ch in ((b"dS0 overlaps S0", dict(dS0=FAKE * 32)), (b"dS0 overlaps S0", dict(dS0=FAKE * 32 + big - 16)),
                     (b"dS0 overlaps dST", dict(dS0=FAKE * 64 + 16)), (b"dk is dq", dict(dk=heads(FAKE * 2))),
                     (b"dv is dk", dict(dv=heads(FAKE * 3, n=2))), (b"dq is dv", dict(dq=heads(FAKE * 4)))):
        refused(lib, lib.ccq_decay_attention_bwd, good, INVALID, text, **ch)
    step = dict(q=heads(), k=heads(FAKE * 2), v=heads(FAKE * 3, n=1), dtype=1, ld=FAKE, scale=0.1, state=FAKE, rows=9, slots=FAKE, sb=8,
                o=heads(), B=5, H=4, d=64, stream=None)
    for name, at in (("q", 1), ("k", 2), ("v", 3)):
        refused(lib, lib.ccq_decay_attention_step, step, INVALID, b"o is " + name.encode(), o=heads(FAKE * at))
    rotary = dict(x=heads() + heads(FAKE * 2), y=heads() + heads(FAKE * 2), count=2, dtype=0, B=2, T=32, width=128, part=64, positions=FAKE,
                  pb=8, freqs=FAKE, amplitude=1.0, inter=0, inverse=0, stream=None)
    for text, y in ((b"other strides", heads(token=1024, batch=1 << 15) + heads(FAKE * 2)), (b"is x[1]", heads(FAKE * 2) + heads(FAKE * 3)),
                    (b"is x[0]", heads(FAKE * 3) + heads()), (b"is y[1]", heads(FAKE * 3) + heads(FAKE * 3))):
        refused(lib, lib.ccq_rotary, rotary, INVALID, text, y=y)


def test_plans_of_tensors_without_heads_are_none():
    """(the call then goes the way that says what is wrong with them)"""
    one, two = (torch.bfloat16, torch.Size([4]), (1,)), (torch.bfloat16, torch.Size([4, 2, 64]), (128, 64, 1))
    pos, freqs = (torch.int64, torch.Size([4]), (1,)), (torch.float64, torch.Size([32]), (1,))
    assert ops._rotary_plan(two, two, pos, freqs) is not None
    for q, k in ((one, one), (one, two), (two, one)):
        assert ops._rotary_plan(q, k, pos, freqs) is None
