"""Host-side checks of ccq_zero_outside: what it refuses, and calls without tokens."""
import struct

import pytest

from paper_2606_01294_gb300 import _build, ccq, ops

FAKE = 0x10000  # aligned, never dereferenced on these paths
INVALID, UNSUPPORTED = ccq.CCQ_ERR_INVALID_ARG, ccq.CCQ_ERR_UNSUPPORTED


def heads(p=FAKE, batch=0, token=512, head=128, n=4):
    return struct.pack("5q", p, batch, token, head, n)


def test_refusals():
    _build.build()
    lib = ops._library()
    assert "ccq_zero_outside" in ccq.header_symbols()
    good = dict(x=heads(), dtype=0, T=32, width=128, cu=FAKE, cb=8, n=3, stream=None)
    for status, text, ch in ((INVALID, b"NULL", dict(x=None)), (INVALID, b"dtype", dict(dtype=4)), (INVALID, b"sizes", dict(T=-1)),
                             (UNSUPPORTED, b"2^31", dict(T=1 << 31)), (INVALID, b"width", dict(width=0)), (INVALID, b"width", dict(width=1 << 17)),
                             (UNSUPPORTED, b"sequences", dict(n=-1)), (UNSUPPORTED, b"sequences", dict(n=1 << 25)),
                             (INVALID, b"cu_bytes", dict(cb=2)), (INVALID, b"cu is NULL", dict(cu=None)), (INVALID, b"aligned", dict(cu=FAKE + 4)),
                             (INVALID, b"x is NULL", dict(x=heads(0))), (INVALID, b"aligned", dict(x=heads(FAKE + 1))),
                             (INVALID, b"overlap", dict(x=heads(token=256))), (INVALID, b"heads", dict(x=heads(n=0))),
                             (INVALID, b"stride", dict(x=heads(token=-512))),
                             (UNSUPPORTED, b"2^24", dict(x=heads(head=65536, token=1 << 36, n=1 << 10), width=65536))):
        assert lib.ccq_zero_outside(*dict(good, **ch).values()) == status, ch
        assert text in lib.ccq_last_error(), (ch, lib.ccq_last_error())
    assert lib.ccq_zero_outside(*dict(good, T=0).values()) == 0
