"""Host-side checks of the outputs that a call refuses because they share an element with what other blocks still read or write:
exactly those that do, for any strides.  (No call gets as far as a launch: those that pass this check are refused by a later one.)"""
import itertools
import random
import struct

import numpy as np
import pytest
import torch

from paper_2606_01294_gb300 import _build, ccq, ops

INVALID = ccq.CCQ_ERR_INVALID_ARG
BASE, FAR, STATES = 1 << 30, 1 << 40, 1 << 50  # addresses, never dereferenced


@pytest.fixture(scope="module")
def lib():
    _build.build()
    return ops._library()


def view(at, batch, token, head, n):
    """A tensor of 2-byte elements from element `at` on."""
    return struct.pack("5q", BASE + 2 * at, batch, token, head, n)


def far(i, n, d, B, T):
    return struct.pack("5q", FAR * (i + 1), T * n * d, n * d, d, n)


def attention(lib, q, o, B, T, H, d, k=None, v=None):
    """None where the tensors pass, else what the call says of them."""
    st = lib.ccq_decay_attention(q, k or far(1, H, d, B, T), v or far(2, H, d, B, T), 0, BASE * 2 ** 10, 0.1, STATES, o, STATES + 16, B, T, H, d,
                                 None, 8, B, 1 << 45, 1 << 40, None)
    assert st == INVALID
    text = lib.ccq_last_error()
    return None if b"ST overlaps S0" in text else text


def elements(at, batch, token, head, n, B, T, d):
    i = np.add.outer(np.add.outer(np.add.outer(np.arange(B) * batch, np.arange(T) * token), np.arange(n) * head), np.arange(d))
    return i.ravel() + at


def layout(rng, B, T, n, d, dense):
    """Strides of a nested layout: the dimensions in any order, with gaps."""
    order = [("batch", B), ("token", T), ("head", n)]
    rng.shuffle(order)
    reach, s = d, {}
    for name, extent in order:
        s[name] = reach + (0 if dense else rng.choice([0, 0, 1, 7, 64, d, 3 * d]))
        reach = s[name] * extent
    return s["batch"], s["token"], s["head"]


def test_exactly_those_that_share_an_element(lib):
    rng = random.Random(5)
    counts = [0, 0]
    for _ in range(4000):
        d, H = 64, rng.choice([1, 2, 3, 4])
        B, T = rng.choice([1, 2, 3]), rng.choice([1, 2, 5, 9])
        dense = rng.random() < 0.3
        o = layout(rng, B, T, H, d, dense)
        n = rng.choice([x for x in range(1, H + 1) if H % x == 0])
        kind = rng.random()
        if kind < 0.4 and n == H:
            q = o
        elif kind < 0.6:
            q = tuple(rng.choice([0, 1, 8, 64, 100, 640]) for _ in range(3))  # an input may overlap itself
        else:
            q = layout(rng, B, T, n, d, dense)
        size = max(o[0] * B + o[1] * T + o[2] * H, 300)
        at = rng.choice([rng.randrange(-size, size), d * rng.randrange(-size // d, size // d), rng.choice([-1, 1]) * rng.choice(o)])
        if at == 0:
            continue
        mine, theirs = elements(0, *o, H, B, T, d), elements(at, *q, n, B, T, d)
        shared = np.intersect1d(mine, theirs).size > 0
        said = attention(lib, view(at, *q, n), view(0, *o, H), B, T, H, d)
        assert said is None or b"o overlaps q" in said
        assert (said is not None) == shared, (o, q, at, B, T, H, n)
        counts[shared] += 1
    assert min(counts) > 500


def test_slices_of_one_projection(lib):
    """q, k, v and o side by side in one tensor of any order pass, at the sizes of a layer; a token, a head or an element further do not."""
    H, d = 16, 128
    for B, T in ((8, 4096), (1, 20480), (300, 1)):
        strides = (T * 4 * H * d, 4 * H * d, d)
        parts = [view(i * H * d, *strides, H) for i in range(4)]
        for order in itertools.islice(itertools.permutations(parts), 0, 24, 5):
            assert attention(lib, order[0], order[3], B, T, H, d, order[1], order[2]) is None
        for off in (1, -1, d, H * d - 1, -(H * d - 1), 4 * H * d + 5) if T > 1 else (1, -1, d, H * d - 1):
            assert b"o overlaps q" in attention(lib, view(2 * H * d + off, *strides, H), parts[2], B, T, H, d)
            assert b"o overlaps k" in attention(lib, far(0, H, d, B, T), parts[2], B, T, H, d, k=view(2 * H * d + off, *strides, H))
            assert b"o overlaps v" in attention(lib, far(0, H, d, B, T), parts[2], B, T, H, d, v=view(2 * H * d + off, *strides, H))
    # heads first against tokens first, in one piece of memory
    assert b"overlaps" in attention(lib, view(7, 9 * 4 * 64, 64, 9 * 64, 4), view(0, 9 * 4 * 64, 4 * 64, 64, 4), 2, 9, 4, 64)
    # one after another
    assert attention(lib, view(2 * 9 * 4 * 64, 9 * 4 * 64, 64, 9 * 64, 4), view(0, 9 * 4 * 64, 4 * 64, 64, 4), 2, 9, 4, 64) is None


def test_gradients(lib):
    B, T, H, d = 2, 32, 4, 128

    def call(**given):
        tensors = {n: far(i, H, d, B, T) for i, n in enumerate(("q", "k", "v", "dout", "dq", "dk", "dv"))} | given
        t = list(tensors.values())
        st = lib.ccq_decay_attention_bwd(*t[:3], 0, BASE, 0.1, STATES, t[3], None, *t[4:], STATES + 16, B, T, H, d, None, 8, B, BASE, 1 << 30, None)
        assert st == INVALID
        return lib.ccq_last_error()

    strides = (T * H * d, H * d, d)
    assert b"dS0 overlaps S0" in call()
    for out in ("dq", "dk", "dv"):
        for other in ("q", "k", "v", "dout", "dq", "dk", "dv"):
            if other == out:
                continue
            text = call(**{out: view(0, *strides, H), other: view(H * d, *strides, H)})
            assert b"overlaps" in text and out.encode() in text and other.encode() in text
    wide = (T * 2 * H * d, 2 * H * d, d)
    assert b"dS0 overlaps S0" in call(dq=view(0, *wide, H), dk=view(H * d, *wide, H))


def test_rotary(lib):
    B, T, H, d = 2, 32, 4, 128
    strides = (T * 3 * H * d, 3 * H * d, d)
    q, k, v = (view(i * H * d, *strides, H) for i in range(3))

    def call(x, y):
        st = lib.ccq_rotary(x, y, len(x) // 40, 0, B, T, d, d, BASE, 8, BASE, 1.0, 0, 0, None)
        return st, lib.ccq_last_error()

    shifted = [view(i * H * d + off, *strides, H) for i, off in ((0, d), (1, -d), (2, 3 * H * d))]
    for x, y, text in ((q, shifted[0], b"y[0] overlaps x[0]"), (q + k, shifted[1] + v, b"y[0] overlaps x[0]"), (q + k, v + shifted[0], b"y[1] overlaps x[0]"),
                       (q + k, v + shifted[2], b"y[1] overlaps y[0]"), (q + k, q + view(2 * H * d - 1, *strides, H), b"y[1] overlaps x[1]")):
        st, said = call(x, y)
        assert st == INVALID and text in said, said
    if torch.cuda.is_available():
        return  # (the next calls are right, and these are not a device's addresses)
    for x, y in ((q + k, q + k), (q + k, v + k), (q, v), (v + k, q + k)):
        assert call(x, y)[0] == ccq.CCQ_ERR_CUDA
