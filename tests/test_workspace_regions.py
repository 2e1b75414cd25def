"""Calls of every kind and shape may share a workspace: what one call finds at zero and leaves at zero, no other call writes.  Seen from
what the kernels are given (no GPU: tests/fake_args.cpp)."""
import ctypes as C
import os

import pytest

from paper_2412_14468_b200 import binding as ha
from tests import _fake
from tests._fake import PTR, Fake

WS = 1 << 40                                        # the workspace's address
ROOM = 1 << 32
HEADER = 256
COUNTERS = 3 * 1024 * 4                             # decode: three counters of each unit where units are cut (at most 1024 units are)
TICKETS = 160 * 4                                   # attention of new tokens


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    usual, _fake.SRC = _fake.SRC, os.path.join(os.path.dirname(_fake.SRC), "fake_args.cpp")
    try:
        f = Fake(tmp_path_factory.mktemp("fake"), "fake_args")
    finally:
        _fake.SRC = usual
    # kernel, which argument, its 64-bit words
    for text, arg, words in (("chunk_attn_kernel", 3, 26), ("pages_plan_extend_kernel", 2, 5), ("pages_plan_compact_kernel", 3, 5), ("11attn_kernel", 0, 28),
                             ("wide_scan_kernel", 0, 20), ("13select_kernel", 9, 1)):
        f.lib.fake_watch(text.encode(), arg, words)
    return f


def offsets(fake):
    """Offsets into the workspace that kernels were given since the last look, the header's own apart."""
    out, words = [], (C.c_ulonglong * 64)()
    for i in range(fake.lib.fake_seen()):
        out += [words[k] - WS for k in range(fake.lib.fake_words(i, words)) if WS <= words[k] < WS + ROOM]
    assert fake.lib.fake_seen() > 0
    fake.lib.fake_forget()
    return sorted(o for o in out if o > 0)


POOL = ha.ha_tensor(PTR, 8 * 16 * 128, 16 * 128, 128)
ROWS = ha.ha_tensor(PTR, 0, 128, 48 * 128)


def chunk(f, B=3):
    shape = ha.make_shape(B, 32, 8, 0.1)
    return f.lib.ha_chunk_attn_paged(C.byref(shape), C.byref(ROWS), PTR, 7, C.byref(POOL), C.byref(POOL), 50, PTR, 4, 16, PTR, 1, PTR, None, WS, ROOM, None)


def extend(f, B, pages):
    return f.lib.ha_pages_extend(PTR, PTR, B, PTR, 10, 10, 16, PTR, pages, 8, C.byref(POOL), C.byref(POOL), None, 0, 0, WS, ROOM, None)


def compact(f, B, pages):
    return f.lib.ha_pages_compact(PTR, B, PTR, 10, 10, 16, PTR, pages, 8, C.byref(POOL), C.byref(POOL), None, 0, 0, PTR, 10, PTR, PTR, PTR, WS, ROOM, None)


def dense(f, B, Hkv):
    shape = ha.make_shape(B, Hkv * 4, Hkv, 0.1)
    return f.lib.ha_dense_decode(C.byref(shape), PTR, C.byref(POOL), C.byref(POOL), PTR, 5000, PTR, None, WS, ROOM, None)


def score(f):
    shape = ha.make_shape(1, 1, 1, 0.1)
    return f.lib.ha_score_topk(C.byref(shape), PTR, PTR, 1 << 22, 1 << 22, PTR, None, 64, 1 << 21, 64, PTR, 64, 64, PTR, None, WS, ROOM, None)


def wide(f, B, Hkv):
    shape = ha.make_shape(B, Hkv, Hkv, 0.1)
    return f.lib.ha_score_topk_wide(C.byref(shape), 128, PTR, PTR, 1 << 22, 1 << 20, PTR, None, 64, 1 << 19, 64, PTR, 64, 64, PTR, None, WS, ROOM, None)


def test_scratch_of_every_kind_lies_behind_the_counters_of_every_kind(fake):
    first = HEADER + COUNTERS + TICKETS
    for B, Hkv in ((1, 1), (2, 8), (12, 8), (128, 8), (129, 8), (4096, 16)):
        assert dense(fake, B, Hkv) == ha.HA_OK
        at = offsets(fake)
        assert at[0] == HEADER and at[1] >= first, (B, Hkv, at)           # its counters, then its parts
    assert score(fake) == ha.HA_OK
    assert offsets(fake)[0] >= first
    assert chunk(fake) == ha.HA_OK
    at = offsets(fake)
    assert HEADER + COUNTERS <= at[0] <= first - TICKETS and at[1] >= first, at
    for call, B, pages in ((extend, 1, 1), (extend, 500, 7), (extend, 4, 100000), (compact, 1, 1), (compact, 65535, 3)):
        assert call(fake, B, pages) == ha.HA_OK
        at = offsets(fake)
        assert at[0] >= first, (call.__name__, at)
    for B, Hkv in ((1, 1), (9, 8)):
        assert wide(fake, B, Hkv) == ha.HA_OK
        at = offsets(fake)
        assert at[0] >= first, at


def test_every_workspace_has_room_for_the_counters(fake):
    """ha_workspace_init clears what it is given: a workspace of any kind, prepared once, serves calls of any kind that fit it."""
    first = HEADER + COUNTERS + TICKETS
    shape = ha.make_shape(1, 1, 1, 0.1)
    for n in (ha.ha_workspace_bytes(shape, 0, 0), ha.ha_workspace_bytes_chunk(), ha.ha_workspace_bytes_pages(0, 0), ha.ha_workspace_bytes_wide(shape, 0)):
        assert n >= first
