"""Refusals of ha_chunk_attn_paged, ha_rotary*, ha_pages_*: on the host, before anything reaches CUDA."""
import ctypes as C
import math

import pytest
import torch

from paper_2412_14468_b200 import binding as ha
from paper_2412_14468_b200 import build as ha_build

FAKE = 0x1000          # never dereferenced: validation fails first
OK, ARG, UNSUP, WS = ha.HA_OK, ha.HA_ERR_INVALID_ARG, ha.HA_ERR_UNSUPPORTED, ha.HA_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    ha_build.build()
    return ha.lib()


def ref(x):
    return None if x is None else C.byref(x)


ROWS = ha.ha_tensor(FAKE, 0, 128, 48 * 128)
POOL = ha.ha_tensor(FAKE, 8 * 16 * 128, 16 * 128, 128)


def test_chunk_attention(lib):
    def call(shape=ha.make_shape(2, 32, 8, 0.1), q=ROWS, off=FAKE, rows=7, K=POOL, V=POOL, pages=5, table=FAKE, ps=16, lens=FAKE, out=FAKE,
             ws=FAKE, nbytes=1 << 30):
        return lib.ha_chunk_attn_paged(C.byref(shape), ref(q), off, rows, ref(K), ref(V), pages, table, 4, ps, lens, 1, out, None, ws, nbytes, None)

    assert call(rows=0) == OK and call(shape=ha.make_shape(0, 32, 8, 0.1)) == OK     # nothing to do
    for bad in (dict(q=None), dict(off=None), dict(rows=-1), dict(K=None), dict(V=None), dict(pages=-1), dict(table=None), dict(lens=None),
                dict(out=None), dict(out=FAKE + 8), dict(ps=0), dict(ps=12), dict(ps=131072),
                dict(q=ha.ha_tensor(FAKE + 2, 0, 128, 4096)), dict(q=ha.ha_tensor(FAKE, 0, 64, 4096)), dict(q=ha.ha_tensor(FAKE, 0, 132, 4096)),
                dict(q=ha.ha_tensor(FAKE, 0, 128, 4097)), dict(q=ha.ha_tensor(FAKE, 0, 128, -4096)), dict(q=ha.ha_tensor(None, 0, 128, 4096)),
                dict(K=ha.ha_tensor(FAKE, 8 * 16 * 128 + 4, 16 * 128, 128)), dict(V=ha.ha_tensor(FAKE, 8 * 16 * 128, 16 * 128, 120)),
                dict(shape=ha.make_shape(-1, 32, 8, 0.1)), dict(shape=ha.make_shape(2, 32, 8, math.nan))):
        assert call(**bad) == ARG, bad
    for bad in (dict(shape=ha.make_shape(2, 24, 8, 0.1)), dict(shape=ha.make_shape(2, 32, 2, 0.1)), dict(shape=ha.make_shape(2, 32, 8, 0.1, head_dim=64))):
        assert call(**bad) == UNSUP, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(nbytes=ha.ha_workspace_bytes_chunk() - 1)):
        assert call(**bad) == WS, bad


def test_rotary(lib):
    def call(x=ROWS, y=ROWS, rows=3, heads=5, f=FAKE, rot=128, pos=FAKE, scale=1.0):
        return lib.ha_rotary(ref(x), ref(y), rows, heads, f, rot, pos, 0, 0, scale, None)

    assert call(rows=0) == OK
    for bad in (dict(x=None), dict(y=None), dict(rows=-1), dict(heads=0), dict(f=None), dict(f=FAKE + 4), dict(pos=None), dict(scale=math.nan),
                dict(y=ha.ha_tensor(FAKE + 4, 0, 128, 4096)), dict(x=ha.ha_tensor(FAKE, 0, 100, 4096))):
        assert call(**bad) == ARG, bad
    for bad in (dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(heads=70000)):
        assert call(**bad) == UNSUP, bad


def test_rotary_frequencies(lib):
    out = (C.c_double * 64)()

    def call(rot=128, theta=1e4, rule=0, factor=2.0, low=1.0, high=4.0, ctx=8192.0, to=out):
        return lib.ha_rotary_freqs(rot, theta, rule, factor, low, high, ctx, to, None)

    assert all(call(rule=r) == OK for r in range(5))
    for bad in (dict(to=None), dict(theta=1.0), dict(theta=math.nan), dict(theta=math.inf), dict(rule=5), dict(rule=-1), dict(rule=1, factor=0.0),
                dict(rule=2, factor=math.nan), dict(rule=3, low=4.0), dict(rule=4, low=0.0), dict(rule=3, ctx=0.0), dict(rule=4, high=math.inf)):
        assert call(**bad) == ARG, bad
    assert call(rot=136) == UNSUP and call(rot=20) == UNSUP
    with pytest.raises(ha.HashAttnError):
        ha.ha_rotary_freqs(20, 1e4)


def test_rotary_append(lib):
    def call(shape=ha.make_shape(2, 32, 8, 0.1), q=ROWS, k=ROWS, v=ROWS, qo=ROWS, ko=None, off=FAKE, rows=3, f=FAKE, rot=128, K=POOL, V=POOL, pages=5,
             table=FAKE, ps=16, lens=FAKE, ws=None):
        return lib.ha_rotary_append_paged(C.byref(shape), ref(q), ref(k), ref(v), ref(qo), ko, off, rows, f, rot, None, 0, 1.0, ref(K), ref(V), pages,
                                          table, 4, ps, lens, ws, None)

    assert call(rows=0) == OK
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(qo=None), dict(ko=FAKE + 8), dict(off=None), dict(rows=-1), dict(f=None), dict(K=None),
                dict(V=None), dict(table=None), dict(lens=None), dict(ps=3), dict(pages=-2), dict(shape=ha.make_shape(-1, 32, 8, 0.1))):
        assert call(**bad) == ARG, bad
    assert call(rot=24) == UNSUP and call(ws=FAKE + 16) == WS


def test_pages(lib):
    base = dict(lens=FAKE, B=4, table=FAKE, s0=10, width=10, ps=16, ref=FAKE, pages=50, ws=FAKE, nbytes=1 << 20)

    def fork(**kw):
        k = {**base, "p": FAKE, "c": FAKE, "n": 0, **kw}
        return lib.ha_pages_fork(k["p"], k["c"], k["n"], k["lens"], k["B"], k["table"], k["s0"], k["width"], k["ps"], k["ref"], k["pages"], k["ws"], k["nbytes"], None)

    def free(**kw):
        k = {**base, "p": FAKE, "n": 0, **kw}
        return lib.ha_pages_free(k["p"], k["n"], k["lens"], k["B"], k["table"], k["s0"], k["width"], k["ps"], k["ref"], k["pages"], k["ws"], k["nbytes"], None)

    def extend(**kw):
        k = {**base, "add": FAKE, "heads": 8, "K": POOL, "V": POOL, "codes": None, **kw}
        return lib.ha_pages_extend(k["add"], k["lens"], k["B"], k["table"], k["s0"], k["width"], k["ps"], k["ref"], k["pages"], k["heads"], ref(k["K"]),
                                   ref(k["V"]), k["codes"], 0, 0, k["ws"], k["nbytes"], None)

    def compact(**kw):
        k = {**base, "heads": 8, "K": POOL, "V": POOL, "codes": None, "t_out": FAKE, "o0": 10, "r_out": FAKE, "map": FAKE, "used": FAKE, **kw}
        return lib.ha_pages_compact(k["lens"], k["B"], k["table"], k["s0"], k["width"], k["ps"], k["ref"], k["pages"], k["heads"], ref(k["K"]), ref(k["V"]),
                                    k["codes"], 0, 0, k["t_out"], k["o0"], k["r_out"], k["map"], k["used"], k["ws"], k["nbytes"], None)

    assert fork() == OK and free() == OK and extend(B=0) == OK
    for call in (fork, free, extend, compact):
        for bad in (dict(lens=None), dict(B=-1), dict(table=None), dict(s0=9), dict(width=-1), dict(ps=0), dict(ps=24), dict(ref=None), dict(pages=-1)):
            assert call(**bad) == ARG, (call.__name__, bad)
        assert call(B=70000) == UNSUP
        for bad in (dict(ws=None), dict(ws=FAKE + 1), dict(nbytes=ha.ha_workspace_bytes_pages(50, 4) - 1)):
            assert call(**bad) == WS, (call.__name__, bad)
    for bad in (dict(n=-1), dict(n=2, p=None), dict(n=2, c=None)):
        assert fork(**bad) == ARG, bad
    assert fork(n=70000) == UNSUP and free(n=70000) == UNSUP and free(n=-1) == ARG and free(n=1, p=None) == ARG
    assert extend(add=None) == ARG
    for call in (extend, compact):
        for bad in (dict(heads=0), dict(K=None), dict(V=None), dict(codes=FAKE + 2), dict(K=ha.ha_tensor(FAKE, 8, 8, 100))):
            assert call(**bad) == ARG, (call.__name__, bad)
    for bad in (dict(t_out=None), dict(r_out=None), dict(map=None), dict(used=None), dict(o0=9)):
        assert compact(**bad) == ARG, bad
    assert lib.ha_workspace_bytes_pages(-1, 4) == 0 and lib.ha_workspace_bytes_pages(4, 70000) == 0
    with pytest.raises(ha.HashAttnError):
        ha.ha_workspace_bytes_pages(-1, 1)


def test_the_binding_wants_tensors_on_the_device(lib):
    t, i = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(9, dtype=torch.int32)
    pool = torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16)
    shape = ha.make_shape(1, 8, 2, 0.1)
    with pytest.raises(TypeError):
        ha.ha_chunk_attn_paged(shape, t, i, pool, pool, i.view(1, 9), 16, i, t, None)
    with pytest.raises(TypeError):
        ha.ha_rotary(t, t, torch.zeros(64, dtype=torch.float64), i)
    with pytest.raises(TypeError):
        ha.ha_rotary_append_paged(shape, t, t[:, :2], t[:, :2], t, torch.zeros(64, dtype=torch.float64), i, pool, pool, i.view(1, 9), 16, i)
    with pytest.raises(TypeError):
        ha.ha_pages_fork(i, i, i, i.view(1, 9), 16, i, None)
    with pytest.raises(TypeError):
        ha.ha_pages_extend(i, i, i.view(1, 9), 16, i, pool, pool, None, None)
    with pytest.raises(TypeError):
        ha.ha_pages_free(i, i, i.view(1, 9), 16, i, None)
    with pytest.raises(TypeError):
        ha.ha_pages_compact(i, i.view(1, 9), 16, i, pool, pool, None, i.view(1, 9), i, i, i, None)
