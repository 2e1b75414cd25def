"""The driver's encoder of tensor maps is looked up once, also when several threads make their first calls at the same time (no GPU:
tests/fake_args.cpp, whose lookup takes a while)."""
import ctypes as C
import os
import threading

from paper_2412_14468_b200 import binding as ha
from tests import _fake
from tests._fake import PTR, Fake


def test_one_lookup_for_all_threads_and_kernels(tmp_path):
    usual, _fake.SRC = _fake.SRC, os.path.join(os.path.dirname(_fake.SRC), "fake_args.cpp")
    try:
        f = Fake(tmp_path, "fake_lookup")
    finally:
        _fake.SRC = usual
    m = ha.ha_mapping(8, 128, 128, 32, *([PTR] * 6))
    kv, rows = ha.ha_tensor(PTR, 8 * 16 * 128, 16 * 128, 128), ha.ha_tensor(PTR, 0, 128, 48 * 128)
    shape = ha.make_shape(1, 32, 8, 0.1)
    got = []
    prefill = lambda: got.append(f.lib.ha_encode_prefill(C.byref(m), 1, C.byref(kv), 1, 8, 500, PTR, 8 * 512, 512, 0, None, None))  # noqa: E731
    chunk = lambda: got.append(f.lib.ha_chunk_attn_paged(C.byref(shape), C.byref(rows), PTR, 7, C.byref(kv), C.byref(kv), 50, PTR, 4, 16, PTR, 1, PTR, None,  # noqa: E731
                                                         PTR, 1 << 30, None))
    threads = [threading.Thread(target=t) for t in (prefill, prefill, prefill, chunk, chunk)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert got == [ha.HA_OK] * 5
    assert f.lib.fake_lookups() == 1
