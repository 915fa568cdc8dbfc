"""The model operators' C entries on the host: kvs_ops_api.cpp and kvs_api.cpp over stand-ins
for CUDA and the kernels (ops_fake.cpp)."""
import ctypes
import os
import shutil
import subprocess
import threading
import time

import numpy as np
import pytest

from paper_2609_35065_gb300 import build, kvs
from test_ops_cpu import Call

HERE = os.path.dirname(os.path.abspath(__file__))
OPS = ["append", "attend", "weigh", "evict"]


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    cuda = os.path.join(os.path.dirname(os.path.dirname(build.nvcc())), "include")
    if not (shutil.which("g++") and os.path.exists(os.path.join(cuda, "cuda_runtime.h"))):
        pytest.skip("needs g++ and the CUDA headers")
    out = str(tmp_path_factory.mktemp("ops") / "libops.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-pthread", "-Wl,-Bsymbolic", "-I", build.INCLUDE, "-I", build.CSRC,
                    "-I", HERE, "-I", cuda, os.path.join(build.CSRC, "kvs_api.cpp"), os.path.join(build.CSRC, "kvs_ops_api.cpp"),
                    os.path.join(HERE, "ops_fake.cpp"), "-o", out], check=True)
    L = ctypes.CDLL(out)
    L.kvs_last_error.restype = ctypes.c_char_p
    L.kvs_stat_launches.restype = ctypes.c_int64
    L.kvs_attend_workspace.restype = ctypes.c_int64
    return L


def _run(lib, op, c, flags=0):
    b = ctypes.byref
    args = [b(c.geom), b(c.cache), b(c.step)] + ([] if op == "evict" else [c.layer]) + [b(getattr(c, op))]
    return getattr(lib, "kvs_" + op)(*args, None, ctypes.c_uint32(flags))


@pytest.mark.parametrize("op", OPS)
def test_a_valid_call_is_launched_and_counted(library, op):
    before, counted = library.fake_ops(), library.kvs_stat_launches()
    assert _run(library, op, Call()) == kvs.KVS_OK, library.kvs_last_error()
    assert library.fake_ops() == before + 1 and library.kvs_stat_launches() == counted + 1


def _retrieve(lib):
    """A retrieval whose tables are too large to travel with the launch."""
    g = kvs._geometry((2, 8, 128, 2, 16, 256))
    table = np.arange(16 * 200, dtype=np.int32)
    req = kvs.RequestArg(table, [kvs.ChunkArg((1 << 40) + (k << 30), 256, kvs.KVS_SRC_DEVICE) for k in range(200)])
    m = kvs._Marshalled([(1 << 44) + (p << 32) for p in range(4)], len(table), [req])
    return lib.kvs_retrieve(ctypes.byref(g), ctypes.byref(m.cache), m.reqs, m.n, None, ctypes.c_uint32(0))


def test_operators_do_not_wait_for_a_retrieval(library):
    """A retrieval that waits for one of its upload slots holds up no operator of another thread."""
    for op in OPS:
        assert _run(library, op, Call()) == kvs.KVS_OK        # the device's first call
    for _ in range(4):
        assert _retrieve(library) == kvs.KVS_OK               # every slot is in use
    library.fake_hold(1)
    other = threading.Thread(target=_retrieve, args=(library,))
    other.start()
    mine = None
    try:
        end = time.monotonic() + 5
        while not library.fake_held() and time.monotonic() < end:
            time.sleep(0.001)
        assert library.fake_held() == 1
        codes = []

        def operators():
            c = Call()
            codes.extend(_run(library, op, c) for op in OPS)
            codes.append(library.kvs_attend_workspace(ctypes.byref(c.geom), ctypes.byref(c.step), 4))

        mine = threading.Thread(target=operators)
        mine.start()
        mine.join(5)
        waited = mine.is_alive()
    finally:
        library.fake_hold(0)
        other.join()
        if mine:
            mine.join()
    assert codes == [kvs.KVS_OK] * 5
    assert not waited


def test_operators_after_a_shutdown(library):
    """The state that a shutdown frees is made anew by the next call."""
    for _ in range(2):
        for op in OPS:
            assert _run(library, op, Call()) == kvs.KVS_OK
        assert library.kvs_shutdown() == kvs.KVS_OK
    assert _run(library, "attend", Call(), kvs.KVS_F_VALIDATE) == kvs.KVS_OK


def _evict_rows(c, total_q, max_q):
    c.step.q_starts, c.step.total_q, c.step.max_q = None, total_q, max_q
    return c


def test_eviction_needs_no_rows(library):
    """kvs_evict uses no row of the step: without q_starts total_q may be 0, or one row per request."""
    before = library.fake_ops()
    for rows in ((0, 0), (2, 1)):
        assert _run(library, "evict", _evict_rows(Call(), *rows)) == kvs.KVS_OK, library.kvs_last_error()
    assert library.fake_ops() == before + 2
    for rows in ((1, 1), (3, 1), (8, 5)):
        assert _run(library, "evict", _evict_rows(Call(), *rows)) == kvs.KVS_ERR_INVALID_ARG
    for op in ("append", "attend", "weigh"):
        assert _run(library, op, _evict_rows(Call(), 0, 0)) == kvs.KVS_ERR_INVALID_ARG
    assert library.fake_ops() == before + 2
