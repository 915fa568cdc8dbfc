"""The reader of tensors says what their attributes say, leaves alone what it does not know, and is done without
where it cannot be built."""
import ctypes
import shutil

import pytest
import torch

from paper_2609_35065_gb300 import build, kvs


class Read(ctypes.Structure):
    _fields_ = [("at", ctypes.c_uint64), ("shape", ctypes.c_int64 * 4), ("stride", ctypes.c_int64 * 4)]


def _address():
    if not build._has_python_headers() or shutil.which("g++") is None:
        pytest.skip("no Python headers or C++ compiler")
    address = build.load_tensor_reader()
    assert address
    return address


def _read(o, dtype, dims):
    read = ctypes.PYFUNCTYPE(ctypes.c_int, ctypes.py_object, ctypes.py_object, ctypes.c_int, ctypes.POINTER(Read))(_address())
    r = Read()
    return read(o, dtype, dims, ctypes.byref(r)), r


TENSORS = {
    "rows": lambda: torch.empty(5, 3, 64, dtype=torch.bfloat16),
    "view": lambda: torch.empty(5, 7, 96, dtype=torch.float16)[1:4, ::2, 8:72],
    "heads_first": lambda: torch.empty(4, 9, 32, dtype=torch.bfloat16).transpose(0, 1),
    "broadcast": lambda: torch.empty(1, 8).expand(6, 8),
    "empty": lambda: torch.empty(0, 4, 128, dtype=torch.float16),
    "four": lambda: torch.empty(2, 3, 4, 5, dtype=torch.int32),
    "scalar": lambda: torch.empty(()),
    "parameter": lambda: torch.nn.Parameter(torch.empty(3, 2)),
    "leaf": lambda: torch.empty(3, 2, requires_grad=True),
    "bytes": lambda: torch.empty(1000, dtype=torch.uint8)[24:],
    "meta": lambda: torch.empty(3, 2, device="meta"),
}


@pytest.mark.parametrize("name", sorted(TENSORS))
def test_a_tensor_is_read_as_its_attributes_say(name):
    t = TENSORS[name]()
    got, r = _read(t, t.dtype, t.dim())
    assert got == 1 and r.at == t.data_ptr()
    assert tuple(r.shape[:t.dim()]) == tuple(t.shape) and tuple(r.stride[:t.dim()]) == t.stride()
    assert _read(t, t.dtype, t.dim() + 1)[0] == 0
    assert _read(t, torch.float64, t.dim())[0] == 0


class Own(torch.Tensor):
    pass


@pytest.mark.parametrize("o", [None, 3, "text", [1], object(), torch.zeros(3, 2).numpy(), torch.zeros(3, 2).as_subclass(Own),
                               torch.zeros(3, 2).to_sparse()], ids=lambda o: type(o).__name__)
def test_what_it_does_not_know_is_left_to_the_attributes(o):
    assert _read(o, torch.float32, 2)[0] == 2


def test_a_dtype_that_is_none_is_left_to_the_attributes():
    assert _read(torch.zeros(2), "float32", 1)[0] == 2


@pytest.mark.parametrize("cause", ["no_compiler", "broken_source", "no_extension"])
def test_a_reader_that_is_not_to_be_had_is_done_without(monkeypatch, tmp_path, cause):
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path))
    if cause == "no_compiler":
        monkeypatch.setattr(build.shutil, "which", lambda c: None)
    elif cause == "broken_source":
        (tmp_path / "bad.cpp").write_text("not C++\n")
        monkeypatch.setattr(build, "TENSOR_SOURCE", str(tmp_path / "bad.cpp"))
    else:
        with open(build.tensor_reader(), "w") as f:
            f.write("not a shared object")
    with pytest.warns(RuntimeWarning, match="their attributes are read"):
        assert build.load_tensor_reader() == 0


def test_the_reader_of_another_torch_is_not_loaded(monkeypatch):
    here = build.tensor_reader()
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "1.0.0+other")
    assert build.tensor_reader() != here and "1_0_0_other" in build.tensor_reader()


def test_the_extension_takes_an_address_or_none():
    kvs.lib()
    if kvs._ops is None:
        pytest.skip("no extension")
    for wrong in ((), (None,), (-1,), (1.0,), (0, 0)):
        with pytest.raises(TypeError):
            kvs._ops.use_reader(*wrong)


def test_calls_pass_on_the_same_with_and_without_it():
    kvs.lib()
    if kvs._ops is None:
        pytest.skip("no extension")
    P = ctypes.c_void_p
    seen = []

    @ctypes.CFUNCTYPE(ctypes.c_int, P, P, P, ctypes.c_int32, P, ctypes.c_int32, P, ctypes.c_uint32)
    def called(geom, cache, step, layer, args, sinks, stream, flags):
        seen.append((ctypes.string_at(args, ctypes.sizeof(kvs.kvs_attend_args)), layer, sinks, flags))
        return 0

    planes = [torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2)]
    step = kvs.Step((1, 2, 64, 2, 16, 256), planes, 4, torch.zeros(3, 4, dtype=torch.int32), torch.ones(3, dtype=torch.int32))
    q = torch.zeros(8, 3, 64, dtype=torch.bfloat16).transpose(0, 1)
    out, lse, work = torch.zeros(3, 8, 64, dtype=torch.bfloat16), torch.zeros(3, 8), torch.zeros(100, dtype=torch.uint8)
    address = kvs._reader
    try:
        for reader in (_address(), 0):
            kvs._ops.use_reader(reader)
            assert kvs._ops.attend_sinks(ctypes.cast(called, P).value, *step.ext, 0, None, 0, q, out, lse, 0.125, True, 100, 4, work, step.byte) == 0
            for wrong in (q.float(), q[:, :7], q[:2], None, 3, q.unsqueeze(0)):
                assert kvs._ops.attend_sinks(ctypes.cast(called, P).value, *step.ext, 0, None, 0, wrong, out, lse, 0.125, True, 100, 4, work,
                                             step.byte) is None
    finally:
        kvs._ops.use_reader(address or 0)
    assert len(seen) == 2 and seen[0] == seen[1]
    a = kvs.kvs_attend_args.from_buffer_copy(seen[0][0])
    assert (a.q.row_stride, a.q.head_stride, a.num_q_heads, a.workspace_bytes) == (64, 192, 8, 100)
