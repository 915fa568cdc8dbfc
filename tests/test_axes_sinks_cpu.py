"""The operators with axes and with sinks without a GPU: what is refused, the tables of axes, what the
extension hands over, and the C entries over stand-ins."""
import ctypes

import numpy as np
import pytest

from paper_2609_35065_gb300 import kvs
from test_ops_cpu import ALL, LAYER, ROWS, A, B_, Call, I, U, X, _fields, _spoil, _step, _Stream
from test_ops_host_cpu import library  # noqa: F401  (a fixture)

OPS = ["append_axes", "attend_sinks", "weigh_sinks"]


class LongCall(Call):
    """A valid call of each, whose fields a test then spoils."""

    def __init__(self):
        super().__init__()
        self.axes = kvs.kvs_axes(X, 8, 3, 32)
        self.sinks = 4
        self.attend.window = self.weigh.window = 20

    def run(self, op, lib=None):
        b = ctypes.byref
        base = op.split("_")[0]
        more = b(self.axes) if op == "append_axes" else ctypes.c_int32(self.sinks)
        return getattr(lib or kvs.lib(), "kvs_" + op)(b(self.geom), b(self.cache), b(self.step), self.layer, b(getattr(self, base)), more, None,
                                                      ctypes.c_uint32(self.flags))


def _cases(op, own):
    base = op.split("_")[0]
    return [(op, *c) for c in ALL + LAYER] + [(op, f"{base}.{p}", v, e) for p, v, e in ROWS + own]


CASES = (
    _cases("append_axes", [("q_out.base", None, I), ("q_out.head_stride", 0, A), ("k.base", None, I), ("v.base", X + 8, U), ("num_q_heads", 3, I),
                           ("positions", None, I), ("rope", None, I)])
    + [("append_axes", "rope.rot_dim", 66, I), ("append_axes", "rope.rot_dim", 32, I), ("append_axes", "rope.turns", None, I), ("append_axes", "axes.axis", None, I),
       ("append_axes", "axes.num_axes", 0, I), ("append_axes", "axes.num_axes", 5, I), ("append_axes", "axes.stride", 7, I), ("append_axes", "axes.stride", -1, I),
       ("append_axes", "axes.pairs", 31, I), ("append_axes", "axes.pairs", -32, I)]
    + _cases("attend_sinks", [("out.base", None, I), ("out.row_stride", 0, A), ("num_q_heads", 5, I), ("scale", float("nan"), I), ("window", -1, I)])
    + _cases("weigh_sinks", [("lse", None, I), ("weights", None, I), ("head_stride", 63, A), ("request_stride", -1, I), ("decay", float("inf"), I), ("window", -3, I)])
    + [(op, "sinks", s, I) for op in OPS[1:] for s in (-1, -2 ** 31)]
    + [(op, "step.max_kv", (1 << 30) + 1, U) for op in OPS])


@pytest.mark.parametrize("op,path,value,code", CASES, ids=[f"{o}-{p}-{v}" for o, p, v, _ in CASES])
def test_refusals(op, path, value, code):
    c = LongCall()
    _spoil(path, value)(c)
    assert c.run(op) == code, kvs.kvs_last_error()
    assert kvs.kvs_last_error() != ""


@pytest.mark.parametrize("op", OPS)
def test_null_structs(op):
    c = LongCall()
    b = ctypes.byref
    good = [b(c.geom), b(c.cache), b(c.step), 1, b(getattr(c, op.split("_")[0])), b(c.axes) if op == "append_axes" else 4]
    for k in (0, 1, 2, 4) + ((5,) if op == "append_axes" else ()):
        assert getattr(kvs.lib(), "kvs_" + op)(*[None if i == k else x for i, x in enumerate(good)], None, 0) == I


@pytest.mark.parametrize("op", OPS)
def test_an_empty_batch_needs_no_device(op):
    c = LongCall()
    c.step.num_requests, c.step.kv_lens, c.step.block_tables, c.append.positions = 0, None, None, None
    assert c.run(op) == kvs.KVS_OK, kvs.kvs_last_error()


@pytest.mark.parametrize("window,sinks", [(-1, 4), (5, -1)])
def test_a_workspace_of_no_mask_is_refused(window, sinks):
    c = LongCall()
    assert kvs.lib().kvs_attend_sinks_workspace(ctypes.byref(c.geom), ctypes.byref(c.step), 4, 1, window, sinks) == I


def test_struct_sizes():
    assert ctypes.sizeof(kvs.kvs_axes) == 24


@pytest.mark.parametrize("op", OPS)
def test_a_valid_call_is_launched_and_counted(library, op):  # noqa: F811
    before, counted = library.fake_ops(), library.kvs_stat_launches()
    assert LongCall().run(op, library) == kvs.KVS_OK, library.kvs_last_error()
    assert library.fake_ops() == before + 1 and library.kvs_stat_launches() == counted + 1


# ---- tables -------------------------------------------------------------------
def test_axes_in_blocks_and_in_turn():
    turns, axis, scale = kvs.kvs_rope_axes([16, 24, 24], 500000.0)
    assert scale == 1.0 and (axis == np.repeat([0, 1, 2], [16, 24, 24])).all()
    assert (turns == kvs.kvs_rope_turns(128, 500000.0)[0]).all()
    turns, axis, _ = kvs.kvs_rope_axes([24, 20, 20], cycle=True)
    want = np.zeros(64, int)
    want[1:60:3], want[2:60:3] = 1, 2
    assert (axis == want).all() and (turns == kvs.kvs_rope_turns(128)[0]).all()
    assert (np.bincount(axis) == [24, 20, 20]).all()


@pytest.mark.parametrize("cycle", [False, True])
def test_frequencies_that_begin_anew(cycle):
    parts = [10, 6, 4]
    turns, axis, scale = kvs.kvs_rope_axes(parts, kind=kvs.KVS_ROPE_YARN, factor=4.0, context=4096, low=1.0, high=32.0, cycle=cycle, restart=True)
    for a, n in enumerate(parts):
        want, s = kvs.kvs_rope_turns(2 * n, kind=kvs.KVS_ROPE_YARN, factor=4.0, context=4096, low=1.0, high=32.0)
        assert (turns[axis == a] == want).all() and s == scale


@pytest.mark.parametrize("kw", [dict(parts=[]), dict(parts=[4] * 5), dict(parts=[4, 0]), dict(parts=[4, -1, 5]), dict(parts=[1, 5], cycle=True), dict(parts=[2, 2, 3], cycle=True),
                                dict(parts=[4, 4], base=1.0), dict(parts=[4, 1], kind=kvs.KVS_ROPE_NTK, factor=2.0, restart=True)])
def test_tables_refused(kw):
    with pytest.raises(kvs.KvsError) as ei:
        kvs.kvs_rope_axes(**kw)
    assert ei.value.code == I


def test_tables_refused_by_the_c_entry():
    spec = kvs.kvs_rope_spec(16, 0, 10000.0, 1.0, 0.0, 0.0, 0.0)
    parts, turns, axis, scale = (ctypes.c_int32 * 2)(4, 4), np.zeros((8, 2), np.float32), np.zeros(8, np.uint8), ctypes.c_float()
    good = [ctypes.byref(spec), parts, 2, 0, turns.ctypes.data, axis.ctypes.data, ctypes.byref(scale)]
    f = kvs.lib().kvs_rope_axes
    assert f(*good) == kvs.KVS_OK
    for k in (0, 1, 4, 5, 6):
        assert f(*[None if i == k else x for i, x in enumerate(good)]) == I
    assert f(*good[:3], 4, *good[4:]) == I and f(*good[:3], -1, *good[4:]) == I
    spec.rot_dim = 14
    assert f(*good) == I


# ---- the binding ----------------------------------------------------------------
def test_binding_refuses_what_the_structs_cannot_say():
    import torch
    s = _step()
    q, f = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4)
    u8, i32 = torch.zeros(32, dtype=torch.uint8), torch.int32
    for bad in (u8.int(), u8.view(4, 8), torch.zeros(64, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            kvs.Axes(bad, 3)
    axes, rope, pos = kvs.Axes(u8, 3), kvs.Rope(torch.zeros(32, 2), 64), torch.zeros(3, 2, dtype=i32)
    for call in (lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, axes, pos[:2]),
                 lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, axes, pos[:, :1]),
                 lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, axes, pos.long()),
                 lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, axes, pos[0]),
                 lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, axes, torch.zeros(2, 3, dtype=i32).T),
                 lambda: kvs.kvs_append_axes(s, 0, None, q, q, None, rope, axes, pos),
                 lambda: kvs.kvs_attend_sinks(s, 0, q.half(), q), lambda: kvs.kvs_attend_sinks(s, 0, q, q[:, :2]), lambda: kvs.kvs_attend_sinks(s, 0, q, q.clone(), f[:1]),
                 lambda: kvs.kvs_attend_sinks(s, 0, q, q.clone(), workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20)),
                 lambda: kvs.kvs_weigh_sinks(s, 0, q, f, torch.zeros(2, 2, 63)), lambda: kvs.kvs_weigh_sinks(s, 0, q, f[:1], torch.zeros(2, 2, 64))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, None, axes, pos),
                 lambda: kvs.kvs_append_axes(s, 0, q, q[:, :2], q[:, :2], None, rope, kvs.Axes(u8[:16], 3), pos),
                 lambda: kvs.kvs_attend_sinks(s, 0, q, q.clone(), sinks=-1, window=4), lambda: kvs.kvs_weigh_sinks(s, 0, q, f, torch.zeros(2, 2, 64), sinks=-1),
                 lambda: kvs.kvs_attend_sinks_workspace(s, 3)):
        with pytest.raises(kvs.KvsError) as ei:
            call()
        assert ei.value.code == I


def _recorder(struct, axes, seen):
    sig = [ctypes.c_void_p] * 3 + [ctypes.c_int32, ctypes.POINTER(struct), ctypes.POINTER(kvs.kvs_axes) if axes else ctypes.c_int32, ctypes.c_void_p, ctypes.c_uint32]

    @ctypes.CFUNCTYPE(ctypes.c_int, *sig)
    def fn(*a):
        seen.append((a[:4], _fields(a[4].contents), _fields(a[5].contents) if axes else a[5], a[6:]))
        return 0
    return fn


def test_the_extension_hands_over_what_the_binding_would(monkeypatch):
    import torch
    if kvs.lib() is None or kvs._ops is None:
        pytest.skip("no extension")
    seen, keep, library_ = [], [], kvs.lib()

    class Library:
        def __getattr__(self, name):
            return getattr(library_, name)

    fake = Library()
    for name, struct in (("kvs_append_axes", kvs.kvs_append_args), ("kvs_attend_sinks", kvs.kvs_attend_args), ("kvs_weigh_sinks", kvs.kvs_weigh_args)):
        fn = _recorder(struct, name == "kvs_append_axes", seen)
        keep.append(fn)
        setattr(fake, name, fn)
        monkeypatch.setitem(kvs._address, name, ctypes.cast(fn, ctypes.c_void_p).value)
    step = _step(geom=(2, 2, 64, 2, 16, 256), planes=[X] * 4)
    qkv = torch.zeros(2, 8 * 64, dtype=torch.bfloat16)
    q, k, v = qkv[:, :256].view(2, 4, 64), qkv[:, 256:384].view(2, 2, 64), qkv[:, 384:].view(2, 2, 64)
    out, lse, w = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4), torch.zeros(3, 2, 2, 80)[1]
    rope, axes = kvs.Rope(torch.zeros(16, 2), 32, True, 0.5), kvs.Axes(torch.zeros(16, dtype=torch.uint8), 3)
    pos, ws = torch.zeros(3, 5, dtype=torch.int32)[:, 1:3], torch.zeros(99, dtype=torch.uint8)
    calls = [lambda: kvs.kvs_append_axes(step, 1, q, k, v, out, rope, axes, pos, _Stream(), 1), lambda: kvs.kvs_append_axes(step, 0, None, k, v, None, rope, axes, pos),
             lambda: kvs.kvs_append_axes(step, 0, out, k, v, None, rope, axes, pos, 8),
             lambda: kvs.kvs_attend_sinks(step, 1, q, out, lse, 0.25, False, 7, 3, ws, _Stream(), 1), lambda: kvs.kvs_attend_sinks(step, 0, q, out),
             lambda: kvs.kvs_weigh_sinks(step, 1, q, lse, w, 0.5, 0.25, True, 3, 9, _Stream()), lambda: kvs.kvs_weigh_sinks(step, 0, q, lse, w)]
    ops = kvs._ops
    for call in calls:
        monkeypatch.setattr(kvs, "_ops", ops)
        n = len(seen)
        call()
        assert len(seen) == n + 1
        monkeypatch.setattr(kvs, "_ops", None)
        monkeypatch.setattr(kvs, "_lib", fake)
        call()
        monkeypatch.setattr(kvs, "_lib", library_)
        by_ext, by_binding = seen[n:]
        assert by_ext == by_binding


def test_the_extension_leaves_what_is_not_plain_to_the_binding():
    import torch
    if kvs.lib() is None or kvs._ops is None:
        pytest.skip("no extension")
    s, q, f = _step(), torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4)
    k = q[:, :2]
    rope, axes, pos = kvs.Rope(torch.zeros(32, 2), 64), kvs.Axes(torch.zeros(32, dtype=torch.uint8), 3), torch.zeros(3, 2, dtype=torch.int32)
    a = (kvs._address["kvs_append_axes"], *s.ext, 0, None, 0)
    for args in ((q, k, k, None, None, axes, pos), (q, k, k, None, rope, None, pos), (q, k, k, None, rope, axes, None), (q, k, k, None, rope, axes, pos[:2]),
                 (q, k, k, None, rope, axes, pos.T), (q.half(), k, k, None, rope, axes, pos), (q, q, k, None, rope, axes, pos), (q, k, k, None, 3, axes, pos)):
        assert kvs._ops.append_axes(*a, *args) is None
    a = (kvs._address["kvs_attend_sinks"], *s.ext, 0, None, 0)
    for args in ((q, q, f, 0.1, True, 0, 1 << 40, None), (q, q, f, 0.1, True, 0, 1.0, None), (q, q, f, 0.1, True, 0, 0, f), (q, q[:1], f, 0.1, True, 0, 0, None)):
        assert kvs._ops.attend_sinks(*a, *args, torch.uint8) is None
    w = torch.zeros(2, 2, 64)
    a = (kvs._address["kvs_weigh_sinks"], *s.ext, 0, None, 0)
    for args in ((q, f, w, 0.1, 1.0, True, 0, None), (q, f, w, 0.1, 1, True, 0, 0), (q, f, w[..., :63], 0.1, 1.0, True, 0, 0)):
        assert kvs._ops.weigh_sinks(*a, *args) is None
    for f in (kvs._ops.append_axes, kvs._ops.attend_sinks, kvs._ops.weigh_sinks):
        with pytest.raises(TypeError):
            f(*a, q)
