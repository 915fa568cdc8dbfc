"""The model operators' host side without a GPU: what is refused, and the rotary tables."""
import ctypes

import numpy as np
import pytest

from paper_2609_35065_gb300 import kvs

I, B_, A, U = kvs.KVS_ERR_INVALID_ARG, kvs.KVS_ERR_BOUNDS, kvs.KVS_ERR_ALIAS, kvs.KVS_ERR_UNSUPPORTED
X = 1 << 20                              # an aligned address; nothing is followed before the checks are through


class Call:
    """The C structs of one valid call, whose fields a test then spoils."""

    def __init__(self):
        self.geom = kvs.kvs_geometry(2, 2, 64, 2, 16, 256)
        self.planes = (ctypes.c_void_p * 4)(X, X, X, X)
        self.cache = kvs.kvs_paged_cache(ctypes.cast(self.planes, ctypes.POINTER(ctypes.c_void_p)), 10)
        self.step = kvs.kvs_step(X, X, X, 2, 4, 8, 5, 64, kvs.KVS_DTYPE_BF16)
        self.layer, self.flags = 1, 0
        rows = lambda heads: kvs.kvs_rows(X, heads * 64, 64)  # noqa: E731
        self.rope = kvs.kvs_rope(X, 64, 0, 1.0, 0)
        self.append = kvs.kvs_append_args(rows(4), rows(4), rows(2), rows(2), X, ctypes.addressof(self.rope), 4, 0)
        self.attend = kvs.kvs_attend_args(rows(4), rows(4), X, X, 1 << 30, 0.125, 1, 0, 4)
        self.weigh = kvs.kvs_weigh_args(rows(4), X, X, 128, 64, 0.125, 1.0, 1, 0, 4, 0)
        self.evict = kvs.kvs_evict_args(X, 256, 128, 64, 2 * X, 2, 32, 4, 8, X, 2 * X, 3 * X)

    def run(self, op):
        b = ctypes.byref
        args = [b(self.geom), b(self.cache), b(self.step)] + ([] if op == "evict" else [self.layer]) + [b(getattr(self, op))]
        return getattr(kvs.lib(), "kvs_" + op)(*args, None, self.flags)


def _spoil(path, value):
    def f(c):
        o = c
        *parts, last = path.split(".")
        for p in parts:
            o = getattr(o, p)
        if last.isdigit():
            o[int(last)] = value
        else:
            setattr(o, last, value)
    return f


ALL = [("geom.num_layers", 0, I), ("geom.num_kv_heads", -1, I), ("geom.head_dim", 0, I), ("geom.head_dim", 60, U), ("geom.head_dim", 136, U),
       ("geom.elem_bytes", 1, U), ("geom.elem_bytes", 4, U), ("geom.block_size", 0, I), ("step.dtype", 0, I), ("step.dtype", 3, I),
       ("step.num_requests", -1, I), ("step.num_requests", 65536, U), ("step.total_q", -1, I), ("step.max_q", -2, I), ("step.max_q", 9, I),
       ("step.max_kv", -1, I), ("step.max_kv", 65, B_), ("step.table_stride", 3, B_), ("step.kv_lens", None, I), ("step.block_tables", None, I),
       ("step.q_starts", None, I), ("cache.num_blocks", 0, I), ("cache.num_blocks", 1 << 31, I), ("flags", kvs.KVS_F_FORCE_LDG, I)]
LAYER = [("layer", -1, I), ("layer", 2, I), ("planes.2", None, I), ("planes.2", X + 8, U)]
ROWS = [("q.base", X + 2, U), ("q.row_stride", 257, U), ("q.head_stride", -64, I)]


def _cases(op, own, layer=True):
    return [(op, *c) for c in ALL + (LAYER if layer else [("planes.3", None, I), ("planes.0", X + 4, U)])] + [(op, f"{op}.{p}", v, e) for p, v, e in own]


CASES = (
    _cases("append", ROWS + [("q_out.base", None, I), ("q_out.head_stride", 0, A), ("q_out.row_stride", 64, A), ("q_out.row_stride", 512, A),
                             ("k.base", None, I), ("v.base", None, I), ("v.base", X + 8, U), ("num_q_heads", 3, I), ("num_q_heads", 0, I)])
    + [("append", "rope.rot_dim", 0, I), ("append", "rope.rot_dim", 7, I), ("append", "rope.rot_dim", 66, I), ("append", "rope.turns", None, I),
       ("append", "rope.turns", X + 4, U), ("append", "rope.scale", float("nan"), I)]
    + _cases("attend", ROWS + [("out.base", None, I), ("out.head_stride", 32, A), ("out.row_stride", 0, A), ("num_q_heads", 5, I),
                               ("scale", float("inf"), I), ("window", -1, I)])
    + _cases("weigh", ROWS + [("lse", None, I), ("weights", None, I), ("head_stride", 63, A), ("request_stride", 100, A), ("request_stride", -1, I),
                              ("num_q_heads", 5, I), ("scale", float("nan"), I), ("decay", float("inf"), I), ("window", -3, I)])
    + _cases("evict", [("budget", 0, I), ("sinks", -1, I), ("recent", 29, I), ("recent", -1, I), ("weights", None, I), ("kept", None, I),
                       ("dst_tables", None, I), ("dst_tables", X, A), ("dst_stride", 1, B_), ("new_lens", X, A), ("new_weights", X, A),
                       ("layer_stride", -1, I)], layer=False))


@pytest.mark.parametrize("op,path,value,code", CASES, ids=[f"{o}-{p}-{v}" for o, p, v, _ in CASES])
def test_refusals(op, path, value, code):
    c = Call()
    _spoil(path, value)(c)
    assert c.run(op) == code, kvs.kvs_last_error()
    assert kvs.kvs_last_error() != ""


@pytest.mark.parametrize("op", ["append", "attend", "weigh", "evict"])
def test_null_structs(op):
    fn = getattr(kvs.lib(), "kvs_" + op)
    c = Call()
    b = ctypes.byref
    layer = [] if op == "evict" else [1]
    good = [b(c.geom), b(c.cache), b(c.step)] + layer + [b(getattr(c, op))]
    for k in (0, 1, 2, len(good) - 1):
        assert fn(*[None if i == k else x for i, x in enumerate(good)], None, 0) == I


@pytest.mark.parametrize("op", ["append", "attend", "weigh", "evict"])
def test_a_step_without_requests_needs_no_device(op):
    c = Call()
    c.step.num_requests = c.step.total_q = c.step.max_q = c.step.max_kv = 0
    assert c.run(op) == kvs.KVS_OK


def test_struct_sizes():
    assert [ctypes.sizeof(s) for s in (kvs.kvs_step, kvs.kvs_rows, kvs.kvs_rope, kvs.kvs_rope_spec, kvs.kvs_append_args, kvs.kvs_attend_args,
                                       kvs.kvs_weigh_args, kvs.kvs_evict_args)] == [48, 24, 24, 48, 120, 88, 80, 80]


# ---- rotary tables ----------------------------------------------------------
def _radians(turns):
    return turns.astype(np.float64).sum(1) * 2 * np.pi


def test_plain_linear_and_ntk_tables():
    j = np.arange(32)
    plain = 10000.0 ** (-2 * j / 64)
    t, s = kvs.kvs_rope_turns(64, 10000.0)
    assert s == 1.0 and np.allclose(_radians(t), plain, rtol=1e-14, atol=0)
    t, s = kvs.kvs_rope_turns(64, 10000.0, kvs.KVS_ROPE_LINEAR, 4.0)
    assert s == 1.0 and np.allclose(_radians(t), plain / 4, rtol=1e-14, atol=0)
    t, _ = kvs.kvs_rope_turns(64, 10000.0, kvs.KVS_ROPE_NTK, 4.0)
    f = _radians(t)
    assert np.allclose(f, (10000.0 * 4 ** (64 / 62)) ** (-2 * j / 64), rtol=1e-14, atol=0)
    assert np.isclose(f[-1], plain[-1] / 4)                      # the slowest pair is slowed by the whole factor


def test_banded_table():
    t, s = kvs.kvs_rope_turns(128, 500000.0, kvs.KVS_ROPE_BANDS, 8.0, 8192, 1.0, 4.0)
    plain = 500000.0 ** (-2 * np.arange(64) / 128)
    wave = 2 * np.pi / plain
    f = _radians(t)
    assert s == 1.0
    assert np.allclose(f[wave < 8192 / 4], plain[wave < 8192 / 4]) and np.allclose(f[wave > 8192], plain[wave > 8192] / 8)
    mid = (wave >= 8192 / 4) & (wave <= 8192)
    mean = (8192 / wave[mid] - 1.0) / 3.0
    assert mid.any() and np.allclose(f[mid], (1 - mean) * plain[mid] / 8 + mean * plain[mid])


def test_yarn_table():
    t, s = kvs.kvs_rope_turns(128, 10000.0, kvs.KVS_ROPE_YARN, 4.0, 4096, 1.0, 32.0)
    plain = 10000.0 ** (-2 * np.arange(64) / 128)
    f, times = _radians(t), 4096 * plain / (2 * np.pi)            # turns of each pair within the context
    assert np.isclose(s, 0.1 * np.log(4.0) + 1.0)
    assert np.allclose(f[times > 40], plain[times > 40]) and np.allclose(f[times < 0.8], plain[times < 0.8] / 4)
    assert (np.diff(f) < 0).all() and (f <= plain * (1 + 1e-12)).all() and (f >= plain / 4 * (1 - 1e-12)).all()


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=64, base=1.0), dict(rot_dim=64, kind=9), dict(rot_dim=64, base=float("nan")),
                                dict(rot_dim=64, kind=kvs.KVS_ROPE_LINEAR, factor=0.5), dict(rot_dim=2, kind=kvs.KVS_ROPE_NTK, factor=2.0),
                                dict(rot_dim=64, kind=kvs.KVS_ROPE_BANDS, factor=2.0, context=0, low=1, high=4),
                                dict(rot_dim=64, kind=kvs.KVS_ROPE_YARN, factor=2.0, context=4096, low=4, high=4)])
def test_tables_refused(kw):
    with pytest.raises(kvs.KvsError) as ei:
        kvs.kvs_rope_turns(**kw)
    assert ei.value.code == I


# ---- the binding's own checks -----------------------------------------------
def _step(**kw):
    import torch
    a = dict(geom=(1, 2, 64, 2, 16, 256), planes=[X, X], num_blocks=4, block_tables=torch.zeros(2, 4, dtype=torch.int32),
             kv_lens=torch.zeros(2, dtype=torch.int32))
    a.update(kw)
    return kvs.Step(**a)


def test_binding_refuses_what_the_structs_cannot_say():
    import torch
    i32 = torch.int32
    for kw in (dict(block_tables=torch.zeros(2, 4)), dict(kv_lens=torch.zeros(3, dtype=i32)), dict(kv_lens=torch.zeros(2, dtype=torch.int64)),
               dict(planes=[X]), dict(q_starts=torch.zeros(2, dtype=i32), total_q=2, max_q=1), dict(q_starts=torch.zeros(3, dtype=i32)),
               dict(block_tables=torch.zeros(4, 2, dtype=i32).T), dict(block_tables=torch.zeros(1, 4, dtype=i32).expand(2, 4))):
        with pytest.raises(ValueError):
            _step(**kw)
    with pytest.raises(kvs.KvsError):
        _step(max_kv=65)
    s = _step()
    q, f = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4)
    for call in (lambda: kvs.kvs_attend(s, 0, q.half(), q), lambda: kvs.kvs_attend(s, 0, q[:1], q[:1]), lambda: kvs.kvs_attend(s, 0, q, q[:, :2]),
                 lambda: kvs.kvs_attend(s, 0, q[..., :32], q), lambda: kvs.kvs_attend(s, 0, torch.zeros(2, 4, 128, dtype=q.dtype)[..., ::2], q),
                 lambda: kvs.kvs_attend(s, 0, q, q.clone(), f[:1]), lambda: kvs.kvs_attend(s, 0, q, q.clone(), f.half()),
                 lambda: kvs.kvs_weigh(s, 0, q, f, torch.zeros(2, 2, 63)), lambda: kvs.kvs_weigh(s, 0, q, f, torch.zeros(2, 2, 128)[..., ::2]),
                 lambda: kvs.kvs_append(s, 0, None, q, q), lambda: kvs.kvs_append(s, 0, None, q[:, :2], q[:, :2], positions=torch.zeros(1, dtype=i32)),
                 lambda: kvs.kvs_evict(s, torch.zeros(1, 2, 2, 64), torch.zeros(2, 4, dtype=i32), 8, 0, 0, torch.zeros(1, 2, 2, 9, dtype=i32)),
                 lambda: kvs.kvs_evict(s, torch.zeros(1, 2, 2, 64), torch.zeros(3, 4, dtype=i32), 8, 0, 0, torch.zeros(1, 2, 2, 8, dtype=i32))):
        with pytest.raises(ValueError):
            call()


# ---- the extension against the binding's own marshalling --------------------
def _fields(s):
    return {n: (_fields(getattr(s, n)) if isinstance(getattr(s, n), ctypes.Structure) else getattr(s, n)) for n, _ in s._fields_}


def _recorder(struct, layer, seen):
    sig = [ctypes.c_void_p] * 3 + ([ctypes.c_int32] if layer else []) + [ctypes.POINTER(struct), ctypes.c_void_p, ctypes.c_uint32]

    @ctypes.CFUNCTYPE(ctypes.c_int, *sig)
    def fn(*a):
        args = a[4 if layer else 3]
        seen.append((a[:3], a[3] if layer else None, _fields(args.contents), a[-2], a[-1]))
        return 0
    return fn


class _Stream:
    cuda_stream = 4096


def test_the_extension_hands_over_what_the_binding_would(monkeypatch):
    import torch
    if kvs.lib() is None or kvs._ops is None:
        pytest.skip("no extension")
    seen, keep, library = [], [], kvs.lib()

    class Library:
        def __getattr__(self, name):
            return getattr(library, name)

    fake = Library()
    for name, struct in (("kvs_append", kvs.kvs_append_args), ("kvs_attend", kvs.kvs_attend_args), ("kvs_weigh", kvs.kvs_weigh_args),
                         ("kvs_evict", kvs.kvs_evict_args)):
        fn = _recorder(struct, name != "kvs_evict", seen)
        keep.append(fn)
        setattr(fake, name, fn)
        monkeypatch.setitem(kvs._address, name, ctypes.cast(fn, ctypes.c_void_p).value)
    i32 = torch.int32
    step = _step(geom=(2, 2, 64, 2, 16, 256), planes=[X] * 4)
    qkv = torch.zeros(2, 8 * 64, dtype=torch.bfloat16)
    q, k, v = qkv[:, :256].view(2, 4, 64), qkv[:, 256:384].view(2, 2, 64), qkv[:, 384:].view(2, 2, 64)
    out, lse, w = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4), torch.zeros(3, 2, 2, 80)[1]
    rope, pos, ws = kvs.Rope(torch.zeros(16, 2), 32, True, 0.5), torch.zeros(2, dtype=i32), torch.zeros(99, dtype=torch.uint8)
    allw, dst, kept, nw, nl = torch.zeros(2, 2, 2, 70)[..., 1:], torch.zeros(2, 3, dtype=i32)[:, :2], torch.zeros(2, 2, 2, 20, dtype=i32), torch.zeros(2, 2, 2, 20), pos
    calls = [lambda: kvs.kvs_append(step, 1, q, k, v, out, rope, pos, _Stream(), 1), lambda: kvs.kvs_append(step, 0, None, k, v),
             lambda: kvs.kvs_append(step, 0, out, k, v, None, None, None, 8),
             lambda: kvs.kvs_attend(step, 1, q, out, lse, 0.25, False, 7, ws, _Stream(), 1), lambda: kvs.kvs_attend(step, 0, q, out),
             lambda: kvs.kvs_weigh(step, 1, q, lse, w, 0.5, 0.25, True, 3, _Stream()), lambda: kvs.kvs_weigh(step, 0, q, lse, w),
             lambda: kvs.kvs_evict(step, allw, dst, 20, 3, 4, kept, nw, nl, _Stream(), 1), lambda: kvs.kvs_evict(step, allw, dst, 20, 0, 0, kept)]
    ops = kvs._ops
    for call in calls:
        monkeypatch.setattr(kvs, "_ops", ops)
        n = len(seen)
        call()
        assert len(seen) == n + 1
        monkeypatch.setattr(kvs, "_ops", None)
        monkeypatch.setattr(kvs, "_lib", fake)
        call()
        monkeypatch.setattr(kvs, "_lib", library)
        by_ext, by_binding = seen[n:]
        assert by_ext[1:] == by_binding[1:]
        assert by_ext[0] == by_binding[0]


def test_the_extension_leaves_what_is_not_plain_to_the_binding():
    import torch
    if kvs.lib() is None or kvs._ops is None:
        pytest.skip("no extension")
    s, q, f = _step(), torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4)
    a = (kvs._address["kvs_attend"], *s.ext, 0, None, 0)
    for args in ((q.half(), q, f, 0.1, True, 0, None), (q[:1], q, f, 0.1, True, 0, None), (q, q[:, :2], f, 0.1, True, 0, None), (q, q, f[:, :2], 0.1, True, 0, None),
                 (q, q, f, 1, True, 0, None), (q, q, f, 0.1, 1, 0, None), (q, q, f, 0.1, True, 1 << 40, None), (q, q, f, 0.1, True, 0, f),
                 (None, q, f, 0.1, True, 0, None), (q, 3, f, 0.1, True, 0, None), (torch.zeros(2, 4, 128, dtype=q.dtype)[..., ::2], q, f, 0.1, True, 0, None)):
        assert kvs._ops.attend(*a, *args, torch.uint8) is None
    with pytest.raises(TypeError):
        kvs._ops.attend(*a, q, q)


@pytest.mark.parametrize("op,path,value", [(o, "step.max_kv", (1 << 30) + 1) for o in ("append", "attend", "weigh", "evict")] + [("evict", "evict.budget", (1 << 30) + 1)])
def test_positions_above_30_bits_are_refused(op, path, value):
    test_refusals(op, path, value, U)


@pytest.mark.parametrize("op", ["append", "attend", "weigh", "evict"])
def test_rows_without_a_request_need_no_device(op):
    """An empty batch in tensors padded to a fixed number of rows: no array of the step has an entry to read."""
    c = Call()
    c.step.num_requests, c.step.kv_lens, c.step.block_tables = 0, None, None
    assert c.run(op) == kvs.KVS_OK, kvs.kvs_last_error()


@pytest.mark.parametrize("spread", [lambda t: t.expand(1 << 20), lambda t: t.expand(64, 1 << 10), lambda t: t.new_zeros(2 << 20)[::2]])
def test_a_workspace_with_fewer_bytes_than_entries_is_refused(spread):
    """An expanded or strided tensor does not have numel() bytes behind its address."""
    import torch
    s = _step()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="workspace"):
        kvs.kvs_attend(s, 0, q, q.clone(), workspace=spread(torch.zeros(1, dtype=torch.uint8)))
