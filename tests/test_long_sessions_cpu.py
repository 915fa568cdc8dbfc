"""The operators with axes and with sinks without a GPU: numbers that no 32-bit field holds, and where a session's text goes on."""
import ctypes

import pytest

from paper_2609_35065_gb300 import kvs
from test_ops_cpu import _fields, _step

MOST = 2 ** 31 - 1


class _Library:
    """The library with recorders in the operators' place."""

    def __init__(self, seen):
        self.real, self.seen = kvs.lib(), seen

    def __getattr__(self, name):
        if name in ("kvs_attend", "kvs_attend_sinks", "kvs_weigh", "kvs_weigh_sinks", "kvs_append", "kvs_append_axes"):
            def call(g, c, s, layer, args, *more):
                self.seen.append((ctypes.c_int32(layer).value, _fields(args._obj), more))
                return 0
            return call
        if name == "kvs_attend_sinks_workspace":
            return lambda g, s, heads, causal, window, sinks: self.seen.append(tuple(ctypes.c_int32(x).value for x in (heads, window, sinks))) or 0
        return getattr(self.real, name)


@pytest.fixture
def seen(monkeypatch):
    calls = []
    fake = _Library(calls)
    monkeypatch.setattr(kvs, "_lib", fake)
    return calls


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 5, 2 ** 40])
def test_numbers_beyond_32_bits_keep_their_meaning(seen, big):
    """A window or a number of sinks that no 32-bit field holds is not cut to its low bits: it is the largest."""
    import torch
    s, q, f, w = _step(), torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4), torch.zeros(2, 2, 64)
    kvs.kvs_attend(s, 0, q, q.clone(), window=big)
    kvs.kvs_attend_sinks(s, 0, q, q.clone(), window=big, sinks=big + 1)
    kvs.kvs_weigh(s, 0, q, f, w, window=big)
    kvs.kvs_weigh_sinks(s, 0, q, f, w, window=big, sinks=big + 1)
    assert len(seen) == 4
    for layer, a, more in seen:
        assert layer == 0 and a["window"] == MOST
    for k in (1, 3):
        assert ctypes.c_int32(seen[k][2][0]).value == MOST
    kvs.kvs_attend_sinks_workspace(s, 4, True, big, big + 1)
    assert seen[4] == (4, MOST, MOST)


@pytest.mark.parametrize("big", [2 ** 32, 2 ** 33 + 1, -2 ** 32])
def test_a_layer_beyond_32_bits_is_refused(big):
    import torch
    s, q, f, w = _step(), torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 4), torch.zeros(2, 2, 64)
    k = q[:, :2]
    rope, axes, pos = kvs.Rope(torch.zeros(32, 2), 64), kvs.Axes(torch.zeros(32, dtype=torch.uint8), 3), torch.zeros(3, 2, dtype=torch.int32)
    for call in (lambda: kvs.kvs_attend(s, big, q, q.clone()), lambda: kvs.kvs_attend_sinks(s, big, q, q.clone()), lambda: kvs.kvs_weigh(s, big, q, f, w),
                 lambda: kvs.kvs_weigh_sinks(s, big, q, f, w), lambda: kvs.kvs_append(s, big, q, k, k), lambda: kvs.kvs_append_axes(s, big, q, k, k, None, rope, axes, pos),
                 lambda: kvs.kvs_attend_sinks_workspace(s, 2 ** 32 + 4), lambda: kvs.kvs_attend_sinks(s, 0, q, q.clone(), window=-2 ** 32 - 1),
                 lambda: kvs.kvs_weigh_sinks(s, 0, q, f, w, window=4, sinks=-2 ** 32)):
        with pytest.raises(kvs.KvsError) as ei:
            call()
        assert ei.value.code == kvs.KVS_ERR_INVALID_ARG


@pytest.mark.parametrize("n", [1, 90, 100, 101, 102, 150, 195, 196, 197, 690])
def test_text_goes_on_behind_a_picture(n):
    """At the position that a longer prompt gives its text behind the whole picture, or before that where the picture ends early; on one
    axis at the number of tokens."""
    import torch

    from paper_2609_35065_gb300 import prefix_step
    cfg = prefix_step.session()
    at = prefix_step.prompt_positions(cfg, n)
    p = prefix_step.next_position(at)
    assert p.shape == (3, 1) and p.dtype == torch.int32 and p.is_contiguous()
    assert (p == at.max() + 1).all()
    longer = prefix_step.prompt_positions(cfg, n + 1)[:, n]
    if n % 196 == 0 or n % 196 < 100:
        assert (p[:, 0] == longer).all()                # more text, or text behind a whole picture
    flat = prefix_step.prompt_positions(prefix_step.Config(), n)
    assert prefix_step.next_position(flat).tolist() == [n]
