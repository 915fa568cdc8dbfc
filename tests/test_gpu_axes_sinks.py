"""The operators with axes and with sinks against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import ops_ref
from long_ref import Long, rotate_axes
from ops_ref import Small
from paper_2609_35065_gb300 import kvs

pytestmark = pytest.mark.gpu


def _attend(sm, scale=None, decode=False, lse=True, stream=None, on=None):
    step, q, _, _, _cache = on or sm.on_gpu(kvs, decode)
    heads = sm.H * sm.G
    out = torch.full((step.total_q, heads, sm.D), 7.0, dtype=q.dtype, device="cuda")
    z = torch.full((step.total_q, heads), 7.0, device="cuda") if lse else None
    ws = torch.full((kvs.kvs_attend_sinks_workspace(step, heads, sm.causal, sm.window, sm.sinks),), 255, dtype=torch.uint8, device="cuda")
    kvs.kvs_attend_sinks(step, 0, q, out, z, scale, sm.causal, sm.window, sm.sinks, ws, stream, kvs.KVS_F_VALIDATE)
    return out, z


def _check(sm, out, z, scale=None):
    want, bound, lse, lse_bound = sm.attend(sm.D ** -0.5 if scale is None else scale, sm.causal, sm.window)
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()
    z = z.double().cpu().numpy()
    empty = np.isneginf(lse)
    assert (np.isneginf(z) == empty).all()
    assert (np.abs(z[~empty] - lse[~empty]) <= lse_bound[~empty]).all()
    assert (out[torch.from_numpy(empty).cuda()] == 0).all()


def _check_attend(sm, scale=None, decode=False):
    _check(sm, *_attend(sm, scale, decode), scale)


# ---- attention ----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,G", [(128, 2, 4), (64, 3, 7), (80, 1, 1), (72, 2, 5), (8, 2, 3), (120, 1, 16), (128, 1, 40)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (1, 1), (33, 130), (16, 0)])
def test_decode_steps(dtype, D, H, G, window, sinks):
    _check_attend(Long([1] * 7, [1, 2, 17, 101, 129, 700, 0], window, sinks, H, G, D, dtype=dtype), decode=True)


@pytest.mark.parametrize("new", [1, 5, 40, 150])
@pytest.mark.parametrize("B", [1, 3, 8, 16, 48, 128, 256])
def test_block_sizes(B, new):
    for window, sinks in ((60, 3), (130, 20), (7, 200)):
        _check_attend(Long([new, 1], [777, 513], window, sinks, 2, 4, 64, B))


@pytest.mark.parametrize("new,lens", [([0, 3, 0], [5, 3, 0]), ([16], [16]), ([17], [333]), ([130], [130]), ([129, 1, 64], [1000, 999, 64]), ([200], [513]),
                                      ([257], [2049]), ([5, 5], [4, 0]), ([300, 2], [260, 1000])])
@pytest.mark.parametrize("G,D,dtype", [(4, 128, "bf16"), (5, 64, "f16"), (8, 96, "bf16")])
@pytest.mark.parametrize("window,sinks,causal", [(64, 4, True), (200, 129, True), (1, 16, True), (128, 1, False), (31, 300, False)])
def test_chunks(new, lens, G, D, dtype, window, sinks, causal):
    _check_attend(Long(new, lens, window, sinks, 2, G, D, dtype=dtype, causal=causal))


@pytest.mark.parametrize("sinks", [1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 400])
@pytest.mark.parametrize("new,window", [(1, 200), (30, 200), (150, 100)])
def test_sinks_up_to_a_tile_and_beyond(sinks, new, window):
    _check_attend(Long([new], [1100], window, sinks, 1, 4, 128))


@pytest.mark.parametrize("T", list(range(118, 150, 3)) + [160, 161, 200])
def test_a_window_that_just_leaves_the_sinks(T):
    """The window's first token before, at and behind the last sink's, and its block."""
    for new in (1, 25):
        _check_attend(Long([new], [T], 100, 20, 2, 4, 64, given_back=T % 2 == 0))


@pytest.mark.parametrize("new,T,window", [(1, 30000, 20000), (3, 20001, 9000), (140, 20000, 8200), (30, 9000, 4000)])
def test_long_windows_are_split_and_joined(new, T, window):
    _check_attend(Long([new], [T], window, 5, 1, 4, 128))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 30, 150])
@pytest.mark.parametrize("pull", [3.0, 30.0])
def test_sinks_that_take_most_of_the_weight(new, dtype, pull):
    """Scores of the sinks up to e^300 above the window's, for some of the rows."""
    sm = Long([new], [900], 256, 4, 2, 4, 64, dtype=dtype)
    k = sm.cache[0].view(-1, sm.H, sm.D)
    k[sm.slots(0, np.arange(4))] *= pull
    _check_attend(sm)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("new", [1, 30, 150])
def test_scales(scale, new):
    _check_attend(Long([new], [900], 300, 7, 2, 4, 64, spread=2.0), scale)


@pytest.mark.parametrize("new,lens", [([1, 1], [500, 3]), ([40, 3], [700, 400]), ([200], [300])])
def test_what_hides_nothing_is_plain_attention(new, lens):
    """No window, one that all tokens fill, or sinks that reach it: the bits that kvs_attend gives."""
    sm = Small(new, lens, 2, 4, 128)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    heads = sm.H * sm.G
    got = []
    plain = torch.empty(kvs.kvs_attend_workspace(step, heads) + 16, dtype=torch.uint8, device="cuda")
    out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    kvs.kvs_attend(step, 0, q, out, z, workspace=plain)
    for window, sinks in ((0, 0), (0, 50), (step.max_kv, 1), (step.max_kv - 20, 20), (3, step.max_kv), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert kvs.kvs_attend_sinks_workspace(step, heads, True, window, sinks) == kvs.kvs_attend_workspace(step, heads)
        out2, z2 = torch.full_like(out, 7.0), torch.full_like(z, 7.0)
        kvs.kvs_attend_sinks(step, 0, q, out2, z2, None, True, window, sinks, plain)
        assert torch.equal(out, out2) and torch.equal(z, z2)


# more pairs of row tiles than SMs: CTAs go from one to the next
@pytest.mark.parametrize("new,lens,window,sinks,H,G,D,B,dtype,causal", [
    ([1500, 3, 0, 700], [1500, 50, 9, 3000], 100, 4, 8, 4, 128, 16, "bf16", True), ([2100, 1999], [2100, 1999], 128, 4, 4, 8, 64, 16, "f16", True),
    ([1400], [5000], 1024, 64, 8, 4, 128, 16, "bf16", True), ([700, 900], [900, 905], 33, 130, 8, 5, 96, 8, "bf16", True),
    ([1400, 20], [1800, 700], 64, 3, 8, 4, 80, 1, "f16", True), ([1400], [1800], 200, 300, 8, 4, 128, 128, "bf16", True),
    ([1400], [1800], 90, 5, 8, 4, 64, 256, "bf16", True), ([900], [500], 70, 4, 8, 7, 128, 32, "bf16", True), ([2600], [2600], 77, 4, 8, 2, 32, 16, "bf16", True),
    ([200], [330], 50, 4, 2, 130, 64, 16, "bf16", True), ([1400], [1700], 40, 17, 8, 4, 128, 16, "f16", False), ([50] * 100, [400] * 100, 60, 4, 2, 4, 128, 16, "bf16", True),
    ([1400], [1700], 1, 1, 8, 4, 64, 16, "bf16", True), ([700] * 3, [700, 1300, 350], 300, 0, 4, 8, 128, 3, "f16", True)])
def test_many_row_tiles(new, lens, window, sinks, H, G, D, B, dtype, causal):
    sm = Long(new, lens, window, sinks, H, G, D, B, dtype=dtype, causal=causal)
    on = sm.on_gpu(kvs)
    assert kvs.kvs_attend_sinks_workspace(on[0], H * G, causal, window, sinks) == 0
    first = _attend(sm, on=on)
    _check(sm, *first)
    for a, b in zip(first, _attend(sm, on=on)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("new,lens,window,H,G,D,dtype,causal", [
    ([293], [2600], 2048, 8, 5, 128, "bf16", True), ([150], [2600], 2048, 8, 5, 128, "f16", True), ([200], [2600], 2048, 8, 4, 72, "bf16", False),
    ([100, 280], [2500, 290], 2000, 4, 5, 128, "bf16", True), ([280, 0, 100], [3000, 7, 100], 2500, 4, 5, 128, "f16", True), ([400], [1900], 1500, 8, 8, 64, "bf16", True)])
def test_parts_of_two_row_tiles(new, lens, window, H, G, D, dtype, causal):
    """Parts of a pair of row tiles, joined by their cluster; some of the requests have fewer steps than there are parts."""
    sm = Long(new, lens, window, 5, H, G, D, dtype=dtype, causal=causal)
    _check_attend(sm)
    a, b = _attend(sm), _attend(sm)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("new,lens,window,H,G,D,B", [([13] * 30, [400] * 30, 100, 2, 2, 96, 8), ([6, 0, 3] * 9, [300, 5, 3] * 9, 28, 8, 7, 96, 16), ([20, 1], [700, 40], 100, 4, 4, 64, 16),
                                                     ([20, 1], [700, 40], 100, 4, 4, 128, 1)])
def test_one_row_tile_on_ctas_that_stay(new, lens, window, H, G, D, B):
    _check_attend(Long(new, lens, window, 3, H, G, D, B))


def test_the_neighbours_of_a_request_do_not_matter():
    sm = Long([2, 150, 1], [700, 650, 350], 90, 6, 2, 4, 128)
    a, za = _attend(sm)
    for _ in range(3):
        b, zb = _attend(sm)
        assert torch.equal(a, b) and torch.equal(za, zb)
    assert torch.equal(_attend(sm, lse=False)[0], a)


def test_on_another_stream_and_in_strided_outputs():
    sm = Long([2, 150], [700, 650], 90, 6, 2, 4, 128)
    want, z_want = _attend(sm)
    s = torch.cuda.Stream()
    step, q, _, _, _cache = sm.on_gpu(kvs)
    wide = torch.full((8, sm.N, 3 * sm.D), 7.0, dtype=q.dtype, device="cuda")
    out = wide[..., sm.D: 2 * sm.D].transpose(0, 1)
    z = torch.empty_like(z_want)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 8, True, 90, 6) + 16, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    kvs.kvs_attend_sinks(step, 0, q, out, z, None, True, 90, 6, ws, s)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(z, z_want)
    assert (wide[..., : sm.D] == 7.0).all() and (wide[..., 2 * sm.D:] == 7.0).all()


@pytest.mark.parametrize("new,lens,H,window", [([1, 2], [100, 60], 2, 30), ([40, 1], [120, 60], 8, 30), ([1], [1500], 1, 1000), ([20], [1500], 1, 1000),
                                               ([2, 1], [30000, 300], 1, 20000), ([140], [9000], 1, 8200)])
def test_rows_of_no_request_keep_what_they_hold(new, lens, H, window):
    sm = Long(new, lens, window, 4, H, 4, 128)
    want, z_want = _attend(sm)
    step, q, _, _, cache = sm.on_gpu(kvs)
    rows = 3 + sm.N + 5
    padded = kvs.Step((1, H, 128, 2, 16, 16), [cache[0], cache[1]], sm.num_blocks, step._keep[0], step._keep[1], step._keep[2] + 3, total_q=rows, max_q=max(new))
    q2 = torch.full((rows, *q.shape[1:]), float("nan"), dtype=q.dtype, device="cuda")
    q2[3: 3 + sm.N] = q
    out, z = _attend(sm, on=(padded, q2, None, None, cache))
    mine = slice(3, 3 + sm.N)
    assert torch.equal(out[mine], want) and torch.equal(z[mine], z_want)
    for x in (out, z):
        assert (x[:3] == 7.0).all() and (x[3 + sm.N:] == 7.0).all()


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("where", [0, 300, 899])
def test_a_seen_block_out_of_bounds_is_recorded(new, where):
    """Of the sinks, within the window and the last one; the other request comes out right."""
    sm = Long([new, new], [900, 900], 700, 4, 2, 4, 64)
    want = _attend(sm)[0]
    sm.tables[1, where // sm.B] = sm.num_blocks
    step, q, _, _, _cache = sm.on_gpu(kvs)
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 8, True, 700, 4) + 16, dtype=torch.uint8, device="cuda")
    kvs.kvs_attend_sinks(step, 0, q, out, None, None, True, 700, 4, ws)
    with pytest.raises(kvs.KvsError) as ei:
        kvs.kvs_check_errors()
    assert ei.value.code == kvs.KVS_ERR_BOUNDS
    kvs.kvs_check_errors()
    assert torch.equal(out[:new], want[:new])


def test_a_graph_follows_the_lengths():
    """A captured step's window moves on with the lengths that it reads anew."""
    sm = Long([1, 1], [1700, 900], 200, 4, 2, 4, 64, given_back=False)
    sm.cache.nan_to_num_(0.5)
    step, q, _, _, _cache = sm.on_gpu(kvs, decode=True)
    out, z = torch.zeros(q.shape, dtype=q.dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.zeros(kvs.kvs_attend_sinks_workspace(step, 8, True, 200, 4), dtype=torch.uint8, device="cuda")
    w = torch.zeros(2, 2, step.max_kv, device="cuda")
    lens = step._keep[1]
    s = torch.cuda.Stream()
    args = (step, 0, q, out, z, None, True, 200, 4, ws)
    kvs.kvs_attend_sinks(*args, s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        kvs.kvs_attend_sinks(*args, torch.cuda.current_stream())
        kvs.kvs_weigh_sinks(step, 0, q, z, w, None, 0.5, True, 200, 4, torch.cuda.current_stream())
    for lengths in ([1700, 900], [1699, 205], [204, 1], [33, 0]):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        before = w.cpu().numpy()
        g.replay()
        torch.cuda.synchronize()
        sm.lens, sm.hidden = lengths, [np.zeros(T, dtype=bool) for T in lengths]
        want, bound, *_ = sm.attend(sm.D ** -0.5, True, 200)
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
        want, bound = sm.weigh(z.cpu().numpy(), before, 0.5, sm.D ** -0.5, True, 200)
        assert (np.abs(w.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("new,lens,window", [([1, 1], [700, 300], 100), ([40, 3], [700, 400], 100), ([1500], [1800], 100), ([300], [2000], 1500)])
def test_rows_of_heads_behind_one_another(new, lens, window):
    """Queries and outputs that lie head by head: [heads][tokens][dims]."""
    sm = Long(new, lens, window, 5, 4, 4, 64)
    step, q, _, _, cache = sm.on_gpu(kvs)
    want, z_want = _attend(sm, on=(step, q, None, None, cache))
    by_head = q.transpose(0, 1).contiguous().transpose(0, 1)
    out, z = torch.empty(16, sm.N, 64, dtype=q.dtype, device="cuda").transpose(0, 1), torch.empty_like(z_want)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 16, True, window, 5) + 16, dtype=torch.uint8, device="cuda")
    kvs.kvs_attend_sinks(step, 0, by_head, out, z, None, True, window, 5, ws, flags=kvs.KVS_F_VALIDATE)
    assert torch.equal(out, want) and torch.equal(z, z_want)
    w = torch.zeros(2, sm.R, 4, step.max_kv, device="cuda")
    for x, rows in zip(w, (q, by_head)):
        kvs.kvs_weigh_sinks(step, 0, rows, z, x, None, 1.0, True, window, 5, flags=kvs.KVS_F_VALIDATE)
    assert torch.equal(w[0], w[1])


def test_calls_at_once():
    """Calls of both kinds on streams of their own, many times over."""
    cases = [Long([1500], [1800], 100, 5, 8, 4, 128), Long([2], [30000], 20000, 5, 1, 4, 128), Long([700, 700], [700, 1300], 64, 4, 4, 8, 64), Long([30], [9000], 4000, 4, 1, 4, 64)]
    on = [sm.on_gpu(kvs) for sm in cases]
    want = [_attend(sm, on=o) for sm, o in zip(cases, on)]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [(torch.zeros_like(a), torch.zeros_like(z), torch.zeros(sm.R, sm.H, o[0].max_kv, device="cuda"),
             torch.empty(kvs.kvs_attend_sinks_workspace(o[0], sm.H * sm.G, True, sm.window, sm.sinks) + 16, dtype=torch.uint8, device="cuda"))
            for sm, o, (a, z) in zip(cases, on, want)]
    torch.cuda.synchronize()
    for _ in range(5):
        for sm, o, s, (a, z, w, ws) in zip(cases, on, streams, outs):
            kvs.kvs_attend_sinks(o[0], 0, o[1], a, z, None, True, sm.window, sm.sinks, ws, s)
            kvs.kvs_weigh_sinks(o[0], 0, o[1], z, w, None, 0.0, True, sm.window, sm.sinks, s)
    torch.cuda.synchronize()
    kvs.kvs_check_errors()
    for sm, o, (a, z, w, _), (a0, z0) in zip(cases, on, outs, want):
        assert torch.equal(a, a0) and torch.equal(z, z0)
        again = torch.zeros_like(w)
        kvs.kvs_weigh_sinks(o[0], 0, o[1], z, again, None, 0.0, True, sm.window, sm.sinks)
        assert torch.equal(w, again)


@pytest.mark.parametrize("new,lens,window,H,G,D,B", [([1, 1], [700, 300], 100, 2, 4, 64, 16), ([1], [9000], 4000, 1, 4, 128, 16), ([6, 3], [700, 300], 100, 2, 4, 64, 16),
                                                      ([40, 3], [700, 400], 100, 2, 4, 128, 48), ([300], [3000], 2000, 2, 4, 128, 16), ([1500], [1800], 100, 4, 4, 64, 16),
                                                      ([1500], [1800], 100, 4, 4, 72, 1)])
def test_calls_behind_kernels_that_write_what_they_read(new, lens, window, H, G, D, B):
    """Queries, tables, lengths, positions and the turns' tables are each the last thing written before a call, by a kernel that has not ended
    when the call is made; what a call writes is read by the next."""
    sm = Long(new, lens, window, 5, H, G, D, B, given_back=False)
    sm.cache.nan_to_num_(0.5)
    step, q, k, v, cache = sm.on_gpu(kvs)
    tables, kv_lens = step._keep[:2]
    turns, axis, scale = kvs.kvs_rope_axes([D // 4, D // 4], restart=True)
    turns, axis = torch.from_numpy(turns).cuda(), torch.from_numpy(axis).cuda()
    rope, axes = kvs.Rope(turns, D, scale=scale), kvs.Axes(axis, 2)
    positions = torch.randint(0, 5000, (2, sm.N), device="cuda").int()
    inputs = [q, tables, kv_lens, positions, turns, axis]
    fewer = [int(n) for n in (torch.tensor(lens) - 1).clamp(min=1)]
    states = [[x.clone() for x in inputs] for _ in range(2)]
    states[1][0].mul_(-0.5)
    full = min(fewer) // B
    states[1][1][:, :full] = tables[:, :full].flip(1)
    states[1][2].copy_(torch.tensor(fewer, dtype=torch.int32))
    states[1][3].add_(77)
    states[1][4].mul_(1.5)
    states[1][5].copy_(axis.flip(0))
    heads, first = H * G, cache.clone()
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, heads, True, window, 5) + 16, dtype=torch.uint8, device="cuda")
    big = torch.zeros(1 << 26, device="cuda")

    def run(state, last, wait):
        cache.copy_(first)
        q_out, out = torch.zeros_like(q), torch.zeros_like(q)
        z, w = torch.zeros(sm.N, heads, device="cuda"), torch.zeros(sm.R, H, step.max_kv, device="cuda")
        for x in range(len(inputs)):
            at = (last + 1 + x) % len(inputs)
            if x == len(inputs) - 1 and not wait:
                big.add_(1.0)                                    # so that the calls are made while the writes are still to come
            torch.add(states[state][at], 0, out=inputs[at])
        calls = [lambda: kvs.kvs_append_axes(step, 0, q, k, v, q_out, rope, axes, positions),
                 lambda: kvs.kvs_attend_sinks(step, 0, q_out, out, z, None, True, window, 5, ws),
                 lambda: kvs.kvs_weigh_sinks(step, 0, q_out, z, w, None, 0.5, True, window, 5),
                 lambda: kvs.kvs_attend_sinks(step, 0, q, out, z, None, True, window, 5, ws),
                 lambda: kvs.kvs_weigh_sinks(step, 0, q, z, w, None, 0.5, True, window, 5)]
        for f in calls:
            f()
            if wait:
                torch.cuda.synchronize()
        return [q_out, out, z, w, cache.clone()]

    want = [run(s, 0, True) for s in range(2)]
    for i in range(6 * len(inputs)):
        got = run(i % 2, i // 2, False)
        for a, b in zip(got, want[i % 2]):
            assert torch.equal(a, b), i
    torch.cuda.synchronize()
    kvs.kvs_check_errors()


def test_a_graph_of_many_rows_follows_the_step():
    """Rows, lengths, tables and positions of a captured prefill are read anew at each replay."""
    sm = Long([900, 300], [1700, 900], 100, 4, 4, 4, 128, given_back=False)
    sm.cache.nan_to_num_(0.5)
    step, q, k, v, cache = sm.on_gpu(kvs)
    turns, axis, axes = _axes([16, 24, 24])
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), 128)
    pos = torch.zeros(3, sm.N, dtype=torch.int32, device="cuda")
    q_out, out, z = torch.zeros(q.shape, dtype=q.dtype, device="cuda"), torch.zeros(q.shape, dtype=q.dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 16, True, 100, 4) + 16, dtype=torch.uint8, device="cuda")

    def layer(s):
        kvs.kvs_append_axes(step, 0, q, k, v, q_out, rope, axes, pos, s)
        kvs.kvs_attend_sinks(step, 0, q_out, out, z, None, True, 100, 4, ws, s)
    s = torch.cuda.Stream()
    layer(s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        layer(torch.cuda.current_stream())
    tables, lens, starts = step._keep[:3]
    for new, lengths in (([900, 300], [1700, 900]), ([5, 700], [5, 1690]), ([0, 899], [33, 1000])):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        starts.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        pos.random_(0, 5000)
        g.replay()
        torch.cuda.synchronize()
        kvs.kvs_check_errors()
        sm.new, sm.lens, sm.N, sm.starts = new, lengths, sum(new), np.concatenate([[0], np.cumsum(new)])
        sm.hidden = [np.zeros(T, dtype=bool) for T in lengths]
        x = q[: sm.N]
        _off(q_out[: sm.N], x, pos[:, : sm.N].cpu().numpy(), axis, turns, False, 1.0, 2.0 ** -8)
        sm.cache, sm.qkv = cache.view(2, -1, 4, 128).cpu(), torch.cat([q_out[: sm.N].reshape(sm.N, -1), torch.zeros(sm.N, 8 * 128, dtype=q.dtype, device="cuda")], 1).cpu()
        _check(sm, out[: sm.N], z[: sm.N])


# ---- weights --------------------------------------------------------------------
def _check_weigh(sm, decay, decode=False, seed=3):
    step, q, _, _, _cache = sm.on_gpu(kvs, decode)
    scale = sm.D ** -0.5
    lse = sm.attend(scale, sm.causal, sm.window)[2].astype(np.float32)
    rng = np.random.default_rng(seed)
    before = rng.random((sm.R, sm.H, step.max_kv)).astype(np.float32)
    if decay in (0.0, 1.0):                                        # not read, or not touched
        for r, T in enumerate(sm.lens):
            before[r, :, :T][:, sm.hidden[r]] = np.nan
    wide = torch.full((sm.H, sm.R, step.max_kv + 5), 9.0, device="cuda")
    w = wide[..., 2: 2 + step.max_kv].transpose(0, 1)
    w.copy_(torch.from_numpy(before))
    kvs.kvs_weigh_sinks(step, 0, q, torch.from_numpy(lse).cuda(), w, scale, decay, sm.causal, sm.window, sm.sinks, flags=kvs.KVS_F_VALIDATE)
    want, bound = sm.weigh(lse, np.nan_to_num(before), decay, scale, sm.causal, sm.window)
    got = w.double().cpu().numpy()
    for r, T in enumerate(sm.lens):
        if decay == 1.0:
            assert np.isnan(got[r, :, :T][:, sm.hidden[r]]).all()
            got[r, :, :T][:, sm.hidden[r]] = 0.0
        assert (np.abs(got[r, :, :T] - want[r, :, :T]) <= bound[r, :, :T]).all()
        assert (got[r, :, T:] == before[r, :, T:]).all()
    assert (wide[..., :2] == 9.0).all() and (wide[..., 2 + step.max_kv:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens,H,G,D,B,causal,window,sinks,decay", [
    ([1, 1, 1], [1, 130, 700], 2, 4, 128, 16, True, 60, 4, 0.5), ([1], [257], 1, 1, 64, 1, True, 31, 3, 1.0), ([3, 0, 40], [500, 9, 300], 2, 7, 80, 16, True, 90, 17, 0.0),
    ([130], [128], 2, 4, 64, 16, True, 64, 4, 0.9), ([200, 1], [600, 1600], 1, 5, 128, 32, True, 100, 1, 0.9), ([20], [590], 2, 3, 96, 3, False, 40, 130, 1.0),
    ([260], [900], 1, 8, 128, 16, True, 128, 256, 1.0), ([4], [0], 2, 2, 64, 16, True, 5, 5, 1.0), ([7], [300], 1, 40, 128, 16, False, 5, 4, 0.25),
    ([1, 2], [40000, 70], 2, 4, 64, 16, True, 500, 4, 0.75), ([50, 3], [40000, 70], 2, 4, 64, 16, True, 500, 4, 0.75), ([30], [3000], 1, 4, 64, 256, True, 70, 4, 0.5),
    ([700], [1500], 1, 4, 128, 16, True, 130, 4, 0.5)])
def test_weights(dtype, new, lens, H, G, D, B, causal, window, sinks, decay):
    _check_weigh(Long(new, lens, window, sinks, H, G, D, B, dtype=dtype, causal=causal), decay, decode=new == [1] * len(new))


@pytest.mark.parametrize("new", [1, 3, 30, 150])
@pytest.mark.parametrize("sinks", [0, 1, 16, 17, 128, 129, 300])
def test_weights_of_sinks(new, sinks):
    _check_weigh(Long([new], [900], 100, sinks, 2, 4, 64), 0.5)


@pytest.mark.parametrize("T", [118, 121, 127, 128, 129, 160])
def test_weights_where_the_window_just_leaves_the_sinks(T):
    for new in (1, 25):
        _check_weigh(Long([new], [T], 100, 20, 2, 4, 64), 0.5)


@pytest.mark.parametrize("new,G,D", [(750, 4, 128), (700, 4, 64)])
def test_weights_of_many_rows(new, G, D):
    """More than 2560 packed rows go by two key tiles at a time."""
    _check_weigh(Long([new], [1100], 90, 5, 1, G, D), 0.5)


@pytest.mark.parametrize("new", [[0, 1], [0, 20], [0, 150]])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_a_request_without_new_tokens_only_fades(new, decay):
    """No token sees its cache, of which no block table entry is read."""
    sm = Long(new, [700, 650], 90, 6, 2, 4, 64)
    sm.tables[0] = -1
    step, q, _, _, _cache = sm.on_gpu(kvs)
    z = _attend(sm, on=(step, q, None, None, _cache))[1]
    w = torch.rand(2, 2, step.max_kv, device="cuda")
    before = w.clone()
    kvs.kvs_weigh_sinks(step, 0, q, z, w, None, decay, True, 90, 6, flags=kvs.KVS_F_VALIDATE)
    assert torch.equal(w[0, :, :700], before[0, :, :700] * decay)
    assert torch.equal(w[0, :, 700:], before[0, :, 700:])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 72, 96, 128])
@pytest.mark.parametrize("window", [300, 0])
def test_weights_of_heavy_tokens(dtype, D, window):
    """Keys of eight tokens lie along all queries, whose lse is near 20: a weight is the exponential of a small difference of two such
    numbers, and an error of the score that all rows share stays.  Products of 16 dims are cut off at 2^-23 of their sum and again where that
    is added, 2 D / 16 times 2^-23 of the score at most as these sums only grow; what is made up for on average is less than
    that.  The exponent's parts, up to log2(e) 21 < 32, are rounded twice, by 2^-20 each, and the exponential once, by 2^-22."""
    new, T, G = 400, 700, 2
    sm = Long([new], [T], window, 8, 1, G, D, 16, dtype=dtype, given_back=False)
    sm.cache.nan_to_num_(0.5)
    g = torch.Generator().manual_seed(1)
    along = torch.randn(D, generator=g)
    q, _, _ = sm.parts(sm.qkv)
    q.copy_((along + 0.1 * torch.randn(q.shape, generator=g)).to(q.dtype))
    sm.cache[0, torch.from_numpy(sm.slots(0, np.arange(8))), 0] = (20.0 / D ** 0.5 * along).to(q.dtype)
    step, qg, _, _, _cache = sm.on_gpu(kvs)
    scale = D ** -0.5
    x, *_ = zip(*[sm.scores(0, 0, i, float(np.float32(scale)), True, window) for i in range(G)])
    x = np.stack(x, 1)                                                       # [new, G, T]
    lse = torch.from_numpy(np.log(np.exp(x).sum(-1))).float()
    assert lse.mean() > 15
    want = np.exp(x - lse.double().numpy()[..., None]).sum((0, 1))
    w = torch.zeros(1, 1, step.max_kv, device="cuda")
    kvs.kvs_weigh_sinks(step, 0, qg, lse.cuda(), w, scale, 0.0, True, window, 8)
    off = w[0, 0, :T].double().cpu().numpy() - want
    bound = 21 * (2 * -(-D // 16)) * 2.0 ** -23 + 2 * 2.0 ** -20 * np.log(2) + 2.0 ** -22
    assert np.linalg.norm(off) <= bound * np.linalg.norm(want)


def test_weights_add_up_to_the_rows():
    sm = Long([3, 150], [700, 650], 90, 6, 2, 4, 128)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    _, z = _attend(sm)
    w = torch.zeros(2, 2, step.max_kv, device="cuda")
    kvs.kvs_weigh_sinks(step, 0, q, z, w, None, 0.0, True, 90, 6)
    rows = torch.tensor([3.0, 150.0], device="cuda")[:, None] * 4
    # each row's weights add up to one within the error of lse and of the products
    assert ((w.sum(-1) - rows).abs() <= rows * 1e-4).all()


# ---- append -----------------------------------------------------------------------
def _axes(parts, **kw):
    turns, axis, scale = kvs.kvs_rope_axes(parts, **kw)
    return turns, axis, kvs.Axes(torch.from_numpy(axis).cuda(), len(parts))


def _off(got, x, positions, axis, turns, inter, scale, unit):
    """Whether `got` is x rotated, within what the angles and one rounding may take."""
    x = x.double().cpu().numpy()
    y = rotate_axes(x, positions, axis, turns, inter, scale)
    off = np.abs(got.double().cpu().numpy() - y)
    rot = 2 * len(axis)
    big = np.abs(x).max(-1, keepdims=True)
    assert (off <= unit * np.abs(y) + scale * 2.0 ** -19 * big + 2.0 ** -25).all()
    assert (off[..., rot:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,parts,cycle,restart,inter", [
    (128, [16, 24, 24], False, False, False), (128, [24, 20, 20], True, False, False), (128, [32, 32], False, True, False), (128, [22, 21, 21], True, True, True),
    (128, [1, 2, 3, 10], False, False, False), (72, [18, 18], False, True, False), (72, [12, 12, 12], True, False, True), (80, [10, 10], False, False, False),
    (80, [40], False, False, False), (64, [5, 5, 4], False, False, False), (64, [3, 3, 3], False, False, False), (64, [2, 1], True, False, True),
    (120, [30, 30], False, True, False), (96, [7, 6], False, False, False), (8, [1, 1], False, False, False), (8, [1], False, False, False),
    (128, [31, 32], False, False, False), (128, [60, 1, 1, 1], False, False, False)])
@pytest.mark.parametrize("new,lens", [([1, 1], [1, 40]), ([3, 0, 33], [3, 7, 100])])
def test_append_axes(dtype, D, parts, cycle, restart, inter, new, lens):
    sm = Small(new, lens, 2, 3, D, dtype=dtype)
    step, q, k, v, cache = sm.on_gpu(kvs, decode=new == [1, 1])
    turns, axis, axes = _axes(parts, cycle=cycle, restart=restart)
    positions = np.random.default_rng(2).integers(-1000, 200000, (len(parts), sm.N)).astype(np.int32)
    positions[:, 0] = [1 << 24, -(1 << 24), 0, 1][: len(parts)]
    wide = torch.full((len(parts), sm.N + 3), 99, dtype=torch.int32, device="cuda")       # axes lie apart
    wide[:, 2: 2 + sm.N] = torch.from_numpy(positions).cuda()
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), 2 * len(axis), inter, 1.5)
    q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    before = cache.clone()
    kvs.kvs_append_axes(step, 0, q, k, v, q_out, rope, axes, wide[:, 2: 2 + sm.N], None, kvs.KVS_F_VALIDATE)
    at = np.concatenate([sm.slots(r, np.arange(T - n, T)) for r, (n, T) in enumerate(zip(new, lens))])
    got_k = cache.view(2, -1, sm.H, D)[0, at]
    for x, got in ((q, q_out), (k, got_k)):
        _off(got, x, positions, axis, turns, inter, 1.5, ops_ref.UNIT[dtype])
    want = before.view(2, -1, sm.H, D).clone()
    want[0, at], want[1, at] = got_k, v
    assert torch.equal(cache.view(torch.int16), want.view(cache.shape).view(torch.int16))
    # in place, and without queries
    step2, q2, k2, v2, cache2 = sm.on_gpu(kvs, decode=new == [1, 1])
    kvs.kvs_append_axes(step2, 0, q2, k2, v2, None, rope, axes, wide[:, 2: 2 + sm.N])
    assert torch.equal(q2, q_out) and torch.equal(cache2.view(torch.int16), cache.view(torch.int16))
    step3, _, k3, v3, cache3 = sm.on_gpu(kvs, decode=new == [1, 1])
    kvs.kvs_append_axes(step3, 0, None, k3, v3, None, rope, axes, wide[:, 2: 2 + sm.N])
    assert torch.equal(cache3.view(torch.int16), cache.view(torch.int16))


def test_append_of_many_rows_and_wide_models():
    """More rows than the GPU has warps for at once, and more heads than a warp takes."""
    for new, lens, H, G in (([700, 0, 4000], [700, 3, 4100], 1, 2), ([2, 1], [30, 40], 40, 2)):
        sm = Small(new, lens, H, G, 64)
        step, q, k, v, cache = sm.on_gpu(kvs)
        turns, axis, axes = _axes([8, 12, 12])
        positions = np.random.default_rng(3).integers(0, 5000, (3, sm.N)).astype(np.int32)
        q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        kvs.kvs_append_axes(step, 0, q, k, v, q_out, kvs.Rope(torch.from_numpy(turns).cuda(), 64), axes, torch.from_numpy(positions).cuda(), None, kvs.KVS_F_VALIDATE)
        at = np.concatenate([sm.slots(r, np.arange(T - n, T)) for r, (n, T) in enumerate(zip(new, lens))])
        for x, got in ((q, q_out), (k, cache.view(2, -1, H, 64)[0, at])):
            _off(got, x, positions, axis, turns, False, 1.0, ops_ref.UNIT["bf16"])
        assert torch.equal(cache.view(2, -1, H, 64)[1, at], v)


def test_a_text_token_comes_out_as_on_one_axis():
    sm = Small([5, 40], [700, 60], 2, 4, 128)
    turns, axis, axes = _axes([16, 24, 24])
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), 128)
    pos = torch.randint(0, 100000, (sm.N,), dtype=torch.int32, device="cuda")
    got = []
    for three in (False, True):
        step, q, k, v, cache = sm.on_gpu(kvs)
        if three:
            kvs.kvs_append_axes(step, 0, q, k, v, None, rope, axes, pos.expand(3, -1).contiguous())
        else:
            kvs.kvs_append(step, 0, q, k, v, None, rope, pos)
        at = np.concatenate([sm.slots(r, np.arange(T - n, T)) for r, (n, T) in enumerate(zip(sm.new, sm.lens))])
        got.append((q, cache.view(2, -1, 2, 128)[:, at]))
    for a, b in zip(*got):
        # both are within half a unit of the same value
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * a.float().abs() + 2.0 ** -18).all()


@pytest.mark.parametrize("bad", [4, 255])
def test_an_axis_out_of_bounds_is_recorded_and_turns_by_nothing(bad):
    sm = Small([3], [50], 2, 2, 64)
    step, q, k, v, _cache = sm.on_gpu(kvs)
    turns, axis, axes = _axes([16, 16])
    axes.axis[5] = bad
    pos = torch.randint(1, 1000, (2, 3), dtype=torch.int32, device="cuda")
    x = q.clone()
    with pytest.raises(kvs.KvsError) as ei:
        kvs.kvs_append_axes(step, 0, q, k, v, None, kvs.Rope(torch.from_numpy(turns).cuda(), 64), axes, pos, None, kvs.KVS_F_VALIDATE)
    assert ei.value.code == kvs.KVS_ERR_BOUNDS
    assert torch.equal(q[..., [5, 37]], x[..., [5, 37]])
    keep = np.r_[0:5, 6:32]
    y = rotate_axes(x.double().cpu().numpy(), pos.cpu().numpy(), axis, turns, False)
    off = np.abs(q.double().cpu().numpy() - y)[..., np.r_[keep, keep + 32]]
    assert (off <= 2.0 ** -8 * 8 + 1e-3).all()


@pytest.mark.parametrize("new,lens", [([3, 0, 4], [9, 0, 4]), ([5], [3]), ([1] * 40, [7] * 40)])
def test_append_leaves_other_rows_and_tokens_alone(new, lens):
    """Rows of no request keep what they hold; new tokens beyond the cached ones have their queries rotated only."""
    sm = Small(new, lens, 2, 3, 72)
    turns, axis, axes = _axes([18, 18], restart=True)
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), 72)
    step, q, k, v, cache = sm.on_gpu(kvs)
    before = cache.clone()
    rows = 3 + sm.N + 5
    positions = torch.randint(0, 5000, (2, rows), dtype=torch.int32, device="cuda")
    padded = kvs.Step((1, 2, 72, 2, 16, 16), [cache[0], cache[1]], sm.num_blocks, step._keep[0], step._keep[1], step._keep[2] + 3, total_q=rows, max_q=max(new))

    def pad(x):
        y = torch.full((rows, *x.shape[1:]), 3.0, dtype=x.dtype, device="cuda")
        y[3: 3 + sm.N] = x
        return y
    q2 = pad(q)
    kvs.kvs_append_axes(padded, 0, q2, pad(k), pad(v), None, rope, axes, positions, None, kvs.KVS_F_VALIDATE)
    mine = slice(3, 3 + sm.N)
    _off(q2[mine], q, positions[:, mine].cpu().numpy(), axis, turns, False, 1.0, 2.0 ** -8)
    assert (q2[:3] == 3.0).all() and (q2[3 + sm.N:] == 3.0).all()
    at = torch.from_numpy(np.concatenate([sm.slots(r, np.arange(max(0, T - n), T)) for r, (n, T) in enumerate(zip(new, lens))])).cuda()
    keep = torch.ones(sm.num_blocks * 16, dtype=torch.bool, device="cuda")
    keep[at] = False
    flat, old = cache.view(2, -1, 2, 72).view(torch.int16), before.view(2, -1, 2, 72).view(torch.int16)
    assert torch.equal(flat[:, keep], old[:, keep])


# ---- together ---------------------------------------------------------------------
def test_offsets_beyond_32_bits():
    """Blocks at the end of planes of more than 2^31 elements: what the same blocks give in small planes."""
    for new, lens in (([1, 2], [600, 33]), ([30, 1], [600, 33]), ([200, 130], [600, 200])):
        sm = Small(new, lens, 8, 4, 128)
        step, q, k, v, cache = sm.on_gpu(kvs)
        NB = (1 << 31) // (16 * 8 * 128) + 200
        shift = NB - sm.num_blocks
        far = torch.empty(2, NB, 16, 8, 128, dtype=cache.dtype, device="cuda")
        far[:, shift:] = cache
        tables, kv_lens, starts = step._keep[:3]
        step2 = kvs.Step((1, 8, 128, 2, 16, 16), [far[0], far[1]], NB, tables + shift, kv_lens, starts, total_q=sm.N, max_q=max(new))
        turns, axis, axes = _axes([16, 24, 24])
        rope = kvs.Rope(torch.from_numpy(turns).cuda(), 128)
        pos = torch.randint(0, 5000, (3, sm.N), dtype=torch.int32, device="cuda")
        got = []
        for s in (step, step2):
            kvs.kvs_append_axes(s, 0, None, k, v, None, rope, axes, pos)
            out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:2], device="cuda")
            ws = torch.empty(kvs.kvs_attend_sinks_workspace(s, 32, True, 100, 4), dtype=torch.uint8, device="cuda")
            kvs.kvs_attend_sinks(s, 0, q, out, z, None, True, 100, 4, ws)
            w = torch.zeros(2, 8, s.max_kv, device="cuda")
            kvs.kvs_weigh_sinks(s, 0, q, z, w, None, 1.0, True, 100, 4, flags=kvs.KVS_F_VALIDATE)
            got.append((out, z, w))
        for a, b in zip(*got):
            assert torch.equal(a, b)
        assert torch.equal(far[:, shift:].view(torch.int16), cache.view(torch.int16))
        del far, step2


@pytest.mark.parametrize("new,lens", [([1, 1], [700, 90]), ([40, 3], [600, 90]), ([150], [800])])
def test_a_step_through_all_operators(new, lens):
    """Positions on axes, appended, attended to with sinks, weighed, and the cache cut by those weights."""
    window, sinks = 64, 4
    sm = Long(new, lens, window, sinks, 2, 4, 64, given_back=False, extra_blocks=40)
    step, q, k, v, cache = sm.on_gpu(kvs)
    turns, axis, axes = _axes([8, 12, 12])
    pos = np.random.default_rng(3).integers(0, 5000, (3, sm.N)).astype(np.int32)
    kvs.kvs_append_axes(step, 0, q, k, v, None, kvs.Rope(torch.from_numpy(turns).cuda(), 64), axes, torch.from_numpy(pos).cuda())
    out, z = _attend(sm, on=(step, q, None, None, cache))
    w = torch.zeros(1, sm.R, 2, step.max_kv, device="cuda")
    kvs.kvs_weigh_sinks(step, 0, q, z, w[0], None, 1.0, True, window, sinks)
    # what the definitions make of the appended cache and the rotated queries
    sm.cache = cache.view(2, -1, 2, 64).cpu()
    sm.qkv[:, : 8 * 64] = q.reshape(sm.N, -1).cpu()
    _check(sm, out, z)
    want, bound = sm.weigh(z.cpu().numpy(), np.zeros(w.shape[1:]), 1.0, 0.125, True, window)
    assert (np.abs(w[0].double().cpu().numpy() - want) <= bound).all()
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[: 5 * sm.R].reshape(sm.R, 5)
    kept = torch.empty(1, sm.R, 2, 68, dtype=torch.int32, device="cuda")
    kvs.kvs_evict(step, w, torch.from_numpy(free.astype(np.int32)).cuda(), 68, sinks, window, kept, flags=kvs.KVS_F_VALIDATE)
    for r, T in enumerate(lens):
        # the sinks and the window are what a step of one token leaves of weight
        assert (kept[0, r].cpu().numpy() == np.r_[:sinks, T - window: T]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_long_session_on_a_retrieved_prefix(dtype):
    """The example's decoder over pictures: a suffix on a retrieved prefix gives what the whole prompt's prefill gives,
    and decoding goes on over the blocks that are left."""
    from dataclasses import replace

    from paper_2609_35065_gb300 import prefix_step
    cfg = replace(prefix_step.session(), dtype=ops_ref.TYPE[dtype])
    r = prefix_step.run(cfg)
    # every rounding of the residual stream (4 layers, 3 products each, 8 or 11 bits) may differ once
    assert (r["suffix"] - r["whole"]).norm() <= 12 * ops_ref.UNIT[dtype] * r["whole"].norm()
    assert r["stored"] == 512 and len(r["suffix"]) == 178 and r["gone"] > 30
    T = r["cached"]
    w = r["weights"]
    assert torch.isfinite(w).all() and len(r["tokens"]) == 12
    # each of twelve tokens gives one unit per query head to what it sees: the sinks and a window that moves
    assert ((w.sum(-1) - 12 * cfg.group).abs() <= 12 * cfg.group * 1e-4).all()
    first = T - 12 + 1 - cfg.window
    assert (w[..., cfg.sinks: first] == 0).all() and (w[..., : cfg.sinks] > 0).all() and (w[..., first: T] > 0).all()


def test_pictures_positions_tell_the_axes_apart():
    """The decoder's logits follow a picture's rows and columns: with all axes alike they are others."""
    from paper_2609_35065_gb300 import prefix_step
    cfg = prefix_step.Config(axes=(8, 12, 12))
    a = prefix_step.run(cfg)
    flat = prefix_step.prompt_positions
    try:
        prefix_step.prompt_positions = lambda c, n: flat(prefix_step.Config(), n).expand(3, -1).contiguous()
        b = prefix_step.run(cfg)
    finally:
        prefix_step.prompt_positions = flat
    c = prefix_step.run(prefix_step.Config())
    # One axis and three alike are the same model: 4 layers x 3 products, whose roundings of 8 bits may differ once each, are
    # off by 12 * 2^-8 at most, and logits that are further off are another model's.
    rounding = 12 * 2.0 ** -8 * c["whole"].norm()
    assert (b["whole"] - c["whole"]).norm() <= rounding
    assert (a["whole"] - b["whole"]).norm() > rounding
