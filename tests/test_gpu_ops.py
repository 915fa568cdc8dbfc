"""The model operators on the paged cache against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import ops_ref
from ops_ref import Small
from paper_2609_35065_gb300 import kvs

pytestmark = pytest.mark.gpu


def _attend(sm, causal=True, window=0, scale=None, decode=False, lse=True, stream=None):
    step, q, _, _, _cache = sm.on_gpu(kvs, decode)
    heads = sm.H * sm.G
    out = torch.full((sm.N, heads, sm.D), 7.0, dtype=q.dtype, device="cuda")
    z = torch.full((sm.N, heads), 7.0, device="cuda") if lse else None
    ws = torch.full((kvs.kvs_attend_workspace(step, heads),), 255, dtype=torch.uint8, device="cuda")
    kvs.kvs_attend(step, 0, q, out, z, scale, causal, window, ws, stream, kvs.KVS_F_VALIDATE)
    return out, z


def _check_attend(sm, causal=True, window=0, scale=None, decode=False):
    out, z = _attend(sm, causal, window, scale, decode)
    want, bound, lse, lse_bound = sm.attend(sm.D ** -0.5 if scale is None else scale, causal, window)
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()
    z = z.double().cpu().numpy()
    empty = np.isneginf(lse)
    assert (np.isneginf(z) == empty).all()
    assert (np.abs(z[~empty] - lse[~empty]) <= lse_bound[~empty]).all()
    assert (out[torch.from_numpy(empty).cuda()] == 0).all()
    return out, z


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,G", [(128, 2, 4), (64, 3, 7), (80, 1, 1), (96, 2, 5), (8, 2, 3), (120, 1, 16), (128, 1, 40)])
def test_decode_steps(dtype, D, H, G):
    _check_attend(Small([1] * 6, [1, 2, 17, 128, 129, 700], H, G, D, dtype=dtype), decode=True)


@pytest.mark.parametrize("B", [1, 3, 8, 16, 48, 256])
def test_block_sizes(B):
    _check_attend(Small([1, 5, 40], [300, 77, 513], 2, 4, 64, B))


@pytest.mark.parametrize("new,lens", [
    ([1], [1]), ([0, 3, 0], [5, 3, 0]), ([16], [16]), ([17], [33]), ([130], [130]), ([129, 1, 64], [1000, 999, 64]),
    ([200], [513]), ([256], [256]), ([257], [2049]), ([5, 5], [4, 0]), ([300, 2], [260, 1000])])
@pytest.mark.parametrize("G,D,dtype", [(4, 128, "bf16"), (5, 64, "f16"), (1, 128, "f16"), (8, 128, "bf16")])
def test_chunks(new, lens, G, D, dtype):
    _check_attend(Small(new, lens, 2, G, D, dtype=dtype))


@pytest.mark.parametrize("window", [1, 7, 64, 129, 5000])
@pytest.mark.parametrize("new,lens", [([1, 1], [500, 3]), ([200, 3], [700, 400]), ([6], [4])])
def test_windows(window, new, lens):
    _check_attend(Small(new, lens, 2, 4, 128), window=window)
    _check_attend(Small(new, lens, 2, 4, 128), causal=False, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,T,window", [(200, 700, 70), (64, 900, 33), (64, 900, 128), (250, 1500, 200)])
def test_rows_that_see_nothing_of_the_first_keys(new, T, window, dtype):
    """The last rows of a tile begin to see keys some steps after the first ones."""
    _check_attend(Small([new], [T], 2, 4, 128, dtype=dtype, spread=0.05), window=window)
    _check_attend(Small([new], [T], 1, 4, 128, dtype=dtype, spread=2.0), window=window, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 150])
def test_maxima_that_jump(new, dtype):
    """Blocks of keys whose scores outgrow those before by up to e^300, and fall again."""
    sm = Small([new], [1100], 2, 4, 64, dtype=dtype)
    k = sm.cache[0].view(-1, sm.H, sm.D)
    at = sm.slots(0, np.arange(1100))
    size = torch.tensor([0.05, 0.5, 4.0, 1.0, 12.0, 0.1, 30.0, 8.0, 40.0])[torch.arange(1100) // 128]
    k[at] *= size[:, None, None].to(k.dtype)
    _check_attend(sm)


@pytest.mark.parametrize("new,lens", [([3, 40], [1, 300]), ([130, 7], [129, 0]), ([300], [50])])
def test_every_cached_token_is_seen_without_causality(new, lens):
    _check_attend(Small(new, lens, 2, 4, 64), causal=False)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
@pytest.mark.parametrize("new", [1, 150])
def test_scales_and_peaked_rows(scale, new):
    """Scores of +-100: rows whose softmax is one token, maxima that grow along the keys."""
    sm = Small([new], [900], 2, 4, 64, spread=2.0)
    k = sm.cache[0].view(-1, sm.H, sm.D)
    at = sm.slots(0, np.arange(900))
    k[at] *= torch.linspace(0.1, 2.0, 900)[:, None, None].to(k.dtype)
    _check_attend(sm, scale=scale)


@pytest.mark.parametrize("new,T", [(1, 20000), (3, 9001), (140, 8200)])
def test_long_caches_are_split_and_joined(new, T):
    sm = Small([new], [T], 1, 4, 128)
    _check_attend(sm)


def test_the_result_does_not_depend_on_the_neighbours():
    """A request's rows come out the same bits alone and in a batch that is split alike, and from call to call."""
    sm = Small([2, 150, 1], [700, 650, 350], 2, 4, 128)
    a, za = _attend(sm)
    for _ in range(3):
        b, zb = _attend(sm)
        assert torch.equal(a, b) and torch.equal(za, zb)


def test_lse_may_be_left_out():
    sm = Small([3], [100])
    assert torch.equal(_attend(sm, lse=False)[0], _attend(sm)[0])


def test_attention_on_another_stream():
    sm = Small([2, 150], [700, 650], 2, 4, 128)
    want = _attend(sm)[0]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert torch.equal(_attend(sm, stream=s)[0], want)


def test_a_graph_follows_the_lengths():
    """A captured call reads lengths, tables and queries anew."""
    sm = Small([1, 1], [700, 300], 2, 4, 128)
    step, q, _, _, cache = sm.on_gpu(kvs, decode=True)
    out, z = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.zeros(kvs.kvs_attend_workspace(step, q.shape[1]), dtype=torch.uint8, device="cuda")
    out, lens = torch.zeros(2, sm.H * sm.G, sm.D, dtype=q.dtype, device="cuda"), step._keep[1]
    s = torch.cuda.Stream()
    kvs.kvs_attend(step, 0, q, out, z, None, True, 0, ws, s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        kvs.kvs_attend(step, 0, q, out, z, None, True, 0, ws, torch.cuda.current_stream())
    for lengths in ([700, 300], [699, 1], [33, 0]):
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        sm.lens = lengths
        want, bound, *_ = sm.attend(sm.D ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()


def test_out_of_bounds_entries_are_recorded_and_not_followed():
    sm = Small([1, 1], [40, 40], 2, 4, 64)
    sm.tables[1, 1] = sm.num_blocks
    with pytest.raises(kvs.KvsError) as ei:
        _attend(sm, decode=True)
    assert ei.value.code == kvs.KVS_ERR_BOUNDS
    good = Small([1, 1], [40, 40], 2, 4, 64)
    assert torch.equal(_attend(good, decode=True)[0], _attend(good, decode=True)[0])     # the word is clear again
    step, q, _, _, _ = good.on_gpu(kvs)
    out = torch.full_like(q, 7.0).contiguous()
    step._keep[1][1] = step.max_kv + 1
    ws = torch.zeros(kvs.kvs_attend_workspace(step, q.shape[1]) + 16, dtype=torch.uint8, device="cuda")
    kvs.kvs_attend(step, 0, q, out, None, None, True, 0, ws)
    with pytest.raises(kvs.KvsError):
        kvs.kvs_check_errors()
    assert (out[1] == 7.0).all() or (out[1] == 0.0).all()


# ---- weights ----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens,H,G,D,B,causal,window,decay", [
    ([1, 1, 1], [1, 130, 700], 2, 4, 128, 16, True, 0, 0.5), ([1], [257], 1, 1, 64, 1, True, 0, 1.0), ([3, 0, 40], [50, 9, 300], 2, 7, 80, 16, True, 0, 0.0),
    ([130], [128], 2, 4, 64, 16, True, 0, 0.9), ([200, 1], [600, 600], 1, 5, 128, 32, True, 100, 0.9), ([20], [90], 2, 3, 96, 3, False, 0, 1.0),
    ([260], [900], 1, 8, 128, 16, True, 0, 1.0), ([4], [0], 2, 2, 64, 16, True, 0, 1.0), ([7], [300], 1, 40, 128, 16, False, 5, 0.25)])
def test_weights(dtype, new, lens, H, G, D, B, causal, window, decay):
    sm = Small(new, lens, H, G, D, B, dtype)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    scale = D ** -0.5
    lse = sm.attend(scale, causal, window)[2].astype(np.float32)
    S = max(max(lens), 1) + 3
    before = np.random.default_rng(1).random((sm.R, H, S)).astype(np.float32)
    step.step.max_kv = step.max_kv = max(lens)
    w = torch.from_numpy(before).cuda()
    if decay == 0.0:
        w[:] = float("nan")
    kvs.kvs_weigh(step, 0, q, torch.from_numpy(lse).cuda(), w, None, decay, causal, window, None, kvs.KVS_F_VALIDATE)
    want, bound = sm.weigh(lse, before, decay, scale, causal, window)
    got = w.double().cpu().numpy()
    for r, T in enumerate(lens):
        off = np.abs(got[r, :, :T] - want[r, :, :T])
        assert (off <= bound[r, :, :T]).all(), (off / bound[r, :, :T]).max()
        rest = w.cpu().numpy()[r, :, T:]
        assert np.isnan(rest).all() if decay == 0.0 else (rest == before[r, :, T:]).all()


def test_weights_add_up_to_the_rows():
    """Every row spreads a weight of one over the tokens it sees."""
    sm = Small([3, 150], [700, 420], 2, 4, 128)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    ws = torch.empty(kvs.kvs_attend_workspace(step, q.shape[1]), dtype=torch.uint8, device="cuda")
    kvs.kvs_attend(step, 0, q, out, z, workspace=ws)
    w = torch.zeros(2, 2, step.max_kv, device="cuda")
    kvs.kvs_weigh(step, 0, q, z, w)
    total = w.double().sum(-1).cpu().numpy()
    rows = np.array(sm.new)[:, None] * sm.G
    assert (np.abs(total / rows - 1) < 1e-4).all()


# ---- append -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,rot,inter", [(128, 128, False), (128, 64, False), (128, 128, True), (64, 64, False), (80, 80, False), (80, 20, True),
                                         (96, 24, False), (8, 8, False), (8, 2, True), (120, 40, False), (128, 6, False), (72, 32, False)])
@pytest.mark.parametrize("new,lens", [([1, 1], [1, 40]), ([3, 0, 33], [3, 7, 100])])
def test_append(dtype, D, rot, inter, new, lens):
    sm = Small(new, lens, 2, 3, D, dtype=dtype)
    step, q, k, v, cache = sm.on_gpu(kvs, decode=new == [1, 1])
    turns, scale = kvs.kvs_rope_turns(rot, 10000.0)
    positions = np.random.default_rng(2).integers(0, 200000, sm.N).astype(np.int32)
    positions[0] = 1 << 24
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), rot, inter, 1.5)
    q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    before = cache.clone()
    kvs.kvs_append(step, 0, q, k, v, q_out, rope, torch.from_numpy(positions).cuda(), None, kvs.KVS_F_VALIDATE)
    want = before.view(2, -1, sm.H, D).clone()
    at = np.concatenate([sm.slots(r, np.arange(T - n, T)) for r, (n, T) in enumerate(zip(new, lens))])
    unit = ops_ref.UNIT[dtype]
    got_k = cache.view(2, -1, sm.H, D)[0, at]
    for x, got in ((q, q_out), (k, got_k)):
        x = x.double().cpu().numpy()
        y = ops_ref.rotate(x, positions, turns, rot, inter, 1.5)
        y[..., rot:] = x[..., rot:]
        off = np.abs(got.double().cpu().numpy() - y)
        big = np.abs(x).max(-1, keepdims=True)
        assert (off <= unit * np.abs(y) + 1.5 * 2.0 ** -19 * big + 2.0 ** -25).all()
        assert (off[..., rot:] == 0).all()
    want[0, at], want[1, at] = got_k, v
    assert torch.equal(cache.view(torch.int16), want.view(cache.shape).view(torch.int16))


def test_append_in_place_without_rope_and_without_queries():
    sm = Small([4], [20], 2, 3, 64)
    step, q, k, v, cache = sm.on_gpu(kvs)
    at = sm.slots(0, np.arange(16, 20))
    kvs.kvs_append(step, 0, None, k, v)
    flat = cache.view(2, -1, sm.H, sm.D)
    assert torch.equal(flat[0, at], k) and torch.equal(flat[1, at], v)
    turns, _ = kvs.kvs_rope_turns(64)
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), 64)
    out = torch.empty_like(q).contiguous()
    kvs.kvs_append(step, 0, q, k, v, out, rope)
    kvs.kvs_append(step, 0, q, k, v, None, rope)                  # positions: the tokens' places
    assert torch.equal(q, out)
    pos = torch.arange(16, 20, dtype=torch.int32, device="cuda")
    step2, q2, k2, v2, _ = sm.on_gpu(kvs)
    kvs.kvs_append(step2, 0, q2, k2, v2, out, rope, pos)
    assert torch.equal(q, out)


def test_tokens_beyond_the_cache_are_not_appended():
    sm = Small([5], [3], 2, 2, 64)
    step, q, k, v, cache = sm.on_gpu(kvs)
    before = cache.clone()
    kvs.kvs_append(step, 0, q, k, v, None, None, None, None, kvs.KVS_F_VALIDATE)
    at = sm.slots(0, np.arange(3))
    want = before.view(2, -1, sm.H, sm.D)
    want[0, at], want[1, at] = k[2:], v[2:]
    assert torch.equal(cache.view(torch.int16), before.view(torch.int16))


# ---- eviction ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens,budget,sinks,recent,B,D,L,H", [
    ([100, 37, 0, 1], 40, 4, 8, 16, 64, 2, 2), ([3000, 1025], 1024, 0, 0, 16, 128, 1, 3), ([513], 1, 0, 1, 8, 80, 3, 1),
    ([600, 599], 77, 70, 7, 1, 8, 2, 2), ([65, 2048], 64, 1, 0, 32, 96, 1, 4)])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
def test_evict(dtype, lens, budget, sinks, recent, B, D, L, H, kind):
    Wd = -(-budget // B)
    R = len(lens)
    sm = Small([0] * R, lens, H, 1, D, B, dtype, L=L, extra_blocks=R * Wd + 3)
    step, _, _, _, cache = sm.on_gpu(kvs)
    rng = np.random.default_rng(3)
    S = step.max_kv + 5
    w = rng.random((L, R, H, S)).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 4).astype(np.float32)
    if kind == "odd":
        pick = rng.integers(0, 8, w.shape)
        w = np.where(pick == 0, np.nan, np.where(pick == 1, np.inf, np.where(pick == 2, -w, np.where(pick == 3, -0.0, np.where(pick == 4, 0.0, w))))).astype(np.float32)
        w[..., 1::7] = -np.inf
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())
    dst = torch.from_numpy(rng.permutation(free)[: R * Wd].reshape(R, Wd).astype(np.int32))
    kept = torch.full((L, R, H, budget), -7, dtype=torch.int32, device="cuda")
    nw = torch.full((L, R, H, budget), -7.0, device="cuda")
    nl = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    before = cache.clone()
    kvs.kvs_evict(step, torch.from_numpy(w).cuda(), dst.cuda(), budget, sinks, recent, kept, nw, nl, None, kvs.KVS_F_VALIDATE)
    want = ops_ref.evict(w, lens, budget, sinks, recent)
    assert (kept.cpu().numpy() == want).all()
    assert nl.tolist() == [min(T, budget) for T in lens]
    want_w, flat = np.zeros(want.shape, np.float32), before.view(2 * L, -1, H, D).clone()
    src = before.view(2 * L, -1, H, D)
    for l in range(L):
        for r in range(R):
            J = min(lens[r], budget)
            if not J:
                continue
            j = np.arange(J)
            to = torch.from_numpy(dst[r].numpy().astype(np.int64)[j // B] * B + j % B).cuda()
            for h in range(H):
                want_w[l, r, h, :J] = w[l, r, h, want[l, r, h, :J]]
                at = torch.from_numpy(sm.slots(r, want[l, r, h, :J])).cuda()
                for p in (2 * l, 2 * l + 1):
                    flat[p, to, h] = src[p, at, h]
    assert np.array_equal(nw.cpu().numpy().view(np.uint32), want_w.view(np.uint32))
    assert torch.equal(cache.view(torch.int16), flat.view(cache.shape).view(torch.int16))


def test_a_step_through_all_operators():
    """Append, attend, weigh, evict, and attend again over what was kept: with every token kept,
    the second attention is the first."""
    sm = Small([3, 1], [90, 64], 2, 4, 64, extra_blocks=20)
    step, q, k, v, cache = sm.on_gpu(kvs)
    turns, scale = kvs.kvs_rope_turns(64)
    kvs.kvs_append(step, 0, q, k, v, None, kvs.Rope(torch.from_numpy(turns).cuda(), 64, scale=scale))
    out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    kvs.kvs_attend(step, 0, q, out, z, workspace=torch.empty(kvs.kvs_attend_workspace(step, 8), dtype=torch.uint8, device="cuda"))
    w = torch.zeros(1, 2, 2, step.max_kv, device="cuda")
    kvs.kvs_weigh(step, 0, q, z, w[0])
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:12].reshape(2, 6)
    dst = torch.from_numpy(free.astype(np.int32)).cuda()
    kept = torch.empty(1, 2, 2, 96, dtype=torch.int32, device="cuda")
    lens = torch.empty(2, dtype=torch.int32, device="cuda")
    kvs.kvs_evict(step, w, dst, 96, 4, 8, kept, None, lens)
    again = kvs.Step((1, 2, 64, 2, 16, 16), [cache[0], cache[1]], sm.num_blocks, dst, lens, step._keep[2], total_q=4, max_q=3)
    out2 = torch.empty_like(out)
    kvs.kvs_attend(again, 0, q, out2, workspace=torch.empty(kvs.kvs_attend_workspace(again, 8) + 16, dtype=torch.uint8, device="cuda"))
    assert torch.equal(out, out2)


def test_a_model_on_a_retrieved_prefix():
    """The example's serving loop: a suffix on a retrieved prefix gives what the whole prompt's prefill gives."""
    from paper_2609_35065_gb300 import prefix_step
    for dtype in (torch.bfloat16, torch.float16):
        r = prefix_step.run(prefix_step.Config(dtype=dtype))
        # every rounding of the residual stream (4 layers, 3 products each, 8 or 11 bits) may differ once
        unit = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
        assert (r["suffix"] - r["whole"]).norm() <= 12 * unit * r["whole"].norm()
        assert r["stored"] == 512 and len(r["suffix"]) == 178
        kept = r["kept"].cpu().numpy()
        T = r["cached"]
        assert (np.diff(kept, axis=-1) > 0).all() and (kept[..., :4] == np.arange(4)).all() and (kept[..., -64:] == np.arange(T - 64, T)).all()
        assert torch.isfinite(r["weights"]).all() and len(r["tokens"]) == 24


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 300])
@pytest.mark.parametrize("new,lens", [([1, 5], [500, 3]), ([200, 130], [700, 60])])
def test_a_window_beyond_every_position_hides_nothing(new, lens, window):
    """Also where a request's first rows lie before its first cached token."""
    sm = Small(new, lens, 2, 4, 64)
    (a, za), (b, zb) = _attend(sm), _attend(sm, window=window)
    assert torch.equal(a, b) and torch.equal(za, zb)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    w = torch.zeros(2, 2, 2, step.max_kv, device="cuda")
    kvs.kvs_weigh(step, 0, q, za, w[0])
    kvs.kvs_weigh(step, 0, q, za, w[1], window=window)
    assert torch.equal(w[0], w[1])


@pytest.mark.parametrize("G,D,dtype", [(9, 128, "bf16"), (16, 64, "f16"), (17, 128, "f16"), (31, 80, "bf16"), (48, 64, "bf16"), (64, 128, "bf16"), (65, 96, "f16"),
                                       (128, 64, "f16"), (129, 128, "bf16")])
def test_weights_of_wide_groups(G, D, dtype):
    """Nine to some hundred packed rows of a decode step, and of two new tokens."""
    for new, lens in (([1, 1, 1], [129, 1, 700]), ([2, 0, 1], [300, 77, 15])):
        sm = Small(new, lens, 1, G, D, dtype=dtype)
        z = torch.from_numpy(sm.attend(D ** -0.5)[2].astype(np.float32))
        rng = np.random.default_rng(5)
        step, q, _, _, _cache = sm.on_gpu(kvs)
        before = rng.random((3, 1, step.max_kv)).astype(np.float32)
        w = torch.from_numpy(before).cuda()
        kvs.kvs_weigh(step, 0, q, z.cuda(), w, decay=0.9, flags=kvs.KVS_F_VALIDATE)
        want, bound = sm.weigh(z.numpy(), before, float(np.float32(0.9)), D ** -0.5)
        off = np.abs(w.double().cpu().numpy() - want)
        assert (off <= bound).all(), (off - bound).max()


@pytest.mark.parametrize("new,lens,window", [([1], [1000], 0), ([3], [2500], 0), ([1, 1], [5000, 0], 0), ([2, 0, 1], [900, 3000, 40], 0), ([2], [4000], 300), ([5], [3], 0),
                                             ([30], [2000], 0), ([64, 9], [1500, 700], 0), ([100], [5000], 333), ([20, 70], [0, 2600], 0), ([250], [900], 0)])
@pytest.mark.parametrize("G,D,dtype", [(1, 8, "f16"), (4, 64, "bf16"), (5, 80, "bf16"), (7, 128, "f16"), (3, 120, "f16")])
def test_one_head_in_parts(new, lens, window, G, D, dtype):
    """Few heads: a head's keys are split, some of the parts see nothing of some rows, or are empty."""
    _check_attend(Small(new, lens, 1, G, D, dtype=dtype), window=window)


@pytest.mark.parametrize("kind", ["random", "ties"])
def test_evict_from_caches_of_more_than_16384_tokens(kind):
    lens, budget, B = [20000, 16385, 300], 5000, 16
    Wd = -(-budget // B)
    sm = Small([0] * 3, lens, 2, 1, 8, B, extra_blocks=3 * Wd)
    step, _, _, _, cache = sm.on_gpu(kvs)
    w = np.random.default_rng(4).random((1, 3, 2, step.max_kv)).astype(np.float32)
    if kind == "ties":
        w = np.floor(w * 3).astype(np.float32)
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())
    dst = torch.from_numpy(free[: 3 * Wd].reshape(3, Wd).astype(np.int32))
    kept = torch.full((1, 3, 2, budget), -7, dtype=torch.int32, device="cuda")
    nw, nl = torch.full(kept.shape, -7.0, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    kvs.kvs_evict(step, torch.from_numpy(w).cuda(), dst.cuda(), budget, 4, 100, kept, nw, nl, None, kvs.KVS_F_VALIDATE)
    want = ops_ref.evict(w, lens, budget, 4, 100)
    assert (kept.cpu().numpy() == want).all() and nl.tolist() == [5000, 5000, 300]
    flat = cache.view(2, -1, 2, 8)
    for r in range(3):
        j = np.arange(min(lens[r], budget))
        to = torch.from_numpy(dst[r].numpy().astype(np.int64)[j // B] * B + j % B).cuda()
        for h in range(2):
            assert (nw[0, r, h, : len(j)].cpu().numpy() == w[0, r, h, want[0, r, h, : len(j)]]).all()
            at = torch.from_numpy(sm.slots(r, want[0, r, h, : len(j)])).cuda()
            assert torch.equal(flat[:, to, h], flat[:, at, h])


@pytest.mark.parametrize("new,lens", [([1, 2], [600, 33]), ([30, 1], [600, 33]), ([200, 130], [600, 200])])
def test_offsets_beyond_32_bits(new, lens):
    """Blocks at the end of planes of more than 2^31 elements: what the same blocks give in small planes."""
    sm = Small(new, lens, 8, 4, 128, extra_blocks=60)
    step, q, k, v, cache = sm.on_gpu(kvs)
    NB = (1 << 31) // (16 * 8 * 128) + 200
    shift = NB - sm.num_blocks
    far = torch.empty(2, NB, 16, 8, 128, dtype=cache.dtype, device="cuda")
    far[:, shift:] = cache
    tables, kv_lens, starts = step._keep[:3]
    step2 = kvs.Step((1, 8, 128, 2, 16, 16), [far[0].data_ptr(), far[1].data_ptr()], NB, tables + shift, kv_lens, starts, total_q=sm.N, max_q=max(new))
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:20].reshape(2, 10)
    dst = torch.from_numpy(free.astype(np.int32)).cuda()
    got = []
    for s, d in ((step, dst), (step2, dst + shift)):
        kvs.kvs_append(s, 0, None, k, v)
        out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(q.shape[:2], device="cuda")
        kvs.kvs_attend(s, 0, q, out, z, workspace=torch.empty(kvs.kvs_attend_workspace(s, 32), dtype=torch.uint8, device="cuda"))
        w = torch.zeros(1, 2, 8, s.max_kv, device="cuda")
        kvs.kvs_weigh(s, 0, q, z, w[0])
        kept = torch.empty(1, 2, 8, 160, dtype=torch.int32, device="cuda")
        kvs.kvs_evict(s, w, d, 160, 4, 8, kept, flags=kvs.KVS_F_VALIDATE)
        got.append((out, z, w, kept))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.equal(far[:, shift:].view(torch.int16), cache.view(torch.int16))


def test_a_graph_of_a_decode_step():
    """Append, attention in parts, weights and eviction, captured once and replayed after the lengths changed."""
    sm = Small([1, 1], [4000, 900], 1, 4, 64, extra_blocks=60)
    step, q, k, v, cache = sm.on_gpu(kvs, decode=True)
    q = q.contiguous()
    out, z = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.zeros(kvs.kvs_attend_workspace(step, 4) + 16, dtype=torch.uint8, device="cuda")
    w = torch.zeros(1, 2, 1, step.max_kv, device="cuda")
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:20].reshape(2, 10)
    dst, kept = torch.from_numpy(free.astype(np.int32)).cuda(), torch.zeros(1, 2, 1, 160, dtype=torch.int32, device="cuda")

    def run(s):
        kvs.kvs_append(step, 0, None, k, v, stream=s)
        kvs.kvs_attend(step, 0, q, out, z, workspace=ws, stream=s)
        kvs.kvs_weigh(step, 0, q, z, w[0], decay=0.0, stream=s)
        kvs.kvs_evict(step, w, dst, 160, 4, 8, kept, stream=s)

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    run(s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        run(torch.cuda.current_stream())
    for lengths in ([4000, 900], [3999, 1], [0, 700]):
        step._keep[1].copy_(torch.tensor(lengths, dtype=torch.int32))
        run(s)
        s.synchronize()
        want = [x.clone() for x in (out, z, w, kept, cache)]
        for x in (out, z, w, kept):
            x.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, z, kept), want[:2] + want[3:4]):
            assert torch.equal(x, y)
        for r, T in enumerate(lengths):
            assert torch.equal(w[:, r, :, :T], want[2][:, r, :, :T])
        assert torch.equal(cache.view(torch.int16), want[4].view(torch.int16))


@pytest.mark.parametrize("new,T,G,D,dtype", [(650, 900, 4, 128, "bf16"), (645, 645, 4, 64, "f16"), (300, 1000, 9, 80, "bf16")])
def test_weights_of_long_chunks(new, T, G, D, dtype):
    """More rows than a small grid of key tiles has, around where a CTA takes two of them."""
    sm = Small([new, 3], [T, 130], 1, G, D, dtype=dtype)
    z = torch.from_numpy(sm.attend(D ** -0.5)[2].astype(np.float32))
    step, q, _, _, _cache = sm.on_gpu(kvs)
    before = np.random.default_rng(6).random((2, 1, step.max_kv)).astype(np.float32)
    w = torch.from_numpy(before).cuda()
    kvs.kvs_weigh(step, 0, q, z.cuda(), w, decay=0.5, flags=kvs.KVS_F_VALIDATE)
    want, bound = sm.weigh(z.numpy(), before, 0.5, D ** -0.5)
    off = np.abs(w.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off - bound).max()


def _in_padded_rows(sm, lead, trail):
    """Step, q, k, v and cache of `sm` in tensors with rows before its first and behind its last request."""
    step, q, k, v, cache = sm.on_gpu(kvs)
    rows = lead + sm.N + trail
    starts = step._keep[2] + lead
    padded = kvs.Step((sm.L, sm.H, sm.D, 2, sm.B, sm.B), [cache[p].data_ptr() for p in range(2 * sm.L)], sm.num_blocks, step._keep[0], step._keep[1], starts,
                      total_q=rows, max_q=max(sm.new + [0]), dtype=step.step.dtype)

    def pad(x):
        y = torch.full((rows, *x.shape[1:]), 3.0, dtype=x.dtype, device="cuda")
        y[lead: lead + sm.N] = x
        return y
    return padded, pad(q), pad(k), pad(v), cache


# the three ways to an output row: one part, parts joined by their cluster, parts joined by a kernel
@pytest.mark.parametrize("new,lens,H,ways", [([1, 2], [100, 60], 2, "one"), ([40, 1], [120, 60], 8, "one"), ([1], [1000], 1, "cluster"), ([20], [1000], 1, "cluster"),
                                             ([2, 1], [20000, 300], 1, "join"), ([140], [8200], 1, "join"), ([1, 140, 0], [5, 8200, 0], 1, "join")])
def test_rows_of_no_request_keep_what_they_hold(new, lens, H, ways):
    """Rows before q_starts[0] and behind its last entry are another call's."""
    sm = Small(new, lens, H, 4, 128)
    want, z_want = _attend(sm)
    step, q, _, _, _cache = _in_padded_rows(sm, 3, 5)
    need = kvs.kvs_attend_workspace(step, q.shape[1])
    assert (need > 0) == (ways == "join")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    z = torch.full(q.shape[:2], 7.0, device="cuda")
    kvs.kvs_attend(step, 0, q, out, z, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"), flags=kvs.KVS_F_VALIDATE)
    mine = slice(3, 3 + sm.N)
    assert torch.equal(out[mine], want) and torch.equal(z[mine], z_want)
    for x in (out, z):
        assert (x[:3] == 7.0).all() and (x[3 + sm.N:] == 7.0).all()


@pytest.mark.parametrize("rot,inter", [(64, False), (20, False), (64, True)])
@pytest.mark.parametrize("new,lens", [([3, 0, 4], [9, 0, 4]), ([5], [3]), ([1] * 40, [7] * 40)])
def test_append_leaves_rows_of_no_request_alone(new, lens, rot, inter):
    """Two calls for the two halves of a tensor's rows rotate each of its queries once."""
    sm = Small(new, lens, 2, 3, 64)
    turns, _ = kvs.kvs_rope_turns(rot)
    rope = kvs.Rope(torch.from_numpy(turns).cuda(), rot, inter)
    step, q, k, v, cache = sm.on_gpu(kvs)
    want = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    kvs.kvs_append(step, 0, q, k, v, want, rope)
    kept = cache.clone()
    step, q, k, v, cache = _in_padded_rows(sm, 3, 5)
    mine = slice(3, 3 + sm.N)
    for out in (torch.full_like(q, 3.0), None):
        kvs.kvs_append(step, 0, q, k, v, out, rope, flags=kvs.KVS_F_VALIDATE)
        x = q if out is None else out
        assert torch.equal(x[mine], want)
        assert (x[:3] == 3.0).all() and (x[3 + sm.N:] == 3.0).all()
    assert torch.equal(cache.view(torch.int16), kept.view(torch.int16))


def _with_starts(sm, starts, max_q):
    step, q, k, v, cache = sm.on_gpu(kvs)
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    return kvs.Step((sm.L, sm.H, sm.D, 2, sm.B, sm.B), [cache[p].data_ptr() for p in range(2 * sm.L)], sm.num_blocks, step._keep[0], step._keep[1], s,
                    total_q=sm.N, max_q=max_q), q, k, v, cache


@pytest.mark.parametrize("op", ["append", "attend", "weigh"])
@pytest.mark.parametrize("starts,lens", [([0, 5, 3, 8], [20, 20, 20]), ([0, 3, 4, 9], [20, 20, 20]), ([-1, 3, 4, 8], [20, 20, 20]), ([0, 3, 3, 8], [20, 33, 20]),
                                         ([0, 3, 8, 8], [20, 20, -1]), ([0, 0, 8, 8], [-5, 20, 20])])
def test_every_operator_records_a_request_out_of_bounds(op, starts, lens):
    """Row ranges that fall, overlap or leave the tensor, and lengths out of bounds, also of requests without rows."""
    sm = Small([3, 2, 3], [20, 20, 20], 2, 2, 64, B=16)
    step, q, k, v, cache = _with_starts(sm, starts, 8)
    step._keep[1].copy_(torch.tensor(lens, dtype=torch.int32))
    before = cache.clone()
    out, z = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ws = torch.empty(kvs.kvs_attend_workspace(step, 4), dtype=torch.uint8, device="cuda")
    w = torch.zeros(3, 2, step.max_kv, device="cuda")
    call = {"append": lambda: kvs.kvs_append(step, 0, None, k, v, flags=kvs.KVS_F_VALIDATE),
            "attend": lambda: kvs.kvs_attend(step, 0, q, out, z, workspace=ws, flags=kvs.KVS_F_VALIDATE),
            "weigh": lambda: kvs.kvs_weigh(step, 0, q, z, w, flags=kvs.KVS_F_VALIDATE)}[op]
    with pytest.raises(kvs.KvsError) as ei:
        call()
    assert ei.value.code == kvs.KVS_ERR_BOUNDS
    used = np.concatenate([sm.slots(r, np.arange(20)) for r in range(3)])
    rest = torch.from_numpy(np.setdiff1d(np.arange(sm.num_blocks * sm.B), used)).cuda()
    flat, flat_before = (x.view(2, -1, sm.H, sm.D).view(torch.int16) for x in (cache, before))
    assert torch.equal(flat[:, rest], flat_before[:, rest])


def test_eviction_from_empty_caches_is_over_when_the_stream_has_passed_it():
    """Nothing is kept, so that the copy has nothing to wait for but the selection, which writes `kept`."""
    L, R, H, budget = 8, 64, 4, 500
    sm = Small([0] * R, [0] * R, H, 1, 64, L=L, extra_blocks=R * 40)
    lens = torch.zeros(R, dtype=torch.int32, device="cuda")
    cache = sm.cache.cuda()
    tables = torch.zeros(R, 40, dtype=torch.int32, device="cuda")
    dst = torch.ones(R, 40, dtype=torch.int32, device="cuda")
    step = kvs.Step((L, H, 64, 2, 16, 16), [cache[p].data_ptr() for p in range(2 * L)], sm.num_blocks, tables, lens, total_q=0, max_q=0)
    w = torch.zeros(L, R, H, step.max_kv, device="cuda")
    kept = torch.empty(L, R, H, budget, dtype=torch.int32, device="cuda")
    nw, nl = torch.empty(kept.shape, device="cuda"), torch.empty(R, dtype=torch.int32, device="cuda")
    for _ in range(20):
        for x in (kept, nw, nl):
            x.fill_(7)
        kvs.kvs_evict(step, w, dst, budget, 4, 8, kept, nw, nl)
        copies = [x.clone() for x in (kept, nw, nl)]              # right behind the copy
        assert (copies[0] == -1).all() and (copies[1] == 0).all() and (copies[2] == 0).all()
    kvs.kvs_check_errors()


@pytest.mark.parametrize("digits", [15, 20, 26, 30])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,T,H", [(1, 40000, 1), (1, 1500, 4), (3, 300, 8), (40, 30000, 1), (150, 9000, 2), (150, 3000, 38)])
def test_a_heavy_token_before_many_light_ones(new, T, H, dtype, digits):
    """The first token has 2^digits times the weight of any other, and a value of zero: what comes out
    is what the light ones add up to.  Half rounds weights to multiples of 2^-24, of which the heaviest one's
    is 2^8 for few rows, and for many 2^3 or the tokens' number by 2^10."""
    sm = Small([new], [T], H, 4, 64, dtype=dtype)
    at = torch.from_numpy(sm.slots(0, np.arange(T)))
    sm.cache[:, at] = 0.0
    sm.cache[0, at[0], :, 0] = digits * np.log(2.0)
    sm.cache[1, at[1:]] = 1.0
    sm.qkv[:] = 0.0
    sm.parts(sm.qkv)[0][:, :, 0] = 1.0
    out, _ = _attend(sm, scale=1.0)
    want, bound, _, _ = sm.attend(1.0)
    if dtype == "f16":
        # the rounding of the weights, and of an output below half's normal numbers
        heaviest = 2.0 ** 8 if new * sm.G <= 16 else max(2.0 ** 3, T / 2.0 ** 10)
        bound = bound - T * 2.0 ** -25 + T * 2.0 ** -25 / heaviest + 2.0 ** -25
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens,H,G,D", [([1, 1], [900, 300], 2, 4, 128), ([1], [5000], 1, 8, 64), ([2, 3], [700, 90], 2, 5, 80), ([4], [3000], 1, 4, 128), ([1], [20000], 1, 1, 96)])
def test_few_rows_lose_nothing_by_rounding_weights(new, lens, H, G, D, dtype):
    """Up to 16 packed rows a weight goes into the product with V as two 16-bit numbers, so that what is off
    is the output's own rounding, and the square of the type's of the weights."""
    sm = Small(new, lens, H, G, D, dtype=dtype)
    out, _ = _attend(sm)
    want, bound, _, _ = sm.attend(D ** -0.5)
    mean = Small(new, lens, H, G, D, dtype=dtype)
    mean.cache[1] = mean.cache[1].abs()
    a = mean.attend(D ** -0.5)[0]                                # the mean of |v|
    u = ops_ref.UNIT[dtype]
    bound = bound - 1.01 * u * a + u * u * a
    if dtype == "f16":
        bound = bound + 2.0 ** -25                               # of an output below half's normal numbers
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= bound).all(), (off / bound).max()


# ---- what a request does not see, and what its neighbours hold ---------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens", [([2, 1, 3], [700, 650, 350]), ([5, 30, 4], [700, 650, 350]), ([33, 150, 7], [300, 650, 90])])
def test_the_neighbours_of_a_request_do_not_matter(new, lens, dtype):
    """The middle request's rows have the same bits whatever the requests around it hold, queries that are not
    numbers right before and behind it among that."""
    got = []
    for fill in (None, 1.0, float("nan"), float("inf")):
        sm = Small(new, lens, 2, 5, 128, dtype=dtype)
        rows = slice(sm.starts[1], sm.starts[2])
        if fill is not None:
            for r in (0, 2):
                sm.qkv[sm.starts[r]: sm.starts[r + 1]] = fill
                sm.cache[:, torch.from_numpy(sm.slots(r, np.arange(lens[r])))] = fill
        out, z = _attend(sm)
        step, q, _, _, _cache = sm.on_gpu(kvs)
        w = torch.ones(3, 2, step.max_kv, device="cuda")
        kvs.kvs_weigh(step, 0, q, z, w, decay=0.5, flags=kvs.KVS_F_VALIDATE)
        got.append((out[rows], z[rows], w[1]))
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,G", [(128, 4), (64, 3)])
@pytest.mark.parametrize("new,T,window", [(1, 700, 100), (1, 20000, 300), (3, 500, 129), (30, 900, 64), (200, 1500, 200), (130, 4000, 17)])
def test_tokens_before_the_window_may_be_anything(new, T, window, D, G, dtype):
    """Keys and values that no row of the request sees are not numbers, and reach neither outputs nor weights."""
    sm = Small([new, 2], [T, 60], 2, G, D, dtype=dtype)
    first = T - new + 1 - window
    sm.cache[:, torch.from_numpy(sm.slots(0, np.arange(first)))] = float("nan")
    want = Small([new, 2], [T, 60], 2, G, D, dtype=dtype)
    want.cache[:, torch.from_numpy(want.slots(0, np.arange(first)))] = 0.5
    scale = D ** -0.5
    ref, bound, lse, _ = want.attend(scale, True, window)
    out, z = _attend(sm, window=window)
    assert (np.abs(out.double().cpu().numpy() - ref) <= bound).all()
    step, q, _, _, _cache = sm.on_gpu(kvs)
    w = torch.full((2, 2, step.max_kv), 2.0, device="cuda")
    kvs.kvs_weigh(step, 0, q, torch.from_numpy(lse.astype(np.float32)).cuda(), w, decay=0.5, window=window, flags=kvs.KVS_F_VALIDATE)
    before = np.full((2, 2, step.max_kv), 2.0, np.float32)
    ref_w, bound_w = want.weigh(lse.astype(np.float32), before, 0.5, scale, True, window)
    for r, n in enumerate((T, 60)):
        assert (np.abs(w[r, :, :n].double().cpu().numpy() - ref_w[r, :, :n]) <= bound_w[r, :, :n]).all()
    assert (w[0, :, :first] == 1.0).all()


# ---- entries out of bounds, found on the device -------------------------------
@pytest.mark.parametrize("op", ["append", "weigh"])
@pytest.mark.parametrize("new", [1, 3, 50])
@pytest.mark.parametrize("what", ["length", "block", "negative block"])
def test_out_of_bounds_entries_leave_the_other_requests_right(op, new, what):
    """One request names a block that there is not, or has a length beyond max_kv: it alone is left out."""
    lens = [130, 90]
    good = Small([new, new], lens, 2, 4, 64)
    bad = Small([new, new], lens, 2, 4, 64)
    blk = 89 // bad.B                                             # of the last token, a new one
    if what != "length":
        bad.tables[1, blk] = bad.num_blocks if what == "block" else -1
    lse = good.attend(good.D ** -0.5)[2].astype(np.float32)
    got = []
    for sm in (good, bad):
        step, q, k, v, cache = sm.on_gpu(kvs)
        if sm is bad and what == "length":
            step._keep[1][1] = step.max_kv + 1
        w = torch.full((2, 2, step.max_kv), 3.0, device="cuda")
        flags = kvs.KVS_F_VALIDATE
        call = (lambda: kvs.kvs_append(step, 0, None, k, v, flags=flags)) if op == "append" else \
            (lambda: kvs.kvs_weigh(step, 0, q, torch.from_numpy(lse).cuda(), w, decay=0.0, flags=flags))
        if sm is bad:
            with pytest.raises(kvs.KvsError) as ei:
                call()
            assert ei.value.code == kvs.KVS_ERR_BOUNDS
        else:
            call()
        got.append((cache.view(2, -1, sm.H, sm.D).view(torch.int16), w))
    kvs.kvs_check_errors()                                        # the word is clear again
    (cache_a, w_a), (cache_b, w_b) = got
    if op == "weigh":
        assert torch.equal(w_a[0], w_b[0])
        if what == "length":
            assert (w_b[1] == 3.0).all()
        else:
            assert torch.equal(w_a[1, :, : blk * bad.B], w_b[1, :, : blk * bad.B])
        return
    before = good.cache.cuda().view(torch.int16)
    out = good.slots(1, np.arange(0 if what == "length" else blk * good.B, 90))
    keep = torch.from_numpy(np.setdiff1d(np.arange(good.num_blocks * good.B), out)).cuda()
    out = torch.from_numpy(out).cuda()
    assert torch.equal(cache_a[:, keep], cache_b[:, keep])
    assert torch.equal(cache_b[:, out], before[:, out])


@pytest.mark.parametrize("what", ["length", "source block", "new block"])
def test_eviction_with_entries_out_of_bounds(what):
    lens, budget, B, H, D = [100, 90], 48, 16, 2, 64
    sm = Small([0, 0], lens, H, 1, D, B, extra_blocks=10)
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:6].reshape(2, 3)
    dst = torch.from_numpy(free.astype(np.int32))
    if what == "source block":
        sm.tables[1, 2] = sm.num_blocks + 7
    if what == "new block":
        dst[1, 1] = -3
    step, _, _, _, cache = sm.on_gpu(kvs)
    if what == "length":
        step._keep[1][1] = step.max_kv + 1
    w = np.random.default_rng(8).random((1, 2, H, step.max_kv)).astype(np.float32)
    kept = torch.full((1, 2, H, budget), -7, dtype=torch.int32, device="cuda")
    nl = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    before = cache.clone()
    with pytest.raises(kvs.KvsError) as ei:
        kvs.kvs_evict(step, torch.from_numpy(w).cuda(), dst.cuda(), budget, 4, 8, kept, None, nl, None, kvs.KVS_F_VALIDATE)
    assert ei.value.code == kvs.KVS_ERR_BOUNDS
    want = ops_ref.evict(w, [100, 0 if what == "length" else 90], budget, 4, 8)
    assert (kept.cpu().numpy() == want).all() and nl.tolist() == [48, 0 if what == "length" else 48]
    flat = before.view(2, -1, H, D).clone()
    for r in range(2):
        for h in range(H):
            for j, t in enumerate(want[0, r, h]):
                b = int(dst[r, j // B])
                if t < 0 or b < 0:
                    continue
                blk = int(sm.tables[r, t // B])
                to = b * B + j % B
                flat[:, to, h] = before.view(2, -1, H, D)[:, blk * B + t % B, h] if blk < sm.num_blocks else 0.0
    assert torch.equal(cache.view(torch.int16), flat.view(cache.shape).view(torch.int16))


@pytest.mark.parametrize("L", [224, 225, 500])
def test_eviction_of_more_layers_than_a_launch_carries(L):
    lens, budget, B, H, D = [40, 7], 12, 4, 1, 8
    sm = Small([0, 0], lens, H, 1, D, B, L=L, extra_blocks=6)
    step, _, _, _, cache = sm.on_gpu(kvs)
    dst = torch.from_numpy(np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:6].reshape(2, 3).astype(np.int32))
    w = np.random.default_rng(9).random((L, 2, H, step.max_kv)).astype(np.float32)
    kept = torch.full((L, 2, H, budget), -7, dtype=torch.int32, device="cuda")
    before = cache.view(2 * L, -1, H, D).clone()
    launches = kvs.kvs_stat_launches()
    kvs.kvs_evict(step, torch.from_numpy(w).cuda(), dst.cuda(), budget, 1, 2, kept, flags=kvs.KVS_F_VALIDATE)
    assert kvs.kvs_stat_launches() - launches == 1 + -(-L // 224)
    want = ops_ref.evict(w, lens, budget, 1, 2)
    assert (kept.cpu().numpy() == want).all()
    for r, T in enumerate(lens):
        J = min(T, budget)
        j = np.arange(J)
        to = torch.from_numpy(dst[r].numpy().astype(np.int64)[j // B] * B + j % B).cuda()
        for l in range(L):
            at = torch.from_numpy(sm.slots(r, want[l, r, 0, :J])).cuda()
            before[2 * l: 2 * l + 2, to] = before[2 * l: 2 * l + 2, at]
    assert torch.equal(cache.view(torch.int16), before.view(cache.shape).view(torch.int16))
