"""The operators with axes and with sinks where a single binary32 number shows, on requests that have no new tokens, and
together with what comes before and after them."""
import numpy as np
import pytest
import torch

import ops_ref
from long_ref import Long
from paper_2609_35065_gb300 import kvs

pytestmark = pytest.mark.gpu
LOG2E = 1.4426950408889634


def _scales(near, count):
    """Binary32 scales from `near` / log2(e) up whose products with log2(e), taken in binary32, are 6e-8 of themselves too small."""
    found, s = [], np.float32(near / LOG2E)
    while len(found) < count:
        s = np.nextafter(s, np.float32(1))
        if float(s * np.float32(LOG2E)) < (1 - 6e-8) * float(s) * LOG2E:
            found.append(float(s))
    return found


class Exact(Long):
    """Sums of products that are exact in binary32, whatever their order and however many bits a sum keeps beyond 16: queries are
    +-1, the same for all heads, keys multiples of 1/32 below 8.  A new token's queries have `most` at most, 0.9 of that at least, as
    their product with its own key, and 0 with those of the tokens before the new ones."""

    def __init__(self, new, lens, window, sinks, G, D, dtype, most, seed=5):
        super().__init__(new, lens, window, sinks, 1, G, D, 16, dtype=dtype, given_back=False)
        self.cache.nan_to_num_(0.5)
        g = torch.Generator().manual_seed(seed)
        q = self.parts(self.qkv)[0]
        q.copy_((torch.randint(0, 2, (len(q), 1, D), generator=g) * 2 - 1).to(q.dtype))
        step = 2.0 ** -5
        top = int(most / D / step)
        for r, (n, T) in enumerate(zip(new, lens)):
            own = (torch.randint(int(0.9 * top) + 1, top + 1, (n, 1), generator=g) * step).to(q.dtype) * q[self.starts[r]: self.starts[r + 1], 0]
            self.cache[0, torch.from_numpy(self.slots(r, np.arange(T))), 0] = 0.0
            self.cache[0, torch.from_numpy(self.slots(r, np.arange(T - n, T))), 0] = own

    def lse(self, scale):
        """In 64 bits, [rows, heads]."""
        out = np.zeros((self.N, self.G))
        for r in range(self.R):
            for i in range(self.G):
                s = self.scores(r, 0, i, scale, True, self.window)[0]
                m = s.max(1, keepdims=True)
                out[self.starts[r]: self.starts[r + 1], i] = (m + np.log(np.exp(s - m).sum(1, keepdims=True)))[:, 0]
        return out

    def own(self, r):
        """Request r's new tokens."""
        return slice(self.lens[r] - self.new[r], self.lens[r])


# ---- the scale as it is given ----------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("new,window", [(3, 300), (16, 300), (40, 300), (400, 300), (400, 0)])
def test_weights_of_exact_scores(dtype, D, new, window):
    """Weights near 1, exponentials of a difference of two numbers below 32, of which the score is exact.  Off are: lse's product with
    log2(e) by 2^-20, the difference (below 1/4) and its correction by 2^-26 each, the exponential by 2^-22, and each addition to the
    sum of two such weights by 2^-23 or, where that is less, by what is added."""
    scale = _scales(2.0 ** -4, 1)[0]
    sm = Exact([new], [700], window, 4, 2, D, dtype, 508)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    lse = torch.from_numpy(sm.lse(scale)).float()
    assert 18 < lse.min() and lse.max() < 32 / LOG2E
    w = torch.zeros(1, 1, step.max_kv, device="cuda")
    kvs.kvs_weigh_sinks(step, 0, q, lse.cuda(), w, scale, 0.0, True, window, 4, flags=kvs.KVS_F_VALIDATE)
    each = np.concatenate([np.exp(sm.scores(0, 0, i, scale, True, window)[0] - lse[:, i, None].double().numpy()) for i in range(2)])
    want = each.sum(0)
    off = np.abs(w.double().cpu().numpy()[0, 0, :700] - want)
    bound = want * (np.log(2) * (2.0 ** -20 + 2 * 2.0 ** -26) + 2.0 ** -22) + np.minimum(each, 2.0 ** -23).sum(0)
    assert (off <= bound)[sm.own(0)].all(), (off / bound)[sm.own(0)].max()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("new,lens", [([1] * 40, list(range(300, 700, 10))), ([20], [700]), ([40, 3], [700, 400]), ([400], [700])])
def test_weights_with_the_lse_that_attention_returned(dtype, D, new, lens):
    """A new token's own weight is off by the roundings of lse and of its product with log2(e), whatever the scale: on average over many
    tokens and scales by little, as a mean of n independent errors of at most h each is off by more than h sqrt(2 ln(2 / p) / n) with a
    probability of p at most (Hoeffding).  h: 2^-20 of lse itself, and log2(e)'s multiple of it is rounded three times, by 2^-20 each (as
    the maximum times the scale, with the sum's logarithm, and as the weight's subtrahend); the exponentials, of lse's sum and of the weight,
    may be off by 2^-22 each, always alike.  Products are exact; scores come in 64ths of the largest at least, lse in far more."""
    sm = Exact(new, lens, 250, 4, 2, D, dtype, 508)
    scales = _scales(2.0 ** -4, 16)
    step, q, _, _, _cache = sm.on_gpu(kvs, decode=new == [1] * len(new))
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 2, True, 250, 4), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(q), torch.empty(sm.N, 2, device="cuda")
    off = []
    for scale in scales:
        w = torch.zeros(sm.R, 1, step.max_kv, device="cuda")
        kvs.kvs_attend_sinks(step, 0, q, out, z, scale, True, 250, 4, ws)
        kvs.kvs_weigh_sinks(step, 0, q, z, w, scale, 0.0, True, 250, 4, flags=kvs.KVS_F_VALIDATE)
        want, _ = sm.weigh(sm.lse(scale), np.zeros(w.shape), 0.0, scale, True, 250)
        got = w.double().cpu().numpy()
        off += [(got / np.where(want > 0, want, 1))[r, 0][sm.own(r)] - 1 for r in range(sm.R)]
    off = np.concatenate(off)
    h = np.sqrt(1 + 3 * np.log(2) ** 2) * 2.0 ** -20
    n = len(scales) * min(sm.N, len(np.unique(sm.lse(scales[0]).round(6))))
    bound = h * np.sqrt(2 * np.log(2 / 1e-6) / n) + 2 * 2.0 ** -22
    assert abs(off.mean()) <= bound, (off.mean(), bound)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 72, 128])
@pytest.mark.parametrize("signs", ["one", "both"])
def test_rows_of_heavy_tokens_add_up(signs, D, dtype):
    """Eight tokens have nearly all of the weight of rows whose lse is near 20, by products of one sign or of both.  Scores are not exact,
    but both calls cut their sums off alike, so that a row's weights add up to one but for roundings: those of
    test_weights_with_the_lse_that_attention_returned, and of up to 308 additions to either sum, by 2^-24 of it each."""
    new, T, G, window = 400, 700, 2, 300
    sm = Long([new], [T], window, 8, 1, G, D, 16, dtype=dtype, given_back=False)
    sm.cache.nan_to_num_(0.5)
    g = torch.Generator().manual_seed(1)
    along = torch.randn(D, generator=g)
    along *= D ** 0.5 / along.norm()
    q = sm.parts(sm.qkv)[0]
    x, keys = along + 0.1 * torch.randn(q.shape, generator=g), 17.0 / D ** 0.5 * along.expand(8, D)
    if signs == "both":
        x = x + 2.0 * (torch.randint(0, 2, q.shape, generator=g) * 2 - 1)
        keys = keys + 0.5 * (torch.randint(0, 2, (8, D), generator=g) * 2 - 1)
    q.copy_(x.to(q.dtype))
    sm.cache[0, torch.from_numpy(sm.slots(0, np.arange(8))), 0] = keys.to(q.dtype)
    step, qg, _, _, _cache = sm.on_gpu(kvs)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, G, True, window, 8), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(qg), torch.empty(new, G, device="cuda")
    w = torch.zeros(1, 1, step.max_kv, device="cuda")
    kvs.kvs_attend_sinks(step, 0, qg, out, z, None, True, window, 8, ws)
    kvs.kvs_weigh_sinks(step, 0, qg, z, w, None, 0.0, True, window, 8, flags=kvs.KVS_F_VALIDATE)
    assert 17 < z.mean() < 23 and w[0, 0, :8].sum() > 0.9 * new * G
    off = float(w.double().sum()) / (new * G) - 1
    unit = 2.0 ** -25 * 2.0 ** np.ceil(np.log2(float(z.max()) * LOG2E))
    h = np.sqrt((1 + 3 * np.log(2) ** 2) * unit ** 2 + 2 * 308 * 2.0 ** -48)
    bound = h * np.sqrt(2 * np.log(2 / 1e-6) / (new * G)) + 2 * 2.0 ** -22
    assert abs(off) <= bound, (off, bound)


# ---- requests without new tokens ---------------------------------------------------
@pytest.mark.parametrize("new", [[0, 1], [0, 5], [0, 20], [0, 150]])
@pytest.mark.parametrize("window,sinks", [(0, 6), (0, 0), (704, 1), (600, 104), (2 ** 31 - 1, 0)])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_a_request_without_new_tokens_reads_no_table_entry(new, window, sinks, decay):
    """Where the mask hides nothing, too: its weights fade, and the other request gets its own."""
    sm = Long(new, [700, 650], window, sinks, 2, 4, 64)
    sm.tables[0] = -1
    step, q, _, _, _cache = sm.on_gpu(kvs)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 8, True, window, sinks), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(q), torch.empty(sm.N, 8, device="cuda")
    kvs.kvs_attend_sinks(step, 0, q, out, z, None, True, window, sinks, ws, flags=kvs.KVS_F_VALIDATE)
    w = torch.rand(2, 2, step.max_kv, device="cuda")
    before = w.clone()
    kvs.kvs_weigh_sinks(step, 0, q, z, w, None, decay, True, window, sinks, flags=kvs.KVS_F_VALIDATE)
    assert torch.equal(w[0, :, :700], before[0, :, :700] * decay)
    assert torch.equal(w[0, :, 700:], before[0, :, 700:])
    one = Long(new[1:], [650], window, sinks, 2, 4, 64)                   # as the second request alone
    one.tables, one.qkv, one.cache, one.num_blocks = sm.tables[1:], sm.qkv, sm.cache, sm.num_blocks
    want, bound = one.weigh(z.cpu().numpy(), before[1:, :, :650].cpu().numpy(), decay, 64 ** -0.5, True, 0)
    assert (np.abs(w[1:, :, :650].double().cpu().numpy() - want) <= bound).all()


# ---- the example ------------------------------------------------------------------
@pytest.mark.parametrize("prefix,suffix", [(600, 90), (600, 10), (500, 70)])
def test_a_session_decodes_behind_its_prompt(prefix, suffix, monkeypatch):
    """What is decoded is text: its tokens have the same position on all axes, the first the one behind the prompt's largest."""
    from paper_2609_35065_gb300 import prefix_step
    cfg, seen, append = prefix_step.session(), [], kvs.kvs_append_axes

    def recorded(step, layer, q, k, v, q_out, rope, axes, positions, *a):
        if layer == 0 and positions.shape[1] == 1:
            seen.append(positions[:, 0].tolist())
        return append(step, layer, q, k, v, q_out, rope, axes, positions, *a)

    monkeypatch.setattr(kvs, "kvs_append_axes", recorded)
    prefix_step.run(cfg, prefix, suffix, decode=5)
    first = int(prefix_step.prompt_positions(cfg, prefix + suffix).max()) + 1
    assert seen == [[first + k] * 3 for k in range(5)]


# ---- many row tiles -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,window,sinks,H,G,D", [(2400, 40, 130, 1, 4, 64), (1200, 500, 260, 8, 4, 128), (1200, 1100, 4, 16, 2, 64), (1300, 1200, 4, 30, 1, 64)])
def test_weights_of_shared_row_tiles(dtype, new, window, sinks, H, G, D):
    """The sinks' rows shared by 8, 4 and 2 CTAs and by none, each of which has more row tiles than lse has slots."""
    sm = Long([new], [new + 60], window, sinks, H, G, D, dtype=dtype)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    lse = sm.attend(D ** -0.5, True, window)[2].astype(np.float32)
    w = torch.rand(1, H, step.max_kv, device="cuda")
    before = w.cpu().numpy()
    kvs.kvs_weigh_sinks(step, 0, q, torch.from_numpy(lse).cuda(), w, None, 0.5, True, window, sinks, flags=kvs.KVS_F_VALIDATE)
    want, bound = sm.weigh(lse, before, 0.5, D ** -0.5, True, window)
    T = new + 60
    assert (np.abs(w.double().cpu().numpy() - want) <= bound)[..., :T].all()


# ---- eviction where blocks were given back --------------------------------------------
@pytest.mark.parametrize("decay", [0.5, 1.0])
@pytest.mark.parametrize("new,lens", [([1, 1], [700, 390]), ([40, 3], [600, 300]), ([20, 0], [600, 64])])
def test_tokens_that_were_given_back_are_kept_last(new, lens, decay):
    """Their weights are NaN, which fading leaves and eviction ranks behind every number: while the budget is no larger than what is left, no
    table entry of theirs is read."""
    window, sinks, budget = 64, 4, 76
    sm = Long(new, lens, window, sinks, 2, 4, 64, extra_blocks=40)
    step, q, _, _, cache = sm.on_gpu(kvs)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 8, True, window, sinks), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(q), torch.empty(sm.N, 8, device="cuda")
    kvs.kvs_attend_sinks(step, 0, q, out, z, None, True, window, sinks, ws, flags=kvs.KVS_F_VALIDATE)
    w = torch.rand(1, 2, 2, step.max_kv, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    gone = np.zeros((2, step.max_kv), dtype=bool)
    for r, T in enumerate(lens):
        block = sm.tables[r].numpy()[np.arange(T) // sm.B]
        gone[r, :T] = (block < 0) | (block >= sm.num_blocks)
    assert gone[0].any()
    w.masked_fill_(torch.from_numpy(gone).cuda()[None, :, None], float("nan"))
    kvs.kvs_weigh_sinks(step, 0, q, z, w[0], None, decay, True, window, sinks, flags=kvs.KVS_F_VALIDATE)
    free = np.setdiff1d(np.arange(sm.num_blocks), sm.tables.numpy().ravel())[:10].reshape(2, 5).astype(np.int32)
    kept, lens_out = torch.empty(1, 2, 2, budget, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    kvs.kvs_evict(step, w, torch.from_numpy(free).cuda(), budget, sinks, 60, kept, None, lens_out, flags=kvs.KVS_F_VALIDATE)
    got = kept.cpu().numpy()
    assert (got == ops_ref.evict(w.cpu().numpy(), lens, budget, sinks, 60)).all()
    for r, T in enumerate(lens):
        J = min(T, budget)
        assert lens_out[r] == J and not gone[r][got[0, r, :, :J]].any()
        flat = cache.view(2, -1, 2, 64)
        for h in range(2):
            src = torch.from_numpy(sm.slots(r, got[0, r, h, :J])).cuda()
            dst = torch.from_numpy(free[r][np.arange(J) // sm.B].astype(np.int64) * sm.B + np.arange(J) % sm.B).cuda()
            assert torch.equal(flat[:, dst, h].view(torch.int16), flat[:, src, h].view(torch.int16))


# ---- more query heads to a KV head than a tile has rows ---------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,lens,G,D", [([1, 1], [300, 40], 130, 64), ([3, 0, 2], [300, 9, 500], 200, 128), ([1], [900], 300, 72)])
def test_more_heads_than_a_tile_has_rows(dtype, new, lens, G, D):
    sm = Long(new, lens, 100, 5, 1, G, D, dtype=dtype)
    step, q, _, _, _cache = sm.on_gpu(kvs)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, G, True, 100, 5), dtype=torch.uint8, device="cuda")
    out, z = torch.empty_like(q), torch.empty(sm.N, G, device="cuda")
    kvs.kvs_attend_sinks(step, 0, q, out, z, None, True, 100, 5, ws, flags=kvs.KVS_F_VALIDATE)
    want, bound, lse, lse_bound = sm.attend(D ** -0.5, True, 100)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
    assert (np.abs(z.double().cpu().numpy() - lse) <= lse_bound).all()
    w = torch.zeros(sm.R, 1, step.max_kv, device="cuda")
    kvs.kvs_weigh_sinks(step, 0, q, z, w, None, 0.0, True, 100, 5, flags=kvs.KVS_F_VALIDATE)
    want, bound = sm.weigh(z.cpu().numpy(), np.zeros((sm.R, 1, max(lens))), 0.0, D ** -0.5, True, 100)
    assert (np.abs(w.double().cpu().numpy()[..., : max(lens)] - want) <= bound).all()


# ---- sinks whose scores are -infinity ------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,R,sinks,out", [(3, 2, 60, 40), (40, 2, 60, 40), (150, 1, 300, 200), (400, 12, 60, 40), (400, 12, 300, 200)])
def test_sinks_of_no_weight(new, R, sinks, out, D, dtype):
    """The first `out` sinks score -infinity for every row: they weigh nothing, and the others are weighed against one another, however
    small their scores.  Off are the weights by one rounding, the outputs by another, both of at most the largest value, and by 2^-9 of a
    rounding for all else."""
    sm = Long([new] * R, [new + 300] * R, 100, sinks, 1, 2, D, 16, dtype=dtype, given_back=False)
    sm.cache.nan_to_num_(0.5)
    q = sm.parts(sm.qkv)[0]
    q[..., 0] = 1.0
    q[..., 1] = 16.0
    sm.cache[0, ..., 0] = 0.0
    sm.cache[0, ..., 1] = -16.0                                             # e^-22 to e^-32 against a reference of 0
    for r in range(R):
        sm.cache[0, torch.from_numpy(sm.slots(r, np.arange(out))), 0, 0] = float("-inf")
    step, qg, _, _, _cache = sm.on_gpu(kvs)
    ws = torch.empty(kvs.kvs_attend_sinks_workspace(step, 2, True, 100, sinks), dtype=torch.uint8, device="cuda")
    got, z = torch.empty_like(qg), torch.empty(sm.N, 2, device="cuda")
    kvs.kvs_attend_sinks(step, 0, qg, got, z, None, True, 100, sinks, ws, flags=kvs.KVS_F_VALIDATE)
    for r in range(R):
        for i in range(2):
            s, _, v = sm.scores(r, 0, i, D ** -0.5, True, 100)
            assert np.isneginf(s[:, :out]).all()
            p = np.exp(s - s.max(1, keepdims=True))
            want = p @ v / p.sum(1, keepdims=True)
            rows = slice(int(sm.starts[r]), int(sm.starts[r + 1]))
            off = np.abs(got[rows, i].double().cpu().numpy() - want)
            assert (off <= (2 + 2.0 ** -9) * ops_ref.UNIT[dtype] * np.abs(v).max()).all()
            lse = s.max(1) + np.log(p.sum(1))
            assert (np.abs(z[rows, i].double().cpu().numpy() - lse) <= 2.0 ** -14).all()
