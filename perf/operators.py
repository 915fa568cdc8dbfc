"""Operator cases: a model's work on the paged cache between a retrieval and the next store-back.

A forward step takes each request's new tokens, rotates their queries and keys and appends
keys and values to the cache (`append`), attends over the whole of it, retrieved prefix and
new tokens alike (`attend`), adds up what weight each cached token received (`weigh`) and,
where the cache grows too large, keeps the tokens of the most weight (`evict`).

Keys of a case
  op            "append", "attend", "weigh" or "evict"
  dtype         "bf16" or "f16", of queries, cache and outputs
  L H G D B     layers, KV heads, query heads per KV head, head dim, tokens per paged block
  R             requests
  new_lo/_hi    new tokens of a request, spread evenly over the requests
  past_lo/_hi   tokens in its cache before them
  causal        whether a new token sees only the tokens up to its own
  window        tokens that a new token sees at most, its own included; 0: no limit
  rot, inter    rotated dims of a head; pairs (2i, 2i + 1) instead of (i, i + rot / 2)
  base, factor  base of the rotary frequencies; factor that positions are divided by
  budget, sinks, recent    tokens that eviction keeps; the first and last ones always kept
"""
import math

import numpy as np
import torch

own = False

DECAY = 0.875
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "L": 1, "H": 8, "G": 4, "D": 128, "B": 16, "R": 1, "new_lo": 1, "new_hi": 1,
         "past_lo": 0, "past_hi": 0, "causal": True, "window": 0, "rot": 128, "inter": False, "base": 500000.0, "factor": 1.0,
         "budget": 0, "sinks": 0, "recent": 0}
    c.update(kw)
    return c


def listed():
    return [
        # One decode step of 16 requests of the 8B-shaped model: 16 tokens are rotated and appended;
        # what counts is the time until the kernel has run.
        _case("append_decode", "append", R=16, past_lo=2048, past_hi=4096),
        # The prefill of the benchmark's batch: 16 suffixes of 2048 tokens behind 2048 retrieved ones,
        # positions scaled for long contexts.
        _case("append_suffixes", "append", R=16, new_lo=2048, new_hi=2048, past_lo=2048, past_hi=2048, factor=8.0),
        # One token over a short cache: the smallest call of a model's inner loop.
        _case("decode_short", "attend", past_lo=528, past_hi=528),
        # A decode step of 64 requests whose caches differ in length.
        _case("decode_batch", "attend", R=64, past_lo=2047, past_hi=8191),
        # One token over a long document: one request has to occupy the whole GPU.
        _case("decode_long", "attend", past_lo=131071, past_hi=131071),
        # Five drafted tokens of each of eight requests verified at once, two KV heads of 64 with
        # seven query heads each, half precision, caches of odd lengths.
        _case("verify_drafts", "attend", dtype="f16", H=2, G=7, D=64, R=8, new_lo=5, new_hi=5, past_lo=4001, past_hi=9973),
        # A question of 293 tokens about a retrieved document of 12288, 14B-shaped.
        _case("question_long", "attend", G=5, new_lo=293, new_hi=293, past_lo=12288, past_hi=12288),
        # The prefill of the benchmark's batch: 16 suffixes of 2048 tokens behind 2048 retrieved ones.
        _case("suffix_batch", "attend", R=16, new_lo=2048, new_hi=2048, past_lo=2048, past_hi=2048),
        # The weight that a decode step's 16 tokens give to the cached ones.
        _case("weigh_decode", "weigh", R=16, past_lo=4095, past_hi=8191),
        # The same for the last 1024 tokens of a prompt, 14B-shaped.
        _case("weigh_suffix", "weigh", G=5, new_lo=1024, new_hi=1024, past_lo=12288, past_hi=12288),
        # A small model's cache cut from 512 tokens to 128.
        _case("evict_tiny", "evict", L=2, H=4, D=64, past_lo=512, past_hi=512, budget=128, sinks=4, recent=32),
        # All layers of two requests of the 8B-shaped model cut from about 8192 tokens to 2048.
        _case("evict_batch", "evict", L=32, R=2, past_lo=8000, past_hi=8192, budget=2048, sinks=4, recent=256),
    ]


# Most of what a drawn case may cost: the listed cases' largest scores (query heads x new x cached
# tokens of all requests), cache tokens x KV heads x head dim x layers, and appended rows.
MOST_SCORES = 32 * 16 * 2048 * 4096
MOST_CACHE = 64 * 8192 * 8 * 128
MOST_EVICT = 32 * 2 * 8192 * 8 * 128
MOST_ROWS = 32768 * 8 * 128


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weigh", "evict"])
    D = rng.choice([64, 80, 96, 128, 128, 128])
    H = rng.choice([1, 2, 3, 4, 8, 8, 8])
    G = rng.choice([1, 2, 4, 4, 5, 7, 8])
    kw = {"dtype": rng.choice(["bf16", "bf16", "f16"]), "D": D, "H": H, "G": G, "B": rng.choice([1, 8, 16, 16, 16, 32, 64]),
          "rot": D if rng.random() < 0.6 else D // 4 * 2, "inter": rng.random() < 0.4, "factor": rng.choice([1.0, 4.0, 8.0])}
    if op == "append":
        R = _spread(rng, 1, 64)
        new = _spread(rng, 1, max(1, min(4096, MOST_ROWS // (R * H * D))))
        past = _spread(rng, 1, max(1, min(32768, MOST_CACHE // (R * H * D) - new)))
    elif op == "evict":
        kw["L"] = L = _spread(rng, 1, 40)
        R = _spread(rng, 1, 8)
        new, past = 0, _spread(rng, 64, max(65, min(32768, MOST_EVICT // (R * L * H * D))))
        budget = max(8, min(past, int(past * rng.uniform(0.1, 0.7))))
        kw.update(budget=budget, sinks=rng.randint(0, 4), recent=rng.randint(0, budget // 4))
    else:
        R = _spread(rng, 1, 64)
        past = _spread(rng, 16, max(17, min(131071, MOST_CACHE // (R * H * D))))
        new = 1 if rng.random() < 0.4 else _spread(rng, 2, max(2, min(2048, past, MOST_SCORES // (R * H * G * 2 * past))))
        if rng.random() < 0.25:
            kw["window"] = _spread(rng, 16, 4096)
        kw["causal"] = rng.random() < 0.9
    kw.update(R=R, new_lo=(new + 1) // 2, new_hi=new, past_lo=(past + 1) // 2, past_hi=past)
    c = _case("", op, **kw)
    del c["name"]
    return c


# ---- what the cases are made of --------------------------------------------
def _even(lo, hi, n, step):
    """n whole numbers over [lo, hi] at even distances, in a scrambled order."""
    k = [(i * step) % n if math.gcd(step, n) == 1 else i for i in range(n)]
    return [lo + (hi - lo) * i // max(1, n - 1) if n > 1 else hi for i in k]


def _lengths(c):
    """New tokens of each request, and its cached tokens with them."""
    new, past = _even(c["new_lo"], c["new_hi"], c["R"], 7), _even(c["past_lo"], c["past_hi"], c["R"], 11)
    return new, [n + p for n, p in zip(new, past)]


def _pairs(c):
    """Query-key pairs that the masks leave, of one query head, and keys that some query sees."""
    pairs = keys = 0
    for n, T in zip(*_lengths(c)):
        pos = np.arange(T - n, T, dtype=np.int64)
        hi = pos + 1 if c["causal"] else np.full(n, T)
        lo = np.maximum(0, pos + 1 - c["window"]) if c["window"] else np.zeros(n, np.int64)
        pairs += int((hi - lo).sum())
        keys += int(hi.max() - lo.min()) if n else 0
    return pairs, keys


def work(c):
    new, lens = _lengths(c)
    N, H, D = sum(new), c["H"], c["D"]
    q = N * H * c["G"] * D * 2
    if c["op"] == "append":
        return {"bytes": 2 * (q + 2 * N * H * D * 2), "flops": 6 * N * H * (c["G"] + 1) * c["rot"] // 2}
    if c["op"] == "evict":
        kept = sum(min(T, c["budget"]) for T in lens)
        return {"bytes": c["L"] * H * (4 * sum(lens) + kept * (2 * 2 * D * 2 + 8)), "flops": 0}
    pairs, keys = _pairs(c)
    if c["op"] == "attend":
        return {"bytes": 2 * q + N * H * c["G"] * 4 + 2 * keys * H * D * 2, "flops": 4 * pairs * H * c["G"] * D}
    return {"bytes": q + N * H * c["G"] * 4 + keys * H * D * 2 + 2 * sum(lens) * H * 4, "flops": 2 * pairs * H * c["G"] * D}


def _slots(tables, t, B):
    """Cache slots of the tokens t, one row of t for each request."""
    return torch.gather(tables.long(), 1, t // B) * B + t % B


def _turns(c):
    """Turns per position of each rotated pair, as the sum of two 32-bit numbers."""
    f = c["base"] ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"]) / c["factor"] / (2 * math.pi)
    hi = f.astype(np.float32)
    return np.stack([hi, (f - hi).astype(np.float32)], 1)


class State:
    pass


def prepare(c, seed):
    s = State()
    s.c = c
    dev, dt = torch.device("cuda"), TYPES[c["dtype"]]
    gen = torch.Generator(dev).manual_seed(seed)
    H, G, D, B, R, L = c["H"], c["G"], c["D"], c["B"], c["R"], c["L"]
    new, lens = _lengths(c)
    N, s.max_q, s.max_kv = sum(new), max(new), max(lens)
    s.N = N

    # each request's blocks: any of the cache's, in any order
    W = -(-s.max_kv // B)
    Wd = -(-c["budget"] // B) if c["op"] == "evict" else 0
    s.num_blocks = R * (W + Wd) + 3
    perm = torch.randperm(s.num_blocks, generator=gen, device=dev).to(torch.int32)
    s.tables = perm[: R * W].view(R, W).contiguous()
    s.kv_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    s.q_starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)

    # keys whose lengths differ, so that some tokens receive much more weight than others
    s.cache = torch.randn(2 * L, s.num_blocks, B, H, D, generator=gen, device=dev, dtype=dt)
    for l in range(L):
        s.cache[2 * l] *= torch.exp(0.4 * torch.randn(s.num_blocks, B, H, 1, generator=gen, device=dev)).to(dt)

    if c["op"] == "evict":
        s.dst_tables = perm[R * W: R * (W + Wd)].view(R, Wd).contiguous()
        s.weights = torch.rand(L, R, H, s.max_kv, generator=gen, device=dev).pow_(6).mul_(16)
        s.kept = torch.empty(L, R, H, c["budget"], dtype=torch.int32, device=dev)
        s.new_weights = torch.empty(L, R, H, c["budget"], dtype=torch.float32, device=dev)
        s.new_lens = torch.empty(R, dtype=torch.int32, device=dev)
    else:
        s.qkv = torch.randn(N, (H * G + 2 * H) * D, generator=gen, device=dev, dtype=dt)
        s.q = s.qkv[:, : H * G * D].view(N, H * G, D)
        s.k = s.qkv[:, H * G * D: H * (G + 1) * D].view(N, H, D)
        s.v = s.qkv[:, H * (G + 1) * D:].view(N, H, D)
        s.scale = D ** -0.5
    if c["op"] == "append":
        s.turns = torch.from_numpy(_turns(c)).to(dev)
        first = torch.tensor([T - n for n, T in zip(new, lens)], device=dev)
        req = torch.searchsorted(s.q_starts, torch.arange(N, dtype=torch.int32, device=dev), right=True) - 1
        s.positions = (first[req] + torch.arange(N, device=dev) - s.q_starts[req]).to(torch.int32)
        s.q_out = torch.empty(N, H * G, D, dtype=dt, device=dev)
    if c["op"] in ("attend", "weigh"):
        # what blocks hold beyond a request's tokens is whatever they held before: not numbers, here
        t = torch.arange(W * B, device=dev).expand(R, -1)
        used = torch.zeros(s.num_blocks * B, dtype=torch.bool, device=dev)
        used[_slots(s.tables, t, B)[t < s.kv_lens[:, None]]] = True
        s.cache.view(2, -1, H, D)[:, ~used] = float("nan")
        s.out = torch.empty(N, H * G, D, dtype=dt, device=dev)
        s.lse = torch.empty(N, H * G, dtype=torch.float32, device=dev)
    if c["op"] == "weigh":
        s.weights = torch.rand(R, H, s.max_kv, generator=gen, device=dev)
        s.lse = _attend(s, only_lse=True)

    if own:
        from paper_2609_35065_gb300 import kvs
        s.kvs = kvs
        s.step = kvs.Step((L, H, D, 2, B, 256 if 256 % B == 0 else B), [s.cache[p].data_ptr() for p in range(2 * L)], s.num_blocks,
                          s.tables, s.kv_lens, None if s.max_q <= 1 and N == R else s.q_starts, s.max_kv, total_q=N, max_q=s.max_q,
                          dtype=kvs.KVS_DTYPE_BF16 if dt == torch.bfloat16 else kvs.KVS_DTYPE_F16)
        if c["op"] == "append":
            s.rope = kvs.Rope(s.turns, c["rot"], c["inter"])
        if c["op"] == "attend":
            s.workspace = torch.empty(kvs.kvs_attend_workspace(s.step, H * G), dtype=torch.uint8, device=dev)
    return s


# ---- the operators in plain form -------------------------------------------
def _rows(s):
    """Request of each query row, and the row's place among the request's new tokens."""
    n = torch.arange(s.N, dtype=torch.int32, device=s.q_starts.device)
    req = torch.searchsorted(s.q_starts, n, right=True) - 1
    return req, (n - s.q_starts[req]).long()


def _padded(s, x):
    """Rows of all requests as [request, new token, ...], and those requests' counts."""
    at = s.q_starts[:-1, None].long() + torch.arange(s.max_q, device=x.device)
    return x[at.clamp(max=s.N - 1)]


def _scores(s):
    """Masked scores [R, H, G, new, cached], the slots of the cached tokens and which are there."""
    c = s.c
    H, G, D, B = c["H"], c["G"], c["D"], c["B"]
    t = torch.arange(s.max_kv, device=s.cache.device).expand(c["R"], -1)
    slots = _slots(s.tables, t, B)
    there = t < s.kv_lens[:, None]
    k = s.cache[0].view(-1, H, D)[slots].float()
    k = torch.where(there[:, :, None, None], k, 0.0).permute(0, 2, 3, 1)                    # [R, H, D, T]
    q = _padded(s, s.q).float().view(c["R"], s.max_q, H, G, D).permute(0, 2, 3, 1, 4)       # [R, H, G, new, D]
    scores = torch.matmul(q.reshape(c["R"], H, G * s.max_q, D), k).view(c["R"], H, G, s.max_q, s.max_kv).mul_(s.scale)
    new = (s.q_starts[1:] - s.q_starts[:-1])[:, None]
    i = torch.arange(s.max_q, device=s.cache.device)[None, :]
    pos = (s.kv_lens[:, None] - new + i)[:, :, None]
    seen = there[:, None, :] & (i < new)[:, :, None]
    if c["causal"]:
        seen = seen & (t[:, None, :] <= pos)
    if c["window"]:
        seen = seen & (t[:, None, :] > pos - c["window"])
    return scores.masked_fill_(~seen[:, None, None], float("-inf")), slots, there


def _attend(s, only_lse=False):
    c = s.c
    H, G, D = c["H"], c["G"], c["D"]
    p, slots, there = _scores(s)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    req, i = _rows(s)
    lse = (m + l.log()).squeeze(-1)[req, :, :, i].reshape(s.N, H * G)
    if only_lse:
        return lse
    v = s.cache[1].view(-1, H, D)[slots].float()
    v = torch.where(there[:, :, None, None], v, 0.0).permute(0, 2, 1, 3)                    # [R, H, T, D]
    o = torch.matmul(p.view(c["R"], H, G * s.max_q, s.max_kv), v).view(c["R"], H, G, s.max_q, D)
    o = o / torch.where(l == 0, 1.0, l)
    return {"out": o[req, :, :, i].reshape(s.N, H * G, D).to(s.q.dtype), "lse": lse}


def _weigh(s):
    c = s.c
    p, _, there = _scores(s)
    lse = _padded(s, s.lse).view(c["R"], s.max_q, c["H"], c["G"]).permute(0, 2, 3, 1)
    p = p.sub_(lse[..., None]).exp_()
    p = torch.where(p == p, p, 0.0).sum((2, 3))
    w = s.weights[:, :, : s.max_kv]
    w.copy_(torch.where(there[:, None, :], w * DECAY + p, w))
    return {"weights": s.weights}


def _append(s):
    c = s.c
    H, D, rot = c["H"], c["D"], c["rot"]
    turns = s.positions.float()[:, None] * (s.turns[:, 0] + s.turns[:, 1])
    angle = (turns - turns.floor())[:, None, :] * (2 * math.pi)
    cos, sin = angle.cos(), angle.sin()

    def rotated(x):
        x = x.float()
        r = x[..., :rot]
        a, b = (r[..., 0::2], r[..., 1::2]) if c["inter"] else (r[..., : rot // 2], r[..., rot // 2:])
        a, b = a * cos - b * sin, b * cos + a * sin
        r = torch.stack([a, b], -1).flatten(-2) if c["inter"] else torch.cat([a, b], -1)
        return torch.cat([r, x[..., rot:]], -1).to(s.q.dtype)

    req, i = _rows(s)
    t = (s.kv_lens[req] - (s.q_starts[req + 1] - s.q_starts[req])).long() + i
    slot = s.tables[req, t // c["B"]].long() * c["B"] + t % c["B"]
    s.cache[0].view(-1, H, D)[slot] = rotated(s.k)
    s.cache[1].view(-1, H, D)[slot] = s.v
    return {"q": rotated(s.q), "cache": s.cache}


def _evict(s):
    c = s.c
    L, R, H, J = c["L"], c["R"], c["H"], c["budget"]
    dev = s.cache.device
    t, lens = torch.arange(s.max_kv, device=dev), s.kv_lens.long()[:, None, None]
    always = (t < c["sinks"]) | (t >= lens - c["recent"])
    key = torch.where(always, float("inf"), s.weights)
    key = torch.where(t < lens, key, float("-inf"))
    first = torch.sort(key, dim=-1, descending=True, stable=True)[1][..., :J]
    count, j = lens.clamp(max=J), torch.arange(J, device=dev)
    first = torch.sort(torch.where(j < count, first, s.max_kv), dim=-1)[0]
    kept = torch.where(j < count, first, -1)
    # the places beyond a short cache's end repeat its last token's copy
    j1 = torch.minimum(j, count - 1).expand(L, R, H, J)
    from_t = torch.gather(kept, 3, j1)
    src = _slots(s.tables, from_t.permute(1, 0, 2, 3).reshape(R, -1), c["B"]).view(R, L, H, J).permute(1, 0, 2, 3)
    dst = _slots(s.dst_tables, j1.permute(1, 0, 2, 3).reshape(R, -1), c["B"]).view(R, L, H, J).permute(1, 0, 2, 3)
    l, h = torch.arange(L, device=dev)[:, None, None, None], torch.arange(H, device=dev)[:, None]
    cache = s.cache.view(L, 2, -1, H, c["D"])
    cache[l, 0, dst, h] = cache[l, 0, src, h]
    cache[l, 1, dst, h] = cache[l, 1, src, h]
    new_weights = torch.where(j < count, torch.gather(s.weights, 3, from_t), 0.0)
    return {"cache": s.cache, "kept": kept.to(torch.int32), "weights": new_weights, "lens": count.flatten().to(torch.int32)}


def run(s):
    c = s.c
    if not own:
        return {"append": _append, "attend": _attend, "weigh": _weigh, "evict": _evict}[c["op"]](s)
    stream = torch.cuda.current_stream()
    if c["op"] == "append":
        s.kvs.kvs_append(s.step, 0, s.q, s.k, s.v, s.q_out, s.rope, s.positions, stream)
        return {"q": s.q_out, "cache": s.cache}
    if c["op"] == "attend":
        s.kvs.kvs_attend(s.step, 0, s.q, s.out, s.lse, s.scale, c["causal"], c["window"], s.workspace, stream)
        return {"out": s.out, "lse": s.lse}
    if c["op"] == "weigh":
        s.kvs.kvs_weigh(s.step, 0, s.q, s.lse, s.weights, s.scale, DECAY, c["causal"], c["window"], stream)
        return {"weights": s.weights}
    s.kvs.kvs_evict(s.step, s.weights, s.dst_tables, c["budget"], c["sinks"], c["recent"], s.kept, s.new_weights, s.new_lens, stream)
    return {"cache": s.cache, "kept": s.kept, "weights": s.new_weights, "lens": s.new_lens}


# ---- the definitions in 64 bits --------------------------------------------
def exact(c, seed):
    if c["op"] == "evict":                        # selects and copies: no value is computed
        return None
    s = prepare(c, seed)
    H, G, D, B = c["H"], c["G"], c["D"], c["B"]
    new, lens = _lengths(c)
    starts = np.concatenate([[0], np.cumsum(new)])
    tables = s.tables.cpu().numpy().astype(np.int64)
    if c["op"] == "append":
        cache, q = s.cache.double(), s.q.double()
        rot = c["rot"]
        angle = s.positions.double()[:, None] * s.turns.double().sum(1) * (2 * math.pi)
        e = torch.polar(torch.ones_like(angle), angle)[:, None]
        lo = torch.arange(0, rot, 2, device=q.device) if c["inter"] else torch.arange(rot // 2, device=q.device)
        hi = lo + (1 if c["inter"] else rot // 2)

        def turn(x):
            z = torch.complex(x[..., lo], x[..., hi]) * e
            x[..., lo], x[..., hi] = z.real, z.imag
            return x

        k, v = turn(s.k.double()), s.v.double()
        for r, (n, T) in enumerate(zip(new, lens)):
            at = np.arange(T - n, T)
            slot = torch.from_numpy(tables[r, at // B] * B + at % B).to(q.device)
            for p, x in enumerate((k, v)):
                cache[p].view(-1, H, D)[slot] = x[starts[r]: starts[r + 1]]
        return {"q": turn(q), "cache": cache}

    out, lse_out = torch.zeros(s.N, H * G, D, dtype=torch.float64, device="cuda"), torch.empty(s.N, H * G, dtype=torch.float64, device="cuda")
    weights = s.weights.double() if c["op"] == "weigh" else None
    for r, (n, T) in enumerate(zip(new, lens)):
        if T:
            at = np.arange(T)
            slot = torch.from_numpy(tables[r, at // B] * B + at % B).to("cuda")
        t = torch.arange(T, device="cuda")
        pos = torch.arange(T - n, T, device="cuda")[:, None]
        bad = t > pos if c["causal"] else torch.zeros(n, T, dtype=torch.bool, device="cuda")
        if c["window"]:
            bad = bad | (t <= pos - c["window"])
        rows = slice(starts[r], starts[r + 1])
        for h in range(H):
            k = s.cache[0].view(-1, H, D)[slot, h].double()
            v = s.cache[1].view(-1, H, D)[slot, h].double()
            if weights is not None:
                weights[r, h, :T] *= DECAY
            for g in range(h * G, h * G + G):
                x = (s.q[rows, g].double() @ k.T * s.scale).masked_fill_(bad, -math.inf)
                if weights is not None:
                    weights[r, h, :T] += torch.exp(x - s.lse[rows, g, None].double()).sum(0)
                    continue
                z = torch.logsumexp(x, 1, keepdim=True)
                lse_out[rows, g] = z[:, 0]
                out[rows, g] = torch.exp(x - z) @ v
    return {"weights": weights} if weights is not None else {"out": out, "lse": lse_out}
