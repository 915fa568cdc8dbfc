"""Operator cases: a long session's work on the paged cache, with images and video in its prompts.

A forward step of a model that sees images gives every token a position on several axes (time,
height, width); new queries and keys are rotated by them on the way into the cache
(`append_axes`). A model that runs on without end attends to a window of the last tokens and to
a few first ones that stay visible, the sinks (`attend_sinks`), and what weight the tokens
received under that mask is added up for eviction (`weigh_sinks`). Blocks of the cache that
neither the window nor the sinks reach any more have been given back.

Keys of a case
  op            "append_axes", "attend_sinks" or "weigh_sinks"
  dtype         "bf16" or "f16", of queries, cache and outputs
  H G D B       KV heads, query heads per KV head, head dim, tokens per paged block
  R             requests
  new_lo/_hi    new tokens of a request, spread evenly over the requests
  past_lo/_hi   tokens in its cache before them
  causal        whether a new token sees only the tokens up to its own
  window, sinks tokens that a new token sees at most, its own included, and first ones that it sees beside them
  freed         whether blocks that no new token sees have been given back (table entries -1)
  decay         what weights are multiplied by before a step's are added
  parts         rotated pairs of each axis, as text "16,24,24"
  cycle         pairs go to the axes in turn (else: in blocks)
  restart       each axis has the whole range of frequencies (else: they go on from axis to axis)
  inter, base   pairs (2i, 2i + 1) instead of (i, i + rot / 2); base of the frequencies
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, **kw):
    c = {"name": name, "op": op, "dtype": "bf16", "H": 8, "G": 4, "D": 128, "B": 16, "R": 1, "new_lo": 1, "new_hi": 1,
         "past_lo": 0, "past_hi": 0}
    if op == "append_axes":
        c.update(parts="16,24,24", cycle=False, restart=False, inter=False, base=500000.0)
    else:
        c.update(causal=True, window=1024, sinks=4, freed=True)
    if op == "weigh_sinks":
        c["decay"] = 0.875
    c.update(kw)
    return c


def listed():
    return [
        # A decode step of 16 requests of the 8B-shaped model behind prompts with images: text
        # tokens, whose three positions are alike; what counts is the time until the kernel has run.
        _case("axes_decode", "append_axes", R=16, past_lo=2048, past_hi=4096),
        # The prefill of 16 suffixes of 2048 tokens, images of several sizes among text, behind 2048
        # retrieved ones; the axes take the pairs in turn.
        _case("axes_prompts", "append_axes", R=16, new_lo=2048, new_hi=2048, past_lo=2048, past_hi=2048, cycle=True),
        # An image encoder's layer: eleven images of about 37 x 37 patches, 16 heads of 72 dims, rows and
        # columns as two axes with a range of frequencies each, half precision.
        _case("axes_patches", "append_axes", dtype="f16", H=16, G=1, D=72, R=11, new_lo=1225, new_hi=1369, parts="18,18",
              restart=True, base=10000.0),
        # One token of one long session: the smallest call of a model's inner loop.
        _case("sinks_one", "attend_sinks", past_lo=131071, past_hi=131071),
        # A decode step of 64 sessions, some of them shorter than the window.
        _case("sinks_batch", "attend_sinks", R=64, past_lo=1500, past_hi=131071, window=4096),
        # Five drafted tokens of each of eight sessions verified at once, two KV heads of 64 with
        # seven query heads each, half precision, odd lengths; nothing was given back.
        _case("sinks_drafts", "attend_sinks", dtype="f16", H=2, G=7, D=64, R=8, new_lo=5, new_hi=5, past_lo=4001, past_hi=9973,
              window=1000, sinks=3, freed=False),
        # A question of 293 tokens behind a session of 12288, 14B-shaped.
        _case("sinks_question", "attend_sinks", G=5, new_lo=293, new_hi=293, past_lo=12288, past_hi=12288, window=2048, sinks=64),
        # The prefill of 16 suffixes of 2048 tokens behind 2048 retrieved ones.
        _case("sinks_suffixes", "attend_sinks", R=16, new_lo=2048, new_hi=2048, past_lo=2048, past_hi=2048),
        # Prompts of about 4096 tokens through a layer with a narrow window, eight query heads of 64 to a KV head.
        _case("sinks_narrow", "attend_sinks", dtype="f16", G=8, D=64, R=4, new_lo=4001, new_hi=4096, window=128),
        # The weight that a decode step's 16 tokens give to the cached ones.
        _case("weigh_session", "weigh_sinks", R=16, past_lo=8191, past_hi=32767, window=4096),
        # The same for the last 1024 tokens of a prompt, 14B-shaped.
        _case("weigh_window", "weigh_sinks", G=5, new_lo=1024, new_hi=1024, past_lo=12288, past_hi=12288),
    ]


# Most of what a drawn case may cost: scores (query heads x new tokens x tokens that they may see
# between them; that they do see), tokens in the cache x KV heads x head dim, appended rows x heads x head dim, and weights.
MOST_SCORES = 32 * 16 * 2048 * (4 + 1024 + 2047)
MOST_PAIRS = 32 * 16 * 2048 * (4 + 1024)
MOST_CACHE = 64 * 4100 * 8 * 128
MOST_ROWS = 16 * 2048 * 48 * 128
MOST_WEIGHTS = 16 * 8 * 32768


def _spread(rng, lo, hi):
    """A whole number in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["append_axes", "append_axes", "attend_sinks", "attend_sinks", "attend_sinks", "weigh_sinks"])
    D = rng.choice([64, 72, 80, 96, 128, 128, 128])
    H = rng.choice([1, 2, 3, 4, 8, 8, 8])
    G = rng.choice([1, 2, 4, 4, 5, 7, 8])
    kw = {"dtype": rng.choice(["bf16", "bf16", "f16"]), "D": D, "H": H, "G": G, "B": rng.choice([1, 8, 16, 16, 16, 32, 64])}
    if op == "append_axes":
        A = rng.choice([2, 2, 3, 3, 3, 4])
        R = _spread(rng, 1, 64)
        new = _spread(rng, 1, max(1, min(4096, MOST_ROWS // (R * H * (G + 2) * D))))
        past = _spread(rng, 1, max(1, min(32768, MOST_CACHE // (R * H * D) - new)))
        pairs = D // 2 if rng.random() < 0.7 else D // 4
        cycle = rng.random() < 0.4
        if cycle:                                  # no axis but the first has more than its turns
            parts = [rng.randint(1, pairs // A) for _ in range(A - 1)]
            parts = [pairs - sum(parts)] + parts
        else:
            cuts = [0] + sorted(rng.sample(range(1, pairs), A - 1)) + [pairs]
            parts = [b - a for a, b in zip(cuts, cuts[1:])]
        kw.update(parts=",".join(map(str, parts)), cycle=cycle, restart=rng.random() < 0.4, inter=rng.random() < 0.3,
                  base=rng.choice([10000.0, 500000.0]))
    else:
        R = _spread(rng, 1, 64)
        window = _spread(rng, 16, max(17, min(8192, MOST_CACHE // (R * H * D) - 300)))
        kw.update(window=window, sinks=rng.choice([1, 3, 4, 4, 4, 16, 64, 300]), freed=rng.random() < 0.7, causal=rng.random() < 0.9)
        # as many new tokens as keep new x (first ones + window + new) and new x (first ones + window) in bounds
        rows, held = R * H * G, kw["sinks"] + window
        most = min(2048, int(math.sqrt(held * held / 4 + MOST_SCORES // rows) - held / 2), MOST_PAIRS // (rows * held))
        new = 1 if rng.random() < 0.4 else _spread(rng, 2, max(2, most))
        past = _spread(rng, 16, 131071 if kw["freed"] else max(17, min(32768, MOST_CACHE // (R * H * D))))
        if op == "weigh_sinks":
            past = min(past, max(16, MOST_WEIGHTS // (R * H)))
            kw["decay"] = rng.choice([0.0, 0.875, 1.0])
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


def _parts(c):
    return [int(x) for x in c["parts"].split(",")]


def _held(c, n, T):
    """First tokens of a request that stay visible behind its window, and the first that its window reaches."""
    lo = max(0, T - n + 1 - c["window"])
    return min(c["sinks"], lo), lo


def _pairs(c):
    """Query-key pairs that the mask leaves, of one query head, and keys that some query sees."""
    pairs = keys = 0
    for n, T in zip(*_lengths(c)):
        pos = np.arange(T - n, T, dtype=np.int64)
        hi = pos + 1 if c["causal"] else np.full(n, T)
        lo = np.maximum(0, pos + 1 - c["window"])
        pairs += int((hi - lo + np.minimum(c["sinks"], lo)).sum())
        sinks, first = _held(c, n, T)
        keys += T - first + sinks
    return pairs, keys


def work(c):
    new, lens = _lengths(c)
    N, H, D = sum(new), c["H"], c["D"]
    q = N * H * c["G"] * D * 2
    if c["op"] == "append_axes":
        parts = _parts(c)
        return {"bytes": 2 * (q + 2 * N * H * D * 2) + 4 * N * len(parts), "flops": 6 * N * H * (c["G"] + 1) * sum(parts)}
    pairs, keys = _pairs(c)
    if c["op"] == "attend_sinks":
        return {"bytes": 2 * q + N * H * c["G"] * 4 + 2 * keys * H * D * 2, "flops": 4 * pairs * H * c["G"] * D}
    # a decay of 0 writes every weight, 1 changes those of seen tokens only
    touched = 4 * sum(lens) if c["decay"] == 0.0 else 8 * keys if c["decay"] == 1.0 else 8 * sum(lens)
    return {"bytes": q + N * H * c["G"] * 4 + keys * H * D * 2 + touched * H, "flops": 2 * pairs * H * c["G"] * D}


def _axes(c):
    """Axis of each rotated pair, and its turns per position as the sum of two 32-bit numbers."""
    parts = _parts(c)
    A, pairs = len(parts), sum(parts)
    if c["cycle"]:
        axis = np.zeros(pairs, dtype=np.uint8)
        for a in range(1, A):
            axis[a: a + A * parts[a]: A] = a
    else:
        axis = np.repeat(np.arange(A, dtype=np.uint8), parts)
    f = c["base"] ** (-np.arange(pairs, dtype=np.float64) / pairs)
    if c["restart"]:
        for a in range(A):
            f[axis == a] = c["base"] ** (-np.arange(parts[a], dtype=np.float64) / parts[a])
    f /= 2 * math.pi
    hi = f.astype(np.float32)
    return axis, np.stack([hi, (f - hi).astype(np.float32)], 1)


def _positions(A, n, first, rng):
    """[A, n] positions of n tokens from `first` on: text, whose axes go alike, and pictures in it, whose
    last two axes are a row and a column; text goes on behind the largest position of a picture."""
    out, at, p = np.empty((A, n), dtype=np.int32), 0, first
    while at < n:
        text = min(n - at, rng.integers(1, 200))
        out[:, at: at + text] = p + np.arange(text)
        at, p = at + text, p + text
        rows, cols = (int(x) for x in rng.integers(8, 48, 2))
        some = min(n - at, rows * cols)
        k = np.arange(some)
        out[:, at: at + some] = p
        out[A - 2, at: at + some] += (k // cols).astype(np.int32)
        out[A - 1, at: at + some] += (k % cols).astype(np.int32)
        at, p = at + some, p + max(rows, cols)
    return out


def _slots(tables, t, B):
    """Cache slots of the tokens t, one row of t for each request."""
    return torch.gather(tables.long(), 1, t // B) * B + t % B


class State:
    pass


def prepare(c, seed):
    s = State()
    s.c = c
    dev, dt = torch.device("cuda"), TYPES[c["dtype"]]
    gen = torch.Generator(dev).manual_seed(seed)
    rng = np.random.default_rng(seed)
    H, G, D, B, R = c["H"], c["G"], c["D"], c["B"], c["R"]
    new, lens = _lengths(c)
    N, s.max_q, s.max_kv = sum(new), max(new), max(lens)
    s.N = N
    s.kv_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    s.q_starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)

    # each request's blocks: any of the cache's, in any order, and none where nothing of a block is seen any more
    W = -(-s.max_kv // B)
    block = np.arange(W)
    used = np.stack([block < -(-T // B) for T in lens])
    if c.get("freed"):
        for r, (n, T) in enumerate(zip(new, lens)):
            sinks, lo = _held(c, n, T)
            used[r] &= (block * B < sinks) | ((block + 1) * B > lo)
    s.num_blocks = int(used.sum()) + 3
    tables = np.full((R, W), -1, dtype=np.int32)
    tables[used] = rng.permutation(s.num_blocks)[: used.sum()]
    s.tables = torch.from_numpy(tables).to(dev)

    s.cache = torch.randn(2, s.num_blocks, B, H, D, generator=gen, device=dev, dtype=dt)
    s.qkv = torch.randn(N, (H * G + 2 * H) * D, generator=gen, device=dev, dtype=dt)
    s.q = s.qkv[:, : H * G * D].view(N, H * G, D)
    s.k = s.qkv[:, H * G * D: H * (G + 1) * D].view(N, H, D)
    s.v = s.qkv[:, H * (G + 1) * D:].view(N, H, D)
    s.scale = D ** -0.5
    if c["op"] == "append_axes":
        axis, turns = _axes(c)
        A = len(_parts(c))
        s.axis, s.turns = torch.from_numpy(axis).to(dev), torch.from_numpy(turns).to(dev)
        s.positions = torch.from_numpy(np.concatenate([_positions(A, n, T - n, rng) for n, T in zip(new, lens)], 1)).to(dev)
        s.q_out = torch.empty(N, H * G, D, dtype=dt, device=dev)
    else:
        # keys whose lengths differ, and first tokens that draw much of every query's weight
        s.cache[0] *= torch.exp(0.4 * torch.randn(s.num_blocks, B, H, 1, generator=gen, device=dev)).to(dt)
        pull = torch.randn(H, 1, D, generator=gen, device=dev)
        pull *= 2 / pull.norm(dim=-1, keepdim=True)
        s.q.view(N, H, G, D).add_(pull.to(dt))
        flat = s.cache.view(2, -1, H, D)
        first = torch.arange(min(4, s.max_kv), device=dev).expand(R, -1)
        there = (first < s.kv_lens[:, None]) & (torch.gather(s.tables.long(), 1, first // B) >= 0)
        flat[0, _slots(s.tables, first, B)[there]] += (pull[:, 0] * (D ** 0.5)).to(dt)
        # what the cache holds that no new token sees is whatever it held before: not numbers, here
        held = torch.zeros(s.num_blocks * B, dtype=torch.bool, device=dev)
        for r, (n, T) in enumerate(zip(new, lens)):
            sinks, lo = _held(c, n, T)
            t = torch.cat([torch.arange(sinks, device=dev), torch.arange(lo, T, device=dev)])
            held[_slots(s.tables[r: r + 1], t[None], B)[0]] = True
        flat[:, ~held] = float("nan")
        s.out = torch.empty(N, H * G, D, dtype=dt, device=dev)
        s.lse = torch.empty(N, H * G, dtype=torch.float32, device=dev)
    if c["op"] == "weigh_sinks":
        s.weights = torch.rand(R, H, s.max_kv, generator=gen, device=dev)
        s.lse = _attend(s, only_lse=True)

    if own:
        from paper_2609_35065_gb300 import kvs
        s.kvs = kvs
        s.step = kvs.Step((1, H, D, 2, B, 256 if 256 % B == 0 else B), [s.cache[p].data_ptr() for p in range(2)], s.num_blocks,
                          s.tables, s.kv_lens, None if s.max_q <= 1 and N == R else s.q_starts, s.max_kv, total_q=N, max_q=s.max_q,
                          dtype=kvs.KVS_DTYPE_BF16 if dt == torch.bfloat16 else kvs.KVS_DTYPE_F16)
        if c["op"] == "append_axes":
            s.rope = kvs.Rope(s.turns, 2 * len(axis), c["inter"])
            s.axes = kvs.Axes(s.axis, len(_parts(c)))
        if c["op"] == "attend_sinks":
            s.workspace = torch.empty(kvs.kvs_attend_sinks_workspace(s.step, H * G, c["causal"], c["window"], c["sinks"]),
                                      dtype=torch.uint8, device=dev)
    return s


# ---- the operators in plain form -------------------------------------------
def _rows(s):
    """Request of each query row, and the row's place among the request's new tokens."""
    n = torch.arange(s.N, dtype=torch.int32, device=s.q_starts.device)
    req = torch.searchsorted(s.q_starts, n, right=True) - 1
    return req, (n - s.q_starts[req]).long()


def _padded(s, x):
    """Rows of all requests as [request, new token, ...]."""
    at = s.q_starts[:-1, None].long() + torch.arange(s.max_q, device=x.device)
    return x[at.clamp(max=s.N - 1)]


def _scores(s):
    """Masked scores [R, H, G, new, held] of the tokens that some row of a request sees, those tokens
    [R, held], which of them there are, and their slots."""
    c = s.c
    H, G, D, B, R = c["H"], c["G"], c["D"], c["B"], c["R"]
    dev = s.cache.device
    new = (s.q_starts[1:] - s.q_starts[:-1]).long()[:, None]
    lens = s.kv_lens.long()[:, None]
    lo = (lens - new + 1 - c["window"]).clamp(min=0)
    sinks = lo.clamp(max=c["sinks"])
    width = min(s.max_kv, c["sinks"] + c["window"] + s.max_q - 1)
    u = torch.arange(width, device=dev).expand(R, -1)
    t = torch.where(u < sinks, u, u - sinks + lo)
    there = t < lens
    slots = _slots(s.tables, torch.where(there, t, 0), B).clamp(min=0)
    k = s.cache[0].view(-1, H, D)[slots].float()
    k = torch.where(there[:, :, None, None], k, 0.0).permute(0, 2, 3, 1)                    # [R, H, D, held]
    q = _padded(s, s.q).float().view(R, s.max_q, H, G, D).permute(0, 2, 3, 1, 4)            # [R, H, G, new, D]
    scores = torch.matmul(q.reshape(R, H, G * s.max_q, D), k).view(R, H, G, s.max_q, width).mul_(s.scale)
    i = torch.arange(s.max_q, device=dev)[None, :]
    pos, at = (lens - new + i)[:, :, None], t[:, None, :]
    seen = there[:, None, :] & (i < new)[:, :, None] & ((at > pos - c["window"]) | (at < c["sinks"]))
    if c["causal"]:
        seen = seen & (at <= pos)
    return scores.masked_fill_(~seen[:, None, None], float("-inf")), t, there, slots


def _attend(s, only_lse=False):
    c = s.c
    H, G, D, R = c["H"], c["G"], c["D"], c["R"]
    p, _, there, slots = _scores(s)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    req, i = _rows(s)
    lse = (m + l.log()).squeeze(-1)[req, :, :, i].reshape(s.N, H * G)
    if only_lse:
        return lse
    v = s.cache[1].view(-1, H, D)[slots].float()
    v = torch.where(there[:, :, None, None], v, 0.0).permute(0, 2, 1, 3)                    # [R, H, held, D]
    o = torch.matmul(p.view(R, H, G * s.max_q, -1), v).view(R, H, G, s.max_q, D)
    o = o / torch.where(l == 0, 1.0, l)
    return {"out": o[req, :, :, i].reshape(s.N, H * G, D).to(s.q.dtype), "lse": lse}


def _weigh(s):
    c = s.c
    p, t, there, _ = _scores(s)
    lse = _padded(s, s.lse).view(c["R"], s.max_q, c["H"], c["G"]).permute(0, 2, 3, 1)
    p = p.sub_(lse[..., None]).exp_()
    p = torch.where(p == p, p, 0.0).sum((2, 3))                                            # [R, H, held]
    cached = (torch.arange(s.max_kv, device=t.device) < s.kv_lens[:, None])[:, None, :]
    w = s.weights
    w.copy_(torch.where(cached, w * c["decay"] if c["decay"] else 0.0, w))
    at = torch.where(there, t, 0)[:, None, :].expand(-1, c["H"], -1)
    w.scatter_add_(2, at, torch.where(there[:, None, :], p, 0.0))
    return {"weights": w}


def _append(s):
    c = s.c
    H, D, rot = c["H"], c["D"], 2 * len(s.axis)
    angle = s.positions[s.axis.long()].double().T * (s.turns[:, 0].double() + s.turns[:, 1]) * (2 * math.pi)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

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


def run(s):
    c = s.c
    if not own:
        return {"append_axes": _append, "attend_sinks": _attend, "weigh_sinks": _weigh}[c["op"]](s)
    stream = torch.cuda.current_stream()
    if c["op"] == "append_axes":
        s.kvs.kvs_append_axes(s.step, 0, s.q, s.k, s.v, s.q_out, s.rope, s.axes, s.positions, stream)
        return {"q": s.q_out, "cache": s.cache}
    if c["op"] == "attend_sinks":
        s.kvs.kvs_attend_sinks(s.step, 0, s.q, s.out, s.lse, s.scale, c["causal"], c["window"], c["sinks"], s.workspace, stream)
        return {"out": s.out, "lse": s.lse}
    s.kvs.kvs_weigh_sinks(s.step, 0, s.q, s.lse, s.weights, s.scale, c["decay"], c["causal"], c["window"], c["sinks"], stream)
    return {"weights": s.weights}


# ---- the definitions in 64 bits --------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    H, G, D, B = c["H"], c["G"], c["D"], c["B"]
    new, lens = _lengths(c)
    starts = np.concatenate([[0], np.cumsum(new)])
    tables = s.tables.cpu().numpy().astype(np.int64)

    def slots(r, at):
        return torch.from_numpy(tables[r, at // B] * B + at % B).to("cuda")

    if c["op"] == "append_axes":
        cache, q = s.cache.double(), s.q.double()
        pairs = len(s.axis)
        where = s.positions.cpu().numpy().astype(np.float64)[s.axis.cpu().numpy()]             # [pairs, N]
        angle = torch.from_numpy(where.T).to("cuda") * s.turns.double().sum(1) * (2 * math.pi)
        e = torch.polar(torch.ones_like(angle), angle)[:, None]
        lo = torch.arange(pairs, device="cuda") * (2 if c["inter"] else 1)
        hi = lo + (1 if c["inter"] else pairs)

        def turn(x):
            z = torch.complex(x[..., lo], x[..., hi]) * e
            x[..., lo], x[..., hi] = z.real, z.imag
            return x

        k, v = turn(s.k.double()), s.v.double()
        for r, (n, T) in enumerate(zip(new, lens)):
            slot = slots(r, np.arange(T - n, T))
            for p, x in enumerate((k, v)):
                cache[p].view(-1, H, D)[slot] = x[starts[r]: starts[r + 1]]
        return {"q": turn(q), "cache": cache}

    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros(s.N, H * G, D, **f64), torch.empty(s.N, H * G, **f64)
    weights = s.weights.double() if c["op"] == "weigh_sinks" else None
    for r, (n, T) in enumerate(zip(new, lens)):
        if weights is not None:
            weights[r, :, :T] = weights[r, :, :T] * c["decay"]
        # every token that is a sink, or in reach of the first new token's window or behind it
        t = np.array(sorted(set(range(min(T, c["sinks"]))) | set(range(max(0, T - n + 1 - c["window"]), T))), dtype=np.int64)
        slot, at = slots(r, t), torch.from_numpy(t).to("cuda")
        pos = torch.arange(T - n, T, device="cuda")[:, None]
        bad = (at <= pos - c["window"]) & (at >= c["sinks"])
        if c["causal"]:
            bad = bad | (at > pos)
        rows = slice(starts[r], starts[r + 1])
        for h in range(H):
            k = s.cache[0].view(-1, H, D)[slot, h].double()
            v = s.cache[1].view(-1, H, D)[slot, h].double()
            for g in range(h * G, h * G + G):
                x = (s.q[rows, g].double() @ k.T * s.scale).masked_fill_(bad, -math.inf)
                if weights is not None:
                    weights[r, h].index_add_(0, at, torch.exp(x - s.lse[rows, g, None].double()).sum(0))
                    continue
                z = torch.logsumexp(x, 1, keepdim=True)
                lse[rows, g] = z[:, 0]
                out[rows, g] = torch.exp(x - z) @ v
    return {"weights": weights} if weights is not None else {"out": out, "lse": lse}
