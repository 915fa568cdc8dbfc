"""The model operators in 64 bits, written from their definitions (numpy on the CPU), and the
small steps that the tests run them on.

Error bounds are those of the operators' arithmetic: products and sums in binary32 (unit
roundoff 2^-24; a matrix product's sum of D terms is off by at most D roundoffs of the sum of
its terms' magnitudes, and twice that where the hardware truncates), exponentials within 2^-21,
one rounding to the 16-bit type (2^-8 for the 8 significant bits of bfloat16, 2^-11 for half) of the attention weights
and one of the outputs."""
import numpy as np
import torch

EPS = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TYPE = {"bf16": torch.bfloat16, "f16": torch.float16}


class Small:
    """One layer's cache and step: `new` and `lens` are the requests' new and cached tokens."""

    def __init__(self, new, lens, H=2, G=2, D=64, B=16, dtype="bf16", seed=0, spread=1.0, L=1, extra_blocks=5):
        self.new, self.lens, self.H, self.G, self.D, self.B, self.dtype, self.L = list(new), list(lens), H, G, D, B, dtype, L
        g = torch.Generator().manual_seed(seed)
        self.R, self.N = len(lens), sum(new)
        self.W = max(1, -(-max(list(lens) + [1]) // B))
        self.num_blocks = self.R * self.W + extra_blocks
        self.tables = torch.randperm(self.num_blocks, generator=g)[: self.R * self.W].view(self.R, self.W).to(torch.int32)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        dt = TYPE[dtype]
        # what no request's tokens use is not a number
        self.cache = torch.full((2 * L, self.num_blocks * B, H, D), float("nan"), dtype=dt)
        for r, T in enumerate(lens):
            at = self.slots(r, np.arange(T))
            self.cache[:, at] = (torch.randn(2 * L, T, H, D, generator=g) * spread).to(dt)
        # rows of a wider buffer, as a fused projection leaves them
        self.qkv = torch.randn(max(1, self.N), (H * G + 2 * H) * D, generator=g).to(dt)[: self.N]

    def slots(self, r, t):
        t = np.asarray(t, dtype=np.int64)
        return self.tables[r].numpy().astype(np.int64)[t // self.B] * self.B + t % self.B

    def parts(self, qkv):
        H, G, D = self.H, self.G, self.D
        return (qkv[:, : H * G * D].view(-1, H * G, D), qkv[:, H * G * D: H * (G + 1) * D].view(-1, H, D),
                qkv[:, H * (G + 1) * D:].view(-1, H, D))

    def on_gpu(self, kvs, decode=False, chunk_tokens=256):
        """(step, q, k, v, cache) on the GPU."""
        cache = self.cache.cuda().view(2 * self.L, self.num_blocks, self.B, self.H, self.D)
        dev = dict(device="cuda", dtype=torch.int32)
        lens, starts = torch.tensor(self.lens, **dev), torch.tensor(self.starts, **dev)
        step = kvs.Step((self.L, self.H, self.D, 2, self.B, self.B), [cache[p].data_ptr() for p in range(2 * self.L)], self.num_blocks,
                        self.tables.cuda(), lens, None if decode else starts, total_q=self.N, max_q=max(self.new + [0]),
                        dtype=kvs.KVS_DTYPE_BF16 if self.dtype == "bf16" else kvs.KVS_DTYPE_F16)
        return (step, *self.parts(self.qkv.cuda()), cache)

    def seen(self, r, causal, window):
        n, T = self.new[r], self.lens[r]
        p, t = np.arange(T - n, T)[:, None], np.arange(T)[None, :]
        ok = np.ones((n, T), dtype=bool)
        if causal:
            ok &= t <= p
        if window:
            ok &= t > p - window
        return ok

    def scores(self, r, h, i, scale, causal, window, layer=0):
        """Of request r's new tokens and query head i: masked scores, their error, V in 64 bits."""
        at = self.slots(r, np.arange(self.lens[r]))
        k = self.cache[2 * layer, at, h].double().numpy()
        v = self.cache[2 * layer + 1, at, h].double().numpy()
        q = self.parts(self.qkv)[0][self.starts[r]: self.starts[r + 1], i].double().numpy()
        ok = self.seen(r, causal, window)
        s = np.where(ok, q @ k.T * scale, -np.inf)
        err = 2 * self.D * EPS * (np.abs(q) @ np.abs(k).T) * abs(scale) + 4 * EPS * np.where(ok, np.abs(s), 0.0)
        return s, err, v

    def attend(self, scale, causal=True, window=0, layer=0):
        """(out, out's error, lse, lse's error)."""
        heads = self.H * self.G
        out, bound = np.zeros((self.N, heads, self.D)), np.zeros((self.N, heads, self.D))
        lse, lse_bound = np.full((self.N, heads), -np.inf), np.zeros((self.N, heads))
        u = UNIT[self.dtype]
        for r, T in enumerate(self.lens):
            rows = slice(self.starts[r], self.starts[r + 1])
            for i in range(heads):
                s, err, v = self.scores(r, i // self.G, i, scale, causal, window, layer)
                some = np.isfinite(s).any(1)
                if not some.any():
                    continue
                m = np.where(some, s.max(1, initial=-np.inf), 0.0)[:, None]
                p = np.exp(s - m)
                l = p.sum(1, keepdims=True)
                o, a = p @ v / np.where(l == 0, 1, l), p @ np.abs(v) / np.where(l == 0, 1, l)
                ds = err.max(1, initial=0.0)[:, None]
                rel = 2 * ds + 2.0 ** -20 + 2 * (T + 16) * EPS
                # half rounds small weights to multiples of 2^-24
                tiny = T * 2.0 ** -25 * np.abs(v).max(initial=0.0) if self.dtype == "f16" else 0.0
                out[rows, i], bound[rows, i] = o, u * (1.01 * a + np.abs(o)) + rel * a + tiny + 1e-30
                with np.errstate(divide="ignore"):
                    lse[rows, i] = np.where(some, (m + np.log(l))[:, 0], -np.inf)
                lse_bound[rows, i] = (ds + 2.0 ** -20 + (T + 16) * EPS)[:, 0] + 4 * EPS * np.where(some, np.abs(lse[rows, i]), 0.0)
        return out, bound, lse, lse_bound

    def weigh(self, lse, before, decay, scale, causal=True, window=0):
        """(weights, their error), from binary32 lse [N, heads] and the weights before."""
        w, bound = before.astype(np.float64).copy(), np.zeros(before.shape)
        lse = lse.astype(np.float64)
        for r, T in enumerate(self.lens):
            rows = slice(self.starts[r], self.starts[r + 1])
            for h in range(self.H):
                old = np.zeros(T) if decay == 0 else w[r, h, :T] * decay
                total, off = old.copy(), 4 * EPS * np.abs(old)
                for i in range(h * self.G, (h + 1) * self.G):
                    s, err, _ = self.scores(r, h, i, scale, causal, window)
                    z = lse[rows, i, None]
                    with np.errstate(invalid="ignore"):
                        p = np.where(np.isfinite(s), np.exp(s - z), 0.0)
                    rel = 1.5 * (err + 8 * EPS * np.abs(np.where(np.isfinite(z), z, 0.0))) + 2.0 ** -20 + (self.new[r] * self.G + 16) * EPS
                    total += p.sum(0)
                    off += (p * rel).sum(0)
                w[r, h, :T], bound[r, h, :T] = total, off + 1e-30
        return w, bound


def rotate(x, positions, turns, rot, interleaved, scale=1.0):
    """Rotary positions in 64 bits; turns [rot / 2, 2]."""
    x = x.astype(np.float64).copy()
    angle = 2 * np.pi * (positions.astype(np.float64)[:, None] * turns.astype(np.float64).sum(1))
    c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    return x


def evict(weights, lens, budget, sinks, recent):
    """kept [L, R, H, budget] by the definition: sorted by (always kept, weight, lower index)."""
    L, R, H, _ = weights.shape
    kept = np.full((L, R, H, budget), -1, dtype=np.int64)
    for l in range(L):
        for r in range(R):
            T = lens[r]
            t = np.arange(T)
            always = (t < sinks) | (t >= T - recent)
            for h in range(H):
                w = weights[l, r, h, :T].astype(np.float64)
                nan = np.isnan(w)
                order = sorted(range(T), key=lambda i: (not always[i], nan[i], 0.0 if nan[i] else -w[i], i))
                keep = sorted(order[:budget])
                kept[l, r, h, : len(keep)] = keep
    return kept
