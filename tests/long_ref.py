"""Definitions in 64 bits of the operators with sinks and with axes, and the small steps that the tests
run them on: ops_ref's with a window's sinks in the mask, and with blocks given back."""
import numpy as np
import torch

import ops_ref
from ops_ref import Small


class Long(Small):
    """A step whose new tokens see a window and `sinks` first tokens.  What no token of a request sees is not a
    number in the cache, and blocks without a seen token are named by no valid table entry."""

    def __init__(self, new, lens, window, sinks, *a, causal=True, given_back=True, **kw):
        super().__init__(new, lens, *a, **kw)
        self.window, self.sinks, self.causal = window, sinks, causal
        rng = np.random.default_rng(7)
        self.hidden = []
        for r, T in enumerate(lens):
            hidden = ~self.seen(r, causal, window).any(0) if new[r] else np.zeros(T, dtype=bool)
            self.hidden.append(hidden)
            if not hidden.any():
                continue
            self.cache[:, torch.from_numpy(self.slots(r, np.nonzero(hidden)[0]))] = float("nan")
            if given_back:
                for b in range(-(-T // self.B)):
                    if hidden[b * self.B: (b + 1) * self.B].all():
                        self.tables[r, b] = int(rng.choice([-1, self.num_blocks, 2 ** 31 - 1, -2 ** 31]))

    def slots(self, r, t):
        """Of tokens that are there; others' slots are those of token 0."""
        t = np.asarray(t, dtype=np.int64)
        b = self.tables[r].numpy().astype(np.int64)[t // self.B]
        return np.where((b >= 0) & (b < self.num_blocks), b * self.B + t % self.B, 0)

    def seen(self, r, causal, window):
        n, T = self.new[r], self.lens[r]
        p, t = np.arange(T - n, T)[:, None], np.arange(T)[None, :]
        ok = np.ones((n, T), dtype=bool)
        if causal:
            ok &= t <= p
        if window:
            ok &= (t > p - window) | (t < self.sinks)
        return ok

    def scores(self, r, h, i, scale, causal, window, layer=0):
        at = self.slots(r, np.arange(self.lens[r]))
        there = ~self.hidden[r][:, None]
        k = np.where(there, self.cache[2 * layer, at, h].double().numpy(), 0.0)
        v = np.where(there, self.cache[2 * layer + 1, at, h].double().numpy(), 0.0)
        q = self.parts(self.qkv)[0][self.starts[r]: self.starts[r + 1], i].double().numpy()
        ok = self.seen(r, causal, window)
        s = np.where(ok, q @ k.T * scale, -np.inf)
        err = 2 * self.D * ops_ref.EPS * (np.abs(q) @ np.abs(k).T) * abs(scale) + 4 * ops_ref.EPS * np.where(ok, np.abs(s), 0.0)
        return s, err, v


def rotate_axes(x, positions, axis, turns, inter, scale=1.0):
    """Rotary positions in 64 bits: positions [axes, rows], axis [pairs], turns [pairs, 2]."""
    x = x.astype(np.float64).copy()
    pairs = len(axis)
    angle = 2 * np.pi * positions.astype(np.float64)[axis].T * turns.astype(np.float64).sum(1)
    c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
    rot = 2 * pairs
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, pairs), slice(pairs, rot))
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    return x
