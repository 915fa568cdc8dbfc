"""A model's forward steps on a retrieved prefix: all operators of the paged cache together.

``python -m paper_2609_35065_gb300.prefix_step`` takes a small decoder of random weights
(projections by torch) through what a serving loop does with this library:

1. prompt A is prefilled and its complete chunks are stored to pinned host memory (``kvs_store``);
2. request B, whose prompt begins with A's, gets that prefix back into other blocks of the cache
   (``kvs_retrieve``) and prefills only its own suffix: each layer rotates and appends its new
   keys and values (``kvs_append``) and attends over prefix and suffix (``kvs_attend``);
3. some tokens are decoded, each layer adding up what its cached tokens were given
   (``kvs_weigh``);
4. the cache is cut to a budget (``kvs_evict``) and decoding goes on over what was kept.

With ``--session`` the decoder is one for long sessions over pictures: positions on three axes
(``kvs_append_axes``), a window beside which the first tokens stay visible (``kvs_attend_sinks``,
``kvs_weigh_sinks``), and blocks that nobody sees any more given back before decoding.

It prints how far B's suffix comes out from a prefill of the whole prompt.
"""
from __future__ import annotations

import sys
from dataclasses import dataclass

import numpy as np
import torch

from . import kvs


@dataclass
class Config:
    layers: int = 4
    kv_heads: int = 2
    group: int = 4                     # query heads per KV head
    head_dim: int = 64
    block: int = 16
    chunk: int = 256
    num_blocks: int = 512
    vocab: int = 1000
    dtype: torch.dtype = torch.bfloat16
    window: int = 0                    # tokens that a token sees; 0: all before it
    sinks: int = 0                     # first tokens that it sees beside a window
    axes: tuple = ()                   # rotated pairs of each axis; (): positions are on one


class Decoder:
    """A decoder of random weights whose attention reads the paged cache."""

    def __init__(self, cfg: Config, seed: int = 0, device: str = "cuda"):
        self.cfg, self.device = cfg, device
        g = torch.Generator(device).manual_seed(seed)
        H, G, D = cfg.kv_heads, cfg.group, cfg.head_dim
        self.width = H * G * D

        def weight(n, m):
            return (torch.randn(n, m, generator=g, device=device) / n ** 0.5).to(cfg.dtype)

        self.embed = torch.randn(cfg.vocab, self.width, generator=g, device=device).to(cfg.dtype)
        self.qkv = [weight(self.width, (G + 2) * H * D) for _ in range(cfg.layers)]
        self.out = [weight(self.width, self.width) for _ in range(cfg.layers)]
        self.cache = torch.zeros(2 * cfg.layers, cfg.num_blocks, cfg.block, H, D, dtype=cfg.dtype, device=device)
        self.geom = (cfg.layers, H, D, 2, cfg.block, cfg.chunk)
        self.planes = [self.cache[p].data_ptr() for p in range(2 * cfg.layers)]
        self.axes = None
        if cfg.axes:
            turns, axis, scale = kvs.kvs_rope_axes(cfg.axes, 10000.0)
            self.axes = kvs.Axes(torch.from_numpy(axis).to(device), len(cfg.axes))
        else:
            turns, scale = kvs.kvs_rope_turns(D, 10000.0)
        self.rope = kvs.Rope(torch.from_numpy(turns).to(device), 2 * len(turns), scale=scale)

    def step(self, tables, kv_lens, q_starts=None, total_q=None, max_q=None):
        return kvs.Step(self.geom, self.planes, self.cfg.num_blocks, tables, kv_lens, q_starts, total_q=total_q, max_q=max_q,
                        dtype=kvs.KVS_DTYPE_F16 if self.cfg.dtype == torch.float16 else kvs.KVS_DTYPE_BF16)

    def forward(self, step, tokens, positions=None, weights=None):
        """Logits of the step's new tokens, which are appended to the cache; ``positions`` [tokens], or [axes,
        tokens] where there are several; ``weights`` [layers, requests, KV heads, tokens] are added to."""
        cfg = self.cfg
        H, G, D = cfg.kv_heads, cfg.group, cfg.head_dim
        n, s = len(tokens), torch.cuda.current_stream()
        mask = dict(window=cfg.window, sinks=cfg.sinks)
        need = kvs.kvs_attend_sinks_workspace(step, H * G, **mask) if cfg.window else kvs.kvs_attend_workspace(step, H * G)
        workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        lse = torch.empty(n, H * G, device=self.device)
        x = self.embed[tokens]
        for layer in range(cfg.layers):
            normed = (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(cfg.dtype)
            qkv = normed @ self.qkv[layer]
            q = qkv[:, : H * G * D].view(n, H * G, D)
            k = qkv[:, H * G * D: H * (G + 1) * D].view(n, H, D)
            v = qkv[:, H * (G + 1) * D:].view(n, H, D)
            if self.axes is None:
                kvs.kvs_append(step, layer, q, k, v, None, self.rope, positions, s)
            else:
                kvs.kvs_append_axes(step, layer, q, k, v, None, self.rope, self.axes, positions, s)
            out = torch.empty(n, H * G, D, dtype=cfg.dtype, device=self.device)
            if cfg.window:
                kvs.kvs_attend_sinks(step, layer, q, out, lse, workspace=workspace, stream=s, **mask)
            else:
                kvs.kvs_attend(step, layer, q, out, lse, workspace=workspace, stream=s)
            if weights is not None and cfg.window:
                kvs.kvs_weigh_sinks(step, layer, q, lse, weights[layer], stream=s, **mask)
            elif weights is not None:
                kvs.kvs_weigh(step, layer, q, lse, weights[layer], stream=s)
            x = x + out.view(n, -1) @ self.out[layer]
        return x.float() @ self.embed.float().T


def prompt_positions(cfg: Config, n: int) -> torch.Tensor:
    """int32 positions of a prompt's tokens; on several axes every 100 tokens of text are followed by a picture of
    8 x 12, whose last two axes are a row and a column."""
    if not cfg.axes:
        return torch.arange(n, dtype=torch.int32)
    at, p = torch.empty(len(cfg.axes), n + 200, dtype=torch.int32), 0
    for start in range(0, n, 196):
        at[:, start: start + 100] = p + torch.arange(100)
        k = torch.arange(96)
        at[:, start + 100: start + 196] = p + 100
        at[-2, start + 100: start + 196] += k // 12
        at[-1, start + 100: start + 196] += k % 12
        p += 112
    return at[:, :n].contiguous()


def next_position(at: torch.Tensor) -> torch.Tensor:
    """Position of a token of text behind those at `at` ([tokens] or [axes, tokens]): behind the largest, the same on every axis."""
    return (at.amax() + 1).to(torch.int32).repeat(at.shape[:-1] + (1,))


def run(cfg: Config = Config(), prefix: int = 600, suffix: int = 90, decode: int = 12, budget: int = 320, seed: int = 0) -> dict:
    """The four steps above; returns what they gave."""
    model = Decoder(cfg, seed)
    dev, rng = model.device, np.random.default_rng(seed)
    perm = rng.permutation(cfg.num_blocks).astype(np.int32)
    per = -(-(prefix + suffix + 2 * decode) // cfg.block)
    tables = [perm[k * per: (k + 1) * per] for k in range(3)]
    prompt = torch.from_numpy(rng.integers(0, cfg.vocab, prefix + suffix)).to(dev)
    at = prompt_positions(cfg, prefix + suffix).to(dev)

    def one(table, cached, new):
        i32 = dict(dtype=torch.int32, device=dev)
        return model.step(torch.from_numpy(table)[None].to(dev), torch.tensor([cached], **i32), torch.tensor([0, new], **i32), new, new)

    # 1: the whole prompt, and its complete chunks to the fast tier
    whole = model.forward(one(tables[0], prefix + suffix, prefix + suffix), prompt, at)
    stored = prefix // cfg.chunk * cfg.chunk
    elems = 2 * cfg.layers * cfg.chunk * cfg.kv_heads * cfg.head_dim
    chunks = [torch.empty(elems, dtype=cfg.dtype, pin_memory=True) for _ in range(stored // cfg.chunk)]
    kvs.kvs_store(model.geom, model.planes, cfg.num_blocks, [kvs.RequestArg(tables[0], [kvs.ChunkArg(c, cfg.chunk) for c in chunks])])

    # 2: the prefix into request B's blocks, and the rest of its prompt on top
    kvs.kvs_retrieve(model.geom, model.planes, cfg.num_blocks, [kvs.RequestArg(tables[1], [kvs.ChunkArg(c, cfg.chunk) for c in chunks])])
    rest = len(prompt) - stored
    logits = model.forward(one(tables[1], len(prompt), rest), prompt[stored:], at[..., stored:].contiguous())

    # 3: decoding, with the weight that each cached token receives; what no token will see is another's by now
    cached = len(prompt)
    if cfg.window:
        block = np.arange(per)
        gone = (block * cfg.block >= cfg.sinks) & ((block + 1) * cfg.block <= cached + 1 - cfg.window)
        model.cache[:, tables[1][gone]] = float("nan")
        tables[1][gone] = -1
    table = torch.from_numpy(tables[1])[None].to(dev)
    weights = torch.zeros(cfg.layers, 1, cfg.kv_heads, per * cfg.block, device=dev)
    lens = torch.tensor([cached], dtype=torch.int32, device=dev)
    position = next_position(at)
    token, tokens = logits[-1:].argmax(-1), []

    def decode_some(step, weights):
        nonlocal token
        for _ in range(decode):
            tokens.append(token)
            step_logits = model.forward(step, token, position, weights)
            token = step_logits.argmax(-1)
            lens.add_(1)
            position.add_(1)

    lens.add_(1)
    decode_some(model.step(table, lens), weights)
    lens.sub_(1)

    if cfg.window:
        kvs.kvs_check_errors()
        return {"whole": whole[stored:], "suffix": logits, "stored": stored, "tokens": torch.cat(tokens), "kept": None, "weights": weights,
                "cached": len(prompt) + decode, "gone": int(gone.sum())}

    # 4: at most `budget` tokens of every head, in fresh blocks; rotary positions go on
    cut = torch.from_numpy(tables[2])[None].to(dev)
    kept = torch.empty(cfg.layers, 1, cfg.kv_heads, budget, dtype=torch.int32, device=dev)
    new_weights, new_lens = torch.empty(kept.shape, device=dev), torch.empty(1, dtype=torch.int32, device=dev)
    kvs.kvs_evict(model.step(table, lens), weights, cut, budget, 4, 64, kept, new_weights, new_lens)
    lens.copy_(new_lens).add_(1)
    weights.zero_()[..., :budget] = new_weights
    decode_some(model.step(cut, lens), weights)
    kvs.kvs_check_errors()
    return {"whole": whole[stored:], "suffix": logits, "stored": stored, "tokens": torch.cat(tokens), "kept": kept, "weights": weights,
            "cached": len(prompt) + decode}


def session() -> Config:
    """A decoder for long sessions over pictures."""
    return Config(window=128, sinks=4, axes=(8, 12, 12))


def main() -> None:
    r = run(session() if "--session" in sys.argv[1:] else Config())
    off = (r["suffix"] - r["whole"]).norm() / r["whole"].norm()
    if r["kept"] is None:
        print(f"{r['stored']} tokens retrieved, {len(r['suffix'])} prefilled on top: logits {off:.2%} off those of the whole prompt's prefill; "
              f"{r['gone']} blocks given back, {len(r['tokens'])} decoded over the rest")
        return
    print(f"{r['stored']} tokens retrieved, {len(r['suffix'])} prefilled on top: logits {off:.2%} off those of the whole prompt's prefill, "
          f"{(r['suffix'].argmax(-1) == r['whole'].argmax(-1)).float().mean():.0%} of the next tokens the same; "
          f"{len(r['tokens'])} decoded, the cache cut from {r['cached']} to {r['kept'].shape[-1]} tokens on the way")


if __name__ == "__main__":
    main()
