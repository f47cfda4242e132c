"""Decoder blocks over requests that start with the same text and answer within a fixed number of cached keys.

The shared text is run once, by a stage (binding.stage_prefill), and its keys and values are exported; every request then
has only its own prompt in a cache, meets the shared keys where they are, and after its prompt and whenever its cache is
full drops the keys that received the least attention.  What the four operators of attn.py do in one block:

    prompt      attn_prompt    rows of all requests over shared and own keys
                attn_received  the weight each own key got from a prompt's last rows
                attn_evict     the `budget` keys worth keeping, into the request's cache
    token       attn_token     one row a request, its weights added to the totals
    cache full  attn_evict     in place, down to the budget again

Projections, norms and the FFN are PyTorch's; a request whose keys all fit gives what a stage gives that ran
shared text and prompt together.  Keys are cached as the stage caches them, after RoPE, so a key that stays needs no work.

    python -m paper_2511_14450_amd.shared --requests 16 --prefix 4096 --prompt 2048 --generate 256 --budget 1024
"""
from __future__ import annotations

import argparse
import json
import time
from typing import Dict, List, Sequence, Tuple

import torch
import torch.nn.functional as F

from . import attn, binding


def shared_prefix(stage: binding.Stage, l_start: int, l_end: int, request: int = 0) -> List[Tuple[torch.Tensor, torch.Tensor]]:
    """Keys and values [kv heads, keys, d] of one request of a stage, a pair for each of its blocks."""
    out = []
    for l in range(l_start, l_end):
        out.append(tuple(t.view(t.shape[0], stage.cfg.n_kv_heads, stage.cfg.head_dim).transpose(0, 1) for t in stage.export_kv(l, request)))
    return out


class SharedBlocks:
    """Blocks over n_requests requests that share `prefix` (shared_prefix of the same blocks).

    budget  own keys of a request and KV head that stay after its prompt and after an eviction
    room    tokens between evictions
    sink, recent  how many of the first and the newest own keys always stay
    window  rows of a prompt's end whose attention decides which of its keys stay (0: all of them)
    """

    def __init__(self, shape, layers: Sequence[Dict[str, torch.Tensor]], prefix: Sequence[Tuple[torch.Tensor, torch.Tensor]],
                 n_requests: int, budget: int, room: int, sink: int = 4, recent: int = 32, window: int = 64):
        if len(prefix) != len(layers):
            raise ValueError("prefix: need keys and values of every block")
        if budget < 1 or room < 1 or sink < 0 or recent < 0 or sink + recent > budget:
            raise ValueError("need budget and room of at least 1, and sink + recent within the budget")
        self.shape, self.layers, self.prefix = shape, list(layers), list(prefix)
        self.n, self.budget, self.room, self.sink, self.recent, self.window = n_requests, budget, room, sink, recent, window
        self.prefix_len = prefix[0][0].shape[1] if prefix else 0
        self.rule = attn.AttnRule(shape.head_dim ** -0.5)
        i = torch.arange(shape.head_dim // 2, dtype=torch.float64, device="cuda")
        self.angle = shape.rope_base ** (-2.0 * i / shape.head_dim)
        dtype = prefix[0][0].dtype
        sizes = (n_requests, shape.n_kv_heads, budget + room)
        self.k = [torch.empty((*sizes, shape.head_dim), dtype=dtype, device="cuda") for _ in layers]
        self.v = [torch.empty_like(k) for k in self.k]
        self.pos = [torch.zeros(sizes, dtype=torch.int32, device="cuda") for _ in layers]
        self.totals = [torch.zeros(sizes, dtype=torch.float32, device="cuda") for _ in layers]
        self.lens = [torch.zeros(n_requests, dtype=torch.int32, device="cuda") for _ in layers]
        self.caches = [attn.AttnCache(k, v, n, prefix_k=p[0], prefix_v=p[1], key_pos=pos)
                       for k, v, n, p, pos in zip(self.k, self.v, self.lens, self.prefix, self.pos)]
        self.now = torch.full((n_requests,), self.prefix_len, dtype=torch.int32, device="cuda")  # position of the next token
        self.most = 0  # keys that the longest request holds
        self.requests = torch.arange(n_requests, device="cuda")

    def _norm(self, x, g):
        y = x.float()
        return (y * torch.rsqrt(y.pow(2).mean(-1, keepdim=True) + self.shape.rms_eps) * g.float()).to(x.dtype)

    def _rope(self, x, turn):
        a, b = x.float().chunk(2, dim=-1)
        cos, sin = turn
        return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1).to(x.dtype)

    def _turn(self, pos):
        angle = (pos.double()[:, None] * self.angle)[:, None]
        return angle.cos().float(), angle.sin().float()

    def _qkv(self, w, x, turn):
        s, h = self.shape, self._norm(x, w["attn_norm_g"])
        q, k, v = (F.linear(h, w[name]).view(x.shape[0], -1, s.head_dim) for name in ("wq", "wk", "wv"))
        return self._rope(q, turn), self._rope(k, turn), v

    def _rest(self, w, x, out):
        x = x + F.linear(out.reshape(x.shape[0], -1), w["wo"])
        h = self._norm(x, w["ffn_norm_g"])
        return x + F.linear(F.silu(F.linear(h, w["w_gate"])) * F.linear(h, w["w_up"]), w["w_down"])

    def prefill(self, hidden: torch.Tensor, seq_lens: Sequence[int]) -> torch.Tensor:
        """Hidden states [sum(seq_lens), H] of the requests' own prompts through the blocks; their caches start anew."""
        if len(seq_lens) != self.n or min(seq_lens) < 1 or hidden.shape[0] != sum(seq_lens):
            raise ValueError("need a prompt of one token or more for every request")
        s, longest = self.shape, max(seq_lens)
        lens = torch.tensor(seq_lens, dtype=torch.int32).cuda()
        start = torch.cat((lens.new_zeros(1), lens.cumsum(0, dtype=torch.int32)))
        request = torch.repeat_interleave(self.requests, lens.long(), output_size=hidden.shape[0])
        slot = torch.arange(hidden.shape[0], device="cuda") - start[request]
        turn = self._turn(self.prefix_len + slot)
        # room for whole prompts, which all blocks use in turn
        k = torch.empty((self.n, s.n_kv_heads, longest, s.head_dim), dtype=hidden.dtype, device="cuda")
        v, totals = torch.empty_like(k), torch.empty(k.shape[:3], dtype=torch.float32, device="cuda")
        x = hidden
        for w, cache, prefix, kept in zip(self.layers, self.caches, self.prefix, self.totals):
            prompt = attn.AttnCache(k, v, lens, prefix_k=prefix[0], prefix_v=prefix[1])
            q, k[request, :, slot], v[request, :, slot] = self._qkv(w, x, turn)
            out, lse = attn.attn_prompt(prompt, self.rule, q, start)
            attn.attn_received(prompt, self.rule, q, start, lse, totals.zero_(), last=self.window)
            attn.attn_evict(prompt, totals, self.budget, self.sink, self.recent, into=cache, totals_out=kept)
            x = self._rest(w, x, out)
        self.now.copy_(lens + self.prefix_len)
        self.most = min(longest, self.budget)
        return x

    def decode_step(self, hidden: torch.Tensor) -> torch.Tensor:
        """The next token of every request, [n_requests, H]."""
        if hidden.shape[0] != self.n:
            raise ValueError("need one row for each request")
        full = self.most == self.budget + self.room
        turn, x = self._turn(self.now), hidden
        for w, cache, k, v, pos, totals, lens in zip(self.layers, self.caches, self.k, self.v, self.pos, self.totals, self.lens):
            if full:
                attn.attn_evict(cache, totals, self.budget, self.sink, self.recent, now=self.now)
            at = lens.long()
            q, k[self.requests, :, at], v[self.requests, :, at] = self._qkv(w, x, turn)
            pos[self.requests, :, at] = self.now[:, None].expand(-1, pos.shape[1])
            totals[self.requests, :, at] = 0.0
            lens += 1
            out, _ = attn.attn_token(cache, self.rule, q, totals=totals)
            x = self._rest(w, x, out)
        self.now += 1
        self.most = (self.budget if full else self.most) + 1
        return x


def main():
    from .chain import MODELS, _Shape, _synthetic_layer
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--model", choices=sorted(MODELS), default="phi3_medium")
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prefix", type=int, default=4096, help="tokens that all requests start with")
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of each request's own prompt")
    ap.add_argument("--generate", type=int, default=256)
    ap.add_argument("--budget", type=int, default=1024, help="own keys that stay")
    ap.add_argument("--room", type=int, default=128, help="tokens between evictions")
    ap.add_argument("--seed", type=int, default=251114450)
    a = ap.parse_args()
    shape = _Shape(MODELS[a.model])
    make = _synthetic_layer(shape, a.seed)
    layers = [make(l) for l in range(a.blocks)]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(a.seed + 11)
    draw = lambda rows: torch.randn((rows, shape.hidden), generator=gen, device="cuda").to(torch.bfloat16)
    stage = binding.stage_create(binding.stage_config(shape, 1, a.prefix, a.prefix), 0, a.blocks, layers)
    binding.stage_prefill(stage, draw(a.prefix), [a.prefix])
    blocks = SharedBlocks(shape, layers, shared_prefix(stage, 0, a.blocks), a.requests, a.budget, a.room)
    stage.destroy()
    prompts, ends = draw(a.requests * a.prompt), torch.arange(1, a.requests + 1, device="cuda") * a.prompt - 1

    def run(steps):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        h = blocks.prefill(prompts, [a.prompt] * a.requests)[ends]
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        for _ in range(steps):
            h = blocks.decode_step(h)
        torch.cuda.synchronize()
        return t1 - t0, time.perf_counter() - t1

    run(2)
    prompt, tokens = run(a.generate)
    key = 2 * shape.n_kv_heads * shape.head_dim * 2 * a.blocks
    print(json.dumps(dict(model=a.model, blocks=a.blocks, requests=a.requests, prefix=a.prefix, prompt=a.prompt, generate=a.generate,
                          budget=a.budget, prompt_ms=prompt * 1e3, token_ms=tokens * 1e3 / max(a.generate, 1),
                          cache_mib=(a.prefix + a.requests * (a.budget + a.room)) * key / 2**20,
                          cache_mib_unshared_whole=a.requests * (a.prefix + a.prompt + a.generate) * key / 2**20)))


if __name__ == "__main__":
    main()
