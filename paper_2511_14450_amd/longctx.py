"""Decoder blocks over long contexts whose caches take 8 or 4 bits a number, and whose tokens read them whole or in selected blocks of keys.

What the four operators of mx.py do in one block:

    prompt   mx_write    the keys and values of a prompt's next chunk become codes, and move the bounds of their blocks of keys along
             mx_read     what its request holds by then, for attn_prompt: a row sees the same numbers as any later token
    token    mx_write    one key and value a request
             mx_select   the blocks of keys that can score highest with the token (read_blocks > 0)
             mx_token    attention over those, or over all

A context may also come from a stage that ran the prompts (`adopt`): its caches are exported and written as codes.

    python -m paper_2511_14450_amd.longctx --requests 8 --prompt 16384 --generate 64 --read-blocks 64
"""
from __future__ import annotations

import argparse
import contextlib
import json
import time
from typing import Dict, List, Sequence

import torch

from . import attn, binding, mx
from .shared import BlockMath


class LongBlocks(BlockMath):
    """Blocks over n_requests requests of up to `most` keys.

    k_format, v_format  "e4m3" (8 bits) or "e2m1" (4)
    read_blocks  blocks of block_keys keys that a token reads for each KV head, the first `sink` and the newest `recent` always; 0: all keys
    page_keys    keys in pages of so many (0: slabs); the page table, the same for all blocks, is the attribute page_table
    """

    def __init__(self, shape, layers: Sequence[Dict[str, torch.Tensor]], n_requests: int, most: int, k_format: str = "e4m3", v_format: str = "e4m3",
                 read_blocks: int = 0, block_keys: int = 64, sink: int = 1, recent: int = 4, page_keys: int = 0):
        if read_blocks < 0 or sink < 0 or recent < 0 or (read_blocks and sink + recent > read_blocks):
            raise ValueError("need sink + recent within read_blocks, none of them negative")
        if n_requests < 1 or most < 1:
            raise ValueError("need n_requests and most of at least 1")
        super().__init__(shape, layers)
        self.n, self.most, self.read_blocks, self.sink, self.recent = n_requests, most, read_blocks, sink, recent
        self.lens = torch.zeros(n_requests, dtype=torch.int32, device="cuda")
        self.page_table = None
        self.caches = []
        for _ in self.layers:
            self.caches.append(mx.MxCache.allocate(n_requests, shape.n_kv_heads, most, shape.head_dim, k_format, v_format, block_keys if read_blocks else 0, page_keys,
                                                   lens=self.lens, page_table=self.page_table))
            self.page_table = self.caches[0].page_table
        self.held = [0] * n_requests   # what lens counts, on the host

    def _grown(self, held: Sequence[int], counts: Sequence[int]) -> List[int]:
        if len(counts) != self.n or min(counts) < 0:
            raise ValueError("need a number of new tokens for every request")
        if any(h + c > self.most for h, c in zip(held, counts)):
            raise ValueError(f"a request would hold more than {self.most} keys")
        return [h + c for h, c in zip(held, counts)]

    @contextlib.contextmanager
    def _holding(self, held: List[int], otherwise: List[int]):
        """The requests hold so many keys, whom the caller counts in lens and writes, or so many others where that fails."""
        self.held = held
        try:
            yield
        except BaseException:
            self.held = otherwise
            self._count(otherwise)
            raise

    def _count(self, held: List[int]) -> None:
        self.lens.copy_(torch.tensor(held, dtype=torch.int32))

    def reset(self) -> None:
        """All requests start anew."""
        self.held = [0] * self.n
        self.lens.zero_()

    def prefill(self, hidden: torch.Tensor, seq_lens: Sequence[int]) -> torch.Tensor:
        """Hidden states [sum(seq_lens), H] of the requests' prompts, or of their next chunks (0 tokens of some, if any), through the blocks."""
        if hidden.shape[0] != sum(seq_lens):
            raise ValueError("need as many rows as seq_lens say")
        past, held, s = self.held, self._grown(self.held, seq_lens), self.shape
        if hidden.shape[0] == 0:
            return hidden
        with self._holding(held, past):
            self._count(held)
            start = torch.tensor([sum(seq_lens[:i]) for i in range(self.n + 1)], dtype=torch.int32).cuda()
            turn = self._turn(torch.cat([torch.arange(p, p + n) for p, n in zip(past, seq_lens)]).cuda())
            # room for what the requests hold, which all blocks use in turn
            k = torch.empty((self.n, s.n_kv_heads, max(held), s.head_dim), dtype=hidden.dtype, device="cuda")
            v = torch.empty_like(k)
            whole = attn.AttnCache(k, v, self.lens)
            x = hidden
            for w, cache in zip(self.layers, self.caches):
                q, new_k, new_v = self._qkv(w, x, turn)
                mx.mx_write(cache, new_k, new_v, q_start=start)
                mx.mx_read(cache, k, v)
                out, _ = attn.attn_prompt(whole, self.rule, q, start)
                x = self._rest(w, x, out)
        return x

    def decode_step(self, hidden: torch.Tensor) -> torch.Tensor:
        """The next token of every request, [n_requests, H]."""
        if hidden.shape[0] != self.n:
            raise ValueError("need one row for each request")
        turn, x = self._turn(self.lens), hidden
        with self._holding(self._grown(self.held, [1] * self.n), self.held):
            self.lens += 1
            for w, cache in zip(self.layers, self.caches):
                q, k, v = self._qkv(w, x, turn)
                mx.mx_write(cache, k, v)
                blocks = mx.mx_select(cache, q, self.read_blocks, self.sink, self.recent) if self.read_blocks else None
                out, _ = mx.mx_token(cache, self.rule, q, blocks=blocks)
                x = self._rest(w, x, out)
        return x

    def adopt(self, stage: binding.Stage, l_start: int, l_end: int) -> None:
        """The contexts of a stage's first n_requests requests, of the blocks [l_start, l_end) of the stage, which are these blocks; what was held is dropped,
        where a call is not refused."""
        s = self.shape
        if l_end - l_start != len(self.layers) or l_start < 0 or l_end > stage.l_end - stage.l_start:
            raise ValueError("need as many blocks of the stage as there are here")
        if (stage.cfg.n_kv_heads, stage.cfg.head_dim) != (s.n_kv_heads, s.head_dim):
            raise ValueError(f"need a stage of {s.n_kv_heads} KV heads of {s.head_dim} features")
        lens = self._grown([0] * self.n, [binding.stage_context_len(stage, b) for b in range(self.n)])
        with self._holding(lens, [0] * self.n):
            self._count(lens)
            start = torch.tensor([sum(lens[:i]) for i in range(self.n + 1)], dtype=torch.int32).cuda()
            for l, cache in zip(range(l_start, l_end), self.caches):
                rows = [torch.cat(t).view(-1, s.n_kv_heads, s.head_dim) for t in zip(*(stage.export_kv(l, b) for b in range(self.n)))]
                mx.mx_write(cache, *rows, q_start=start)

    def cache_bytes(self) -> int:
        return sum(t.numel() * t.element_size() for c in self.caches for t in (c.k, c.v, c.k_scale, c.v_scale, c.lo, c.hi) if t is not None)


def _arguments(models: Sequence[str], argv=None) -> argparse.Namespace:
    def at_least(least):
        def number(text):
            if (value := int(text)) < least:
                raise argparse.ArgumentTypeError(f"{value} is less than {least}")
            return value
        return number

    ap = argparse.ArgumentParser(prog="python -m paper_2511_14450_amd.longctx", description=__doc__.split("\n\n")[0])
    ap.add_argument("--model", choices=models, default="phi3_medium")
    ap.add_argument("--blocks", type=at_least(1), default=2)
    ap.add_argument("--requests", type=at_least(1), default=8)
    ap.add_argument("--prompt", type=at_least(1), default=16384, help="tokens of each request's prompt")
    ap.add_argument("--chunk", type=at_least(1), default=4096, help="of which so many at a time")
    ap.add_argument("--generate", type=at_least(0), default=64)
    ap.add_argument("--k-format", choices=sorted(mx.MX_FORMATS), default="e4m3")
    ap.add_argument("--v-format", choices=sorted(mx.MX_FORMATS), default="e4m3")
    ap.add_argument("--read-blocks", type=at_least(0), default=0, help="blocks of keys that a token reads (0: all keys)")
    ap.add_argument("--block-keys", type=at_least(16), help="keys of a block: a power of two up to 4096, by default 64 or, if less, the page's")
    ap.add_argument("--sink", type=at_least(0), help="first blocks that a token always reads, by default 1 where that leaves room for the newest")
    ap.add_argument("--recent", type=at_least(0), help="newest blocks that a token always reads, by default 4 or, if less, what sink leaves")
    ap.add_argument("--page-keys", type=at_least(0), default=0, help="keys of a page: a power of two from 16 on (0: slabs)")
    ap.add_argument("--seed", type=int, default=251114450)
    a = ap.parse_args(argv)
    power_of_two = lambda v: v & (v - 1) == 0  # noqa: E731
    if a.page_keys and (a.page_keys < 16 or not power_of_two(a.page_keys)):
        ap.error("--page-keys: need a power of two from 16 on")
    if a.block_keys is None:
        a.block_keys = min(64, a.page_keys or 64)
    if a.block_keys > (a.page_keys or 4096) or a.block_keys > 4096 or not power_of_two(a.block_keys):
        ap.error("--block-keys: need a power of two from 16 to 4096 that divides --page-keys")
    if a.sink is None:
        a.sink = min(1, max(0, a.read_blocks - (1 if a.recent is None else a.recent)))
    if a.recent is None:
        a.recent = min(4, max(0, a.read_blocks - a.sink))
    if a.read_blocks and a.sink + a.recent > a.read_blocks:
        ap.error("--sink and --recent: need no more than --read-blocks together")
    return a


def main():
    from .chain import MODELS, _Shape, _synthetic_layer
    a = _arguments(sorted(MODELS))
    shape = _Shape(MODELS[a.model])
    make = _synthetic_layer(shape, a.seed)
    layers = [make(l) for l in range(a.blocks)]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(a.seed + 13)
    draw = lambda rows: torch.randn((rows, shape.hidden), generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    blocks = LongBlocks(shape, layers, a.requests, a.prompt + a.generate, a.k_format, a.v_format, a.read_blocks, a.block_keys, a.sink, a.recent,
                        a.page_keys)
    chunks = [min(a.chunk, a.prompt - at) for at in range(0, a.prompt, a.chunk)]
    inputs = [draw(a.requests * n) for n in chunks]

    def run(steps):
        blocks.reset()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        for n, x in zip(chunks, inputs):
            h = blocks.prefill(x, [n] * a.requests)
        h = h[torch.arange(1, a.requests + 1, device="cuda") * chunks[-1] - 1]
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        for _ in range(steps):
            h = blocks.decode_step(h)
        torch.cuda.synchronize()
        return t1 - t0, time.perf_counter() - t1

    run(min(2, a.generate))  # there is room for no more
    prompt, tokens = run(a.generate)
    print(json.dumps(dict(model=a.model, blocks=a.blocks, requests=a.requests, prompt=a.prompt, generate=a.generate, k_format=a.k_format, v_format=a.v_format,
                          read_blocks=a.read_blocks, block_keys=a.block_keys, sink=a.sink, recent=a.recent, prompt_ms=prompt * 1e3,
                          token_ms=tokens * 1e3 / max(a.generate, 1), cache_mib=blocks.cache_bytes() / 2**20,
                          cache_mib_bf16=a.requests * (a.prompt + a.generate) * 4 * shape.n_kv_heads * shape.head_dim * a.blocks / 2**20)))


if __name__ == "__main__":
    main()
