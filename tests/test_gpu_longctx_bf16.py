"""Blocks over long contexts in bf16: what their attention gives, against the formula in 64 bits over the numbers that the formats hold."""
import pytest
import torch

from tests import mx_reference as ref
from tests.helpers import to_dev
from tests.test_gpu_mx_probabilities import bound
from workloads import synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(v_format="e2m1", page_keys=32), dict(k_format="e2m1", v_format="e2m1", read_blocks=4, block_keys=16, sink=1, recent=2),
                                dict(read_blocks=3, block_keys=16, sink=0, recent=1, page_keys=16)])
def test_attention_of_prompts_and_tokens(kw, monkeypatch):
    from paper_2511_14450_amd import longctx
    shape, lens, more, steps = synth.TINY_BF16, [60, 5, 97], [30, 0, 11], 4
    weights = [{k: to_dev(v, shape.dtype) for k, v in synth.layer_weights(shape, l, 3, sigma=0.05).items()} for l in range(2)]
    blocks = longctx.LongBlocks(shape, weights, 3, 140, **kw)
    formats, G, scale = (kw.get("k_format", "e4m3"), kw.get("v_format", "e4m3")), shape.n_q_heads // shape.n_kv_heads, shape.head_dim ** -0.5
    seen = []  # rows, keys and values of a block as they go into its attention, and what comes out
    qkv, rest = blocks._qkv, blocks._rest

    def _qkv(w, x, turn):
        out = qkv(w, x, turn)
        seen.append([t.cpu() for t in out])
        return out

    def _rest(w, x, out):
        seen[-1].append(out.cpu())
        return rest(w, x, out)

    monkeypatch.setattr(blocks, "_qkv", _qkv)
    monkeypatch.setattr(blocks, "_rest", _rest)
    held = [[[torch.zeros((0, shape.n_kv_heads, shape.head_dim), dtype=torch.float64) for _ in lens] for _ in range(2)] for _ in weights]

    def grown(layer, k, v, counts):
        for mine, new, f in zip(held[layer], (k, v), formats):
            for b, part in enumerate(ref.stored_rows(f, new).split(list(counts))):
                mine[b] = torch.cat([mine[b], part])

    for seed, counts in ((11, lens), (12, more)):
        seen.clear()
        blocks.prefill(to_dev(synth.hidden_states(sum(counts), shape, seed), shape.dtype), counts)
        for layer, (q, k, v, out) in enumerate(seen):
            grown(layer, k, v, counts)
            for b, (rows, got) in enumerate(zip(q.split(counts), out.view(q.shape).split(counts))):
                for i in range(0, rows.shape[0], 7):
                    n = held[layer][0][b].shape[0] - rows.shape[0] + i + 1
                    for h in range(shape.n_q_heads):
                        o, _, o_abs, delta = ref.attend(rows[i, h], held[layer][0][b][:, h // G], held[layer][1][b][:, h // G], list(range(n)), scale=scale)
                        # attn_prompt rounds probabilities to bf16 once
                        assert bool(((got[i, h].double() - o).abs() <= ref.out_bound(o, o_abs, delta, torch.bfloat16)).all()), (layer, b, i, h)
    for step in range(steps):
        seen.clear()
        blocks.decode_step(to_dev(synth.hidden_states(3, shape, 20 + step), shape.dtype))
        for layer, (q, k, v, out) in enumerate(seen):
            grown(layer, k, v, [1] * 3)
            for b in range(3):
                n = held[layer][0][b].shape[0]
                for c in range(shape.n_kv_heads):
                    keys, at = held[layer][0][b][:, c], list(range(n))
                    if kw.get("read_blocks"):
                        size = kw["block_keys"]
                        chosen = ref.select(q[b, c * G:(c + 1) * G], *ref.bounds(keys, size), n, size, kw["read_blocks"], kw["sink"], kw["recent"])
                        at = [j for i in chosen if i >= 0 for j in range(i * size, min(n, (i + 1) * size))]
                    for h in range(c * G, (c + 1) * G):
                        o, _, o_abs, delta = ref.attend(q[b, h], keys, held[layer][1][b][:, c], at, scale=scale)
                        assert bool(((out[b].view(q.shape[1:])[h].double() - o).abs() <= bound(o, o_abs, delta)).all()), (layer, b, h)
    assert blocks.held == blocks.lens.tolist() == [a + m + steps for a, m in zip(lens, more)]
