"""Blocks over requests behind a shared text (paper_2511_14450_amd.shared): with room for all keys what a stage gives, with less what
the formulas give over the keys that stay."""
import dataclasses

import pytest
import torch

import paper_2511_14450_amd as hyp
from tests import attn_reference as ref
from tests.helpers import make_gpu_stage, to_dev
from workloads import synth

pytestmark = pytest.mark.gpu
SHAPE_BF = dataclasses.replace(synth.TINY_BF16, head_dim=128, n_q_heads=4)


def _blocks(shape, n_layers, seed, prefix, n, **kw):
    from paper_2511_14450_amd import shared
    layers = [synth.layer_weights(shape, l, seed, sigma=0.05) for l in range(n_layers)]
    stage = make_gpu_stage(shape, layers, 1, prefix.shape[0], prefix.shape[0])
    stage.prefill(prefix, [prefix.shape[0]])
    pre = shared.shared_prefix(stage, 0, n_layers)
    stage.destroy()
    dev = [{k: to_dev(v, shape.dtype) for k, v in w.items()} for w in layers]
    return layers, dev, pre, shared.SharedBlocks(shape, dev, pre, n, **kw)


# relative error in the Frobenius norm.  f32: a block is some ten sums of up to 1024 products in another order each, 2^-24 of their size a
# step, growing with the root of the length: 10 * 32 * 2^-24 = 2e-5 in each of the two blocks.  bf16: about ten roundings a block on
# either side, each 2^-9 to a value (rms below 2^-9), independent: sqrt(2 * 20) * 2^-9 = 1.3e-2.
@pytest.mark.parametrize("shape,bound", [(synth.TINY, 4e-5), (SHAPE_BF, 1.3e-2)])
def test_with_room_for_all_keys_it_is_the_stage(shape, bound):
    P, lens, steps, seed = 70, [33, 1, 64], 6, 77
    prefix = to_dev(synth.hidden_states(P, shape, seed), shape.dtype)
    own = [to_dev(synth.hidden_states(x, shape, seed + 1 + i), shape.dtype) for i, x in enumerate(lens)]
    layers, _, _, blocks = _blocks(shape, 2, seed, prefix, len(lens), budget=64, room=steps, sink=2, recent=8)
    stage = make_gpu_stage(shape, layers, len(lens), P + 64 + steps, sum(lens) + P * len(lens))
    want = stage.prefill(torch.cat([t for x in own for t in (prefix, x)]), [P + x for x in lens])
    got = blocks.prefill(torch.cat(own), lens)
    ends = [sum(lens[:i + 1]) + P * (i + 1) for i in range(len(lens))]
    mine = torch.cat([want[e - x:e] for e, x in zip(ends, lens)])
    err = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())  # noqa: E731
    assert err(got, mine) <= bound
    h = torch.cat([want[e - 1:e] for e in ends])
    for _ in range(steps):
        want, got = stage.decode_step(h), blocks.decode_step(h)
        assert err(got, want) <= bound
        h = want.clone()
    stage.destroy()


def _own_qkv(blocks, w, x, pos):
    q, k, v = blocks._qkv(w, x, blocks._turn(torch.as_tensor(pos, device="cuda")))
    return q.cpu(), k.cpu(), v.cpu()


def test_with_less_room_it_attends_to_the_keys_that_stay():
    # one block in f32: its queries and keys follow from its inputs, the rest is the formulas'
    shape, P, lens, seed = synth.TINY, 20, [50, 13, 31], 5
    budget, room, sink, recent, window, steps = 16, 5, 2, 4, 8, 17
    prefix = to_dev(synth.hidden_states(P, shape, seed), shape.dtype)
    _, dev, pre, blocks = _blocks(shape, 1, seed, prefix, len(lens), budget=budget, room=room, sink=sink, recent=recent, window=window)
    w, G, scale = dev[0], shape.n_q_heads // shape.n_kv_heads, shape.head_dim ** -0.5
    pk, pv = (t.cpu() for t in pre[0])
    held = []  # [request][kv head]: position, total, key, value
    hidden = [to_dev(synth.hidden_states(x, shape, seed + 1 + i), shape.dtype) for i, x in enumerate(lens)]
    out = blocks.prefill(torch.cat(hidden), lens)

    def evict(cell, now):
        kept = ref.evict([t for _, t, _, _ in cell], len(cell), budget, sink, recent, [p for p, *_ in cell], P, now)
        return [cell[j] for j in kept if j >= 0]

    def rest(x, o):
        return blocks._rest(w, x, o.float().cuda())

    first = 0
    for x in hidden:
        q, k, v = _own_qkv(blocks, w, x, range(P, P + len(x)))
        o, cells = torch.zeros(q.shape, dtype=torch.float64), []
        for c in range(shape.n_kv_heads):
            total = torch.zeros(len(x), dtype=torch.float64)
            for h in range(c * G, (c + 1) * G):
                o[:, h], _, p, _, _ = ref.attend(q[:, h], k[:, c], v[:, c], range(len(x)), scale=scale, prefix=(pk[c], pv[c]))
                total += p[-window:].sum(0)
            cells.append(evict([(P + j, float(total[j]), k[j, c], v[j, c]) for j in range(len(x))], P + len(x)))
        held.append(cells)
        want = rest(x, o)
        assert torch.allclose(out[first:first + len(x)], want, rtol=0, atol=2e-5 * float(want.abs().max()))
        first += len(x)
    h, now, most = torch.cat([x[-1:] for x in hidden]), [P + x for x in lens], budget
    for step in range(steps):
        got = blocks.decode_step(h)
        q, k, v = _own_qkv(blocks, w, h, now)
        o = torch.zeros(q.shape, dtype=torch.float64)
        full = most == budget + room
        most = (budget if full else most) + 1
        for b, cells in enumerate(held):
            for c in range(shape.n_kv_heads):
                cell = evict(cells[c], now[b]) if full else cells[c]
                cell.append((now[b], 0.0, k[b, c], v[b, c]))
                keys, values = torch.stack([x[2] for x in cell]), torch.stack([x[3] for x in cell])
                total = torch.zeros(len(cell), dtype=torch.float64)
                for x in range(c * G, (c + 1) * G):
                    r, _, p, _, _ = ref.attend(q[b:b + 1, x], keys, values, [len(cell) - 1], scale=scale, prefix=(pk[c], pv[c]))
                    o[b, x] = r[0]
                    total += p[0]
                cells[c] = [(p, t + float(total[j]), y, z) for j, (p, t, y, z) in enumerate(cell)]
                n = len(cell)
                assert blocks.pos[0][b, c, :n].tolist() == [x[0] for x in cells[c]], (step, b, c)
            now[b] += 1
        assert blocks.lens[0].tolist() == [len(cells[0]) for cells in held] and int(blocks.lens[0].max()) <= budget + room
        want = rest(h, o)
        assert torch.allclose(got, want, rtol=0, atol=2e-5 * float(want.abs().max()))
        h = want


def test_refusals():
    from paper_2511_14450_amd import shared
    shape, prefix = synth.TINY, to_dev(synth.hidden_states(4, synth.TINY, 1), "f32")
    _, dev, pre, blocks = _blocks(shape, 1, 1, prefix, 2, budget=8, room=2, sink=1, recent=2)
    for kw in (dict(budget=0, room=1), dict(budget=4, room=0), dict(budget=4, room=1, sink=3, recent=2), dict(budget=4, room=1, sink=-1)):
        with pytest.raises(ValueError):
            shared.SharedBlocks(shape, dev, pre, 2, **kw)
    with pytest.raises(ValueError):
        shared.SharedBlocks(shape, dev, [], 2, budget=8, room=2, recent=2)
    with pytest.raises(ValueError):
        blocks.prefill(prefix, [4, 0])
    with pytest.raises(ValueError):
        blocks.decode_step(prefix)
    assert hyp.attn_last_error() is not None
