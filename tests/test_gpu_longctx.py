"""Blocks over long contexts in 8 and 4 bits (paper_2511_14450_amd.longctx): what the formulas give over the numbers that the formats hold."""
import pytest
import torch

from tests import attn_reference
from tests import mx_reference as ref
from tests.helpers import make_gpu_stage, to_dev
from workloads import synth

pytestmark = pytest.mark.gpu


def make(shape, n_layers, n, seed=3, **kw):
    from paper_2511_14450_amd import longctx
    layers = [synth.layer_weights(shape, l, seed, sigma=0.05) for l in range(n_layers)]
    dev = [{k: to_dev(v, shape.dtype) for k, v in w.items()} for w in layers]
    return layers, dev, longctx.LongBlocks(shape, dev, n, **kw)


def rows(shape, n, seed):
    return to_dev(synth.hidden_states(n, shape, seed), shape.dtype)


@pytest.mark.parametrize("kw", [dict(), dict(k_format="e4m3", v_format="e2m1", page_keys=32), dict(k_format="e2m1", v_format="e2m1", read_blocks=4, block_keys=16, sink=1, recent=2),
                                dict(read_blocks=3, block_keys=16, sink=0, recent=1, page_keys=16)])
def test_one_block_against_the_formulas(kw):
    # one block in f32: queries, keys and values follow from its inputs, the rest is the formulas' over the numbers that are held
    shape, lens, more, steps = synth.TINY, [60, 5, 97], [30, 0, 11], 4
    formats = kw.get("k_format", "e4m3"), kw.get("v_format", "e4m3")
    _, dev, blocks = make(shape, 1, 3, most=140, **kw)
    w, G, scale = dev[0], shape.n_q_heads // shape.n_kv_heads, shape.head_dim ** -0.5
    held = [[torch.zeros((0, shape.n_kv_heads, shape.head_dim)) for _ in lens] for _ in range(2)]

    def grow(x, counts):
        pos = torch.cat([torch.arange(h.shape[0], h.shape[0] + c) for h, c in zip(held[0], counts)]).cuda()
        q, k, v = (t.cpu() for t in blocks._qkv(w, x, blocks._turn(pos)))
        for mine, new, f in zip(held, (k, v), formats):
            for b, part in enumerate(ref.stored_rows(f, new).split(list(counts))):
                mine[b] = torch.cat([mine[b].double(), part])
        return q.split(list(counts))

    def same(got, x, out):
        want = blocks._rest(w, x, out.float().cuda())
        assert torch.allclose(got, want, rtol=0, atol=2e-5 * float(want.abs().max()))

    for seed, counts in ((11, lens), (12, more)):
        x = rows(shape, sum(counts), seed)
        got, outs = blocks.prefill(x, counts), []
        for b, q in enumerate(grow(x, counts)):
            o, n = torch.zeros(q.shape, dtype=torch.float64), held[0][b].shape[0]
            for h in range(shape.n_q_heads):
                o[:, h] = attn_reference.attend(q[:, h], held[0][b][:, h // G], held[1][b][:, h // G], range(n - q.shape[0], n), scale=scale)[0]
            outs.append(o)
        same(got, x, torch.cat(outs))
    for step in range(steps):
        x = rows(shape, 3, 20 + step)
        got, outs = blocks.decode_step(x), []
        for b, q in enumerate(grow(x, [1] * 3)):
            o, n = torch.zeros(q.shape[1:], dtype=torch.float64), held[0][b].shape[0]
            for c in range(shape.n_kv_heads):
                at = list(range(n))
                if kw.get("read_blocks"):
                    size = kw["block_keys"]
                    chosen = ref.select(q[0, c * G:(c + 1) * G], *ref.bounds(held[0][b][:, c], size), n, size, kw["read_blocks"], kw["sink"], kw["recent"])
                    at = [j for i in chosen if i >= 0 for j in range(i * size, min(n, (i + 1) * size))]
                for h in range(c * G, (c + 1) * G):
                    o[h] = ref.attend(q[0, h], held[0][b][:, c], held[1][b][:, c], at, scale=scale)[0]
            outs.append(o[None])
        same(got, x, torch.cat(outs))
    assert blocks.lens.tolist() == blocks.held == [a + m + steps for a, m in zip(lens, more)]


# the same numbers, summed in calls of other sizes: twenty sums of up to 1024 products a block, each off by at most 2^-24 of its size a step, growing
# with the root of the length: 20 * 32 * 2^-24 = 4e-5 a block, where no key falls on another side of a rounding (no seed of these does)
def test_chunks_give_what_a_whole_prompt_gives():
    shape, lens = synth.TINY, [64, 9, 40]
    _, _, whole = make(shape, 2, 3, most=80)
    _, _, parts = make(shape, 2, 3, most=80, page_keys=16)
    x = [rows(shape, n, 30 + i) for i, n in enumerate(lens)]
    want = whole.prefill(torch.cat(x), lens)
    cuts, got = [[20, 9, 0], [44, 0, 39], [0, 0, 1]], [[], [], []]
    at = [0, 0, 0]
    for cut in cuts:
        out = parts.prefill(torch.cat([t[a:a + c] for t, a, c in zip(x, at, cut)]), cut).split(cut)
        for b in range(3):
            got[b].append(out[b])
            at[b] += cut[b]
    got = torch.cat([t for part in got for t in part])
    assert float((got - want).norm() / want.norm()) <= 8e-5
    y = rows(shape, 3, 40)
    a, b = whole.decode_step(y), parts.decode_step(y)
    assert float((a - b).norm() / a.norm()) <= 8e-5
    whole.reset()
    again = whole.prefill(torch.cat(x), lens)
    assert torch.equal(again, want)


def test_a_stage_hands_its_contexts_over():
    shape, lens = synth.TINY, [33, 1, 64]
    layers, _, blocks = make(shape, 2, 3, most=70, v_format="e2m1")
    stage = make_gpu_stage(shape, layers, 3, 80, sum(lens))
    out = stage.prefill(rows(shape, sum(lens), 50), lens)
    blocks.adopt(stage, 0, 2)
    assert blocks.held == lens and blocks.lens.tolist() == lens
    import paper_2511_14450_amd as hyp
    for l, cache in enumerate(blocks.caches):
        k, v = (torch.zeros((3, shape.n_kv_heads, 64, shape.head_dim), device="cuda") for _ in range(2))
        hyp.mx_read(cache, k, v)
        for b, n in enumerate(lens):
            for got, fmt, mine in zip((k, v), ("e4m3", "e2m1"), stage.export_kv(l, b)):
                want = ref.stored_rows(fmt, mine.view(n, shape.n_kv_heads, shape.head_dim).cpu())
                assert torch.equal(got[b, :, :n].double().cpu(), want.transpose(0, 1))
    # a step of either: they differ by what 8 and 4 bits leave out, which is not small
    ends = torch.tensor([sum(lens[:i + 1]) - 1 for i in range(3)], device="cuda")
    a, b = stage.decode_step(out[ends]), blocks.decode_step(out[ends])
    assert bool(torch.isfinite(b).all()) and a.shape == b.shape
    stage.destroy()


def test_refusals():
    from paper_2511_14450_amd import longctx
    shape = synth.TINY
    _, dev, blocks = make(shape, 1, 2, most=20)
    for kw in (dict(read_blocks=-1), dict(read_blocks=3, sink=2, recent=2), dict(sink=-1), dict(k_format="int8"), dict(page_keys=24)):
        with pytest.raises((ValueError, RuntimeError)):
            longctx.LongBlocks(shape, dev, 2, 20, **kw).prefill(rows(shape, 2, 1), [1, 1])
    for n, m in ((0, 20), (2, 0)):
        with pytest.raises(ValueError):
            longctx.LongBlocks(shape, dev, n, m)
    for counts in ([3], [4, -1], [2, 2], [3, 0, 0]):
        with pytest.raises(ValueError):
            blocks.prefill(rows(shape, 3, 1), counts)
    blocks.prefill(rows(shape, 23, 1), [20, 3])
    with pytest.raises(ValueError, match="more than 20"):
        blocks.decode_step(rows(shape, 2, 1))
    with pytest.raises(ValueError):
        blocks.decode_step(rows(shape, 3, 1))
    assert blocks.lens.tolist() == blocks.held == [20, 3]
