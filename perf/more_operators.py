"""A cache of keys and values in 8 or 4 bits, and single tokens that read it whole or in the blocks that a bound selects, as cases that can
be timed and compared: the operators' plain form in torch (`own` false) or the library's kernels (`own` true).

Keys of a case
  op         "write"   mx_write: new rows of every request are quantised into its cache; the blocks' bounds move along
             "read"    mx_read: what requests hold, as rows of 16 or 32 bits
             "select"  mx_select: the blocks whose keys may have the largest scores with a token
             "token"   mx_token: attention of one new row a request over its cache, or over listed blocks of it
  dtype      of rows and outputs
  q_heads, kv_heads, head_dim
  k_format, v_format   "e4m3" or "e2m1": 32 features of a key share a power of two
  held       keys each request holds when the operator is called (write: after the call).  NxL stands for N of L
  rows       write: new rows of each request, the newest of its keys
  page       own keys in pages of so many, in shuffled order; 0: one slab
  block      keys of a block (write: 0: no bounds are kept)
  keep, sink, recent   select: blocks that are chosen, and the first and newest ones that always are
  listed     token: blocks that each KV head reads; 0: all keys
  cap        token: scores are cap * tanh(score / cap); 0: not capped
  slopes     token: scores fall with the distance, each head by a slope of its own
"""
import math

import torch

own = False

PHI3 = {"q_heads": 40, "kv_heads": 10, "head_dim": 128, "dtype": "bf16"}
LLAMA3 = {"q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16"}
TINY = {"q_heads": 4, "kv_heads": 2, "head_dim": 64, "dtype": "f32"}
F32 = {"q_heads": 8, "kv_heads": 4, "head_dim": 128, "dtype": "f32"}
PLAIN_USE = {"k_format": "e4m3", "v_format": "e4m3", "rows": "", "page": 0, "block": 0, "keep": 0, "sink": 0, "recent": 0, "listed": 0, "cap": 0.0, "slopes": False}
CHATS = "23,310,64,118,7,201,395,90,33,152,260,71,180,46,129,97"
BATCH32 = "188,410,245,596,115,290,124,477,222,301,101,608,192,499,401,133,275,199,305,156,390,210,510,170,305,125,365,235,190,285,405,160"


def listed():
    def case(name, op, shape, held, **more):
        return {"name": name, "op": op, **shape, **PLAIN_USE, "held": held, **more}

    return [
        # three requests of a narrow float32 block get a token: launches are all there is
        case("write_tiny_f32", "write", TINY, "81,18,64", rows="3x1", block=16),
        # the token that 32 requests get in a step, keys in 8 bits and values in 4, in pages
        case("write_token", "write", PHI3, BATCH32, rows="32x1", page=128, block=32, v_format="e2m1"),
        # a server's chat prompts of every length
        case("write_chats", "write", PHI3, CHATS, rows=CHATS, page=128, block=64, v_format="e2m1"),
        # the next 8192 tokens of four long prompts, in 4 bits
        case("write_chunk", "write", LLAMA3, "4x16384", rows="4x8192", block=64, k_format="e2m1", v_format="e2m1"),
        # what requests hold is read back for a prompt's next chunk, or to move them to another node
        case("read_pages", "read", LLAMA3, "8192,6007,8192,7777", page=128),
        # float32 requests of unequal length out of 4 bits
        case("read_f32", "read", F32, "200,131,77,512", k_format="e2m1", v_format="e2m1"),
        # a few short float32 requests: latency
        case("select_tiny_f32", "select", TINY, "280,117,64", block=16, keep=6, sink=1, recent=2),
        # eight contexts of up to 131072 tokens in blocks of 64, of which 128 are read
        case("select_long", "select", LLAMA3, "131072,90001,131072,77777,120000,131072,50021,101010", block=64, keep=128, sink=1, recent=2, page=128),
        # a few short float32 requests generating: latency
        case("token_tiny_f32", "token", TINY, "80,17,64"),
        # 32 requests generating, keys in 8 bits and values in 4
        case("token_batch", "token", PHI3, BATCH32, v_format="e2m1"),
        # the largest: eight long contexts in pages, capped scores that fall with the distance
        case("token_long", "token", LLAMA3, "8x32768", cap=50.0, slopes=True, page=128),
        # sixteen long contexts in 4 bits, of which 64 blocks of 64 keys are read
        case("token_listed", "token", LLAMA3, "32768,30001,32768,9999,20480,32768,32767,15000,32768,30001,32768,9999,20480,32768,32767,15000",
             k_format="e2m1", v_format="e2m1", block=64, listed=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("write", "write", "read", "select", "token", "token", "token"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if dtype == "bf16":
        nq, nkv, d = rng.choice(((40, 10, 128), (32, 8, 128), (40, 10, 128), (32, 8, 128), (8, 2, 128), (16, 4, 64), (12, 4, 80), (6, 2, 96), (10, 2, 64), (8, 8, 128), (24, 1, 128)))
    else:
        nq, nkv, d = rng.choice(((4, 2, 64), (8, 4, 128), (6, 2, 96), (10, 2, 64)))
    formats = (("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e2m1"))
    case = {"op": op, "dtype": dtype, "q_heads": nq, "kv_heads": nkv, "head_dim": d, **PLAIN_USE}
    case["k_format"], case["v_format"] = rng.choice(formats)
    case["page"] = rng.choice((0, 0, 16, 128, 256))
    n = rng.choice((1, 2, 3, 4, 8, 16, 32))
    if op == "write":
        case["block"] = rng.choice((0, 16, 64, 128))
        top = min(8192, (28000 if dtype == "bf16" else 8000) // n)
    elif op == "read":
        top = min(8192, (28000 if dtype == "bf16" else 8000) // n)
    elif op == "select":
        case["block"] = rng.choice((16, 32, 64, 128))
        top = min(131072, 10000 * case["block"] // n)
    else:
        case["cap"], case["slopes"] = rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.3
        top = min(32768, (200000 if dtype == "bf16" else 50000) // n)
    mean = _log(rng, 1 if op == "token" else 5, max(5, int(top / 1.6)))
    lens = [mean] * n if rng.random() < 0.3 else [min(top, max(1, int(mean * rng.uniform(0.3, 1.6)))) for _ in range(n)]
    case["held"] = ",".join(str(v) for v in lens)
    if case["page"] and case["block"] > case["page"]:
        case["block"] = case["page"]
    if op == "write":
        if rng.random() < 0.3:
            rows = [1] * n
        else:
            rows = [max(1, int(v * rng.uniform(0.2, 1.0))) for v in lens] if rng.random() < 0.5 else lens
        case["rows"] = ",".join(str(v) for v in rows)
    elif op == "select":
        blocks = -(-max(lens) // case["block"])
        case["keep"] = max(1, min(int(blocks * rng.uniform(0.02, 1.2)), 4096))
        case["sink"], case["recent"] = rng.choice((0, case["keep"] // 8)), rng.choice((0, case["keep"] // 4))
    elif op == "token" and rng.random() < 0.4:
        case["block"] = rng.choice([b for b in (16, 32, 64, 128) if not case["page"] or b <= case["page"]])
        case["listed"] = max(1, int(-(-max(lens) // case["block"]) * rng.uniform(0.05, 1.0)))
    return case


# ---------------------------------------------------------------- the numbers of the cache
MOST = {"e4m3": 448.0, "e2m1": 6.0}                         # largest number of a format
TOP = {"e4m3": 8, "e2m1": 2}                                # its power of two
FRACTION = {"e4m3": 0x600000, "e2m1": 0x400000}             # its fraction, as bits of a float
SCALES = {"e4m3": (-117, 119), "e2m1": (-125, 125)}         # powers by which all numbers stay normal floats
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _width(fmt, d):
    return -(-d // 32) * (32 if fmt == "e4m3" else 16)


def _pow2(s):
    return ((127 + s) << 23).to(torch.int32).view(torch.float32)


def _quantised(x, fmt):
    """(values in 32 bits [..., d], codes [..., width], scales [..., groups]) of x [..., d]"""
    d, lo, hi = x.shape[-1], *SCALES[fmt]
    y = torch.nn.functional.pad(x.float(), (0, -d % 32)).unflatten(-1, (-1, 32))
    bits = y.abs().amax(-1, keepdim=True).view(torch.int32)
    power = ((bits >> 23) - 127 - TOP[fmt] + ((bits & 0x7FFFFF) > FRACTION[fmt]).int()).clamp(lo, hi)
    y = (y * _pow2(-power)).clamp(-MOST[fmt], MOST[fmt])
    if fmt == "e4m3":
        code = y.to(torch.float8_e4m3fn)
        value, code = code.float(), code.view(torch.uint8)
    else:
        a = y.abs()
        a = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2))
        index = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
        value, index = torch.where(torch.signbit(y), -a, a), index | (torch.signbit(y).to(torch.uint8) << 3)
        code = index[..., 0::2] | (index[..., 1::2] << 4)
    return (value * _pow2(power)).flatten(-2)[..., :d], code.flatten(-2), (power[..., 0] + 127).to(torch.uint8)


def _values(code, scale, fmt, d):
    """The numbers that codes [..., width] under scales [..., groups] stand for, in 32 bits [..., d]"""
    if fmt == "e4m3":
        y = code.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
        y = table[torch.stack((code & 15, code >> 4), -1).int()].flatten(-2)
    y = y.unflatten(-1, (-1, 32)) * (scale.int() << 23).view(torch.float32)[..., None]
    return y.flatten(-2)[..., :d]


# ---------------------------------------------------------------- inputs
def _counts(text):
    out = []
    for part in text.split(","):
        n, _, length = part.rpartition("x")
        out += [int(length)] * int(n or 1)
    return out


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _slopes(case):
    heads = case["q_heads"]
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _draw_inputs(case, seed):
    """The tensors of a case as the formulas see them: caches as slabs, codes [n, kv heads, room, width], scales [n, kv heads, groups, room],
    bounds [n, kv heads, blocks, d]."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 8191 + 29)
    held, dt, op = _counts(case["held"]), _dtype(case), case["op"]
    n, nq, nkv, d = len(held), case["q_heads"], case["kv_heads"], case["head_dim"]
    unit = max(case["page"], case["block"], 16)
    room = -(-max(held) // unit) * unit

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    # a few features of the keys are larger than the others, in each head its own
    loud = normal(1, nkv, 1, d).mul_(0.7).exp_()
    x = {"room": room}
    if op in ("read", "token"):
        for name, fmt in (("k", case["k_format"]), ("v", case["v_format"])):
            codes = torch.empty((n, nkv, room, _width(fmt, d)), dtype=torch.uint8, device="cuda")
            scales = torch.empty((n, nkv, -(-d // 32), room), dtype=torch.uint8, device="cuda")
            for b in range(n):
                y = normal(1, nkv, room, d)
                _, codes[b], s = (t[0] if t.dim() == 4 else t for t in _quantised(y.mul_(loud) if name == "k" else y, fmt))
                scales[b] = s.transpose(1, 2)
            x[name], x[name + "s"] = codes, scales
    if op == "write":
        rows = sum(_counts(case["rows"]))
        x["new_k"], x["new_v"] = normal(rows, nkv, d).mul_(loud[0, :, 0]).to(dt), normal(rows, nkv, d).to(dt)
        for name, fmt in (("k", case["k_format"]), ("v", case["v_format"])):  # what was cached before is of no account, but for the bounds
            x[name] = torch.zeros((n, nkv, room, _width(fmt, d)), dtype=torch.uint8, device="cuda")
            x[name + "s"] = torch.full((n, nkv, -(-d // 32), room), 127, dtype=torch.uint8, device="cuda")
    if case["block"] and op in ("write", "select"):
        # the keys of a block lie around a place of its own
        middle = normal(n, nkv, room // case["block"], d)
        wide = normal(n, nkv, room // case["block"], d).abs_().add_(0.5)
        x["lo"], x["hi"] = ((middle + f * wide).mul_(loud).to(torch.bfloat16) for f in (-1.0, 1.0))
    if op in ("select", "token"):
        x["q"] = normal(n, nq, d).mul_(1.5).to(dt)
    if case["listed"]:
        # ascending blocks of each KV head out of those that its request holds, -1 behind the last
        count = (_ints(held) + case["block"] - 1) // case["block"]
        mark = torch.rand((n, nkv, room // case["block"]), generator=gen, device="cuda")
        at = torch.arange(mark.shape[2], device="cuda")
        there = at < count[:, None, None]
        best = torch.where(there, mark, -1.0).topk(case["listed"], dim=-1).indices
        best = torch.where(best < count[:, None, None], best, mark.shape[2]).sort(-1).values
        x["blocks"] = torch.where(best < mark.shape[2], best, -1).int()
    if case["page"]:
        pages = room // case["page"]
        x["table"] = torch.randperm(n * pages, generator=gen, device="cuda").reshape(n, pages).to(torch.int32)
    return x


def _paged(slab, table, axis):
    """the slab's keys or blocks, along `axis`, in a pool of pages"""
    n, pages = table.shape
    parts = slab.unflatten(axis, (pages, -1)).movedim(axis, 1).flatten(0, 1)
    pool = torch.empty_like(parts)
    pool[table.reshape(-1).long()] = parts
    return pool


def prepare(case, seed):
    x, held = _draw_inputs(case, seed), _counts(case["held"])
    n, nkv, d, dt = len(held), case["kv_heads"], case["head_dim"], _dtype(case)
    s = {"case": case, "most": max(held), "held": _ints(held), "scale": 1.0 / math.sqrt(d), **x}
    if case["page"]:
        for name, axis in (("k", 2), ("v", 2), ("ks", 3), ("vs", 3), ("lo", 2), ("hi", 2)):
            if name in x:
                s[name] = _paged(x[name], x["table"], axis)
    if case["op"] == "write":
        rows = _counts(case["rows"])
        s["q_start"] = _ints([sum(rows[:i]) for i in range(n + 1)])
        s["k_out"], s["v_out"] = torch.empty_like(s["new_k"]), torch.empty_like(s["new_v"])
    if case["op"] == "read":
        s["out_k"], s["out_v"] = (torch.zeros((n, nkv, max(held), d), dtype=dt, device="cuda") for _ in range(2))
    if case["op"] == "select":  # selecting looks at bounds alone: the least that a cache has for keys
        pages, size = (n * x["table"].shape[1], case["page"]) if case["page"] else (n, x["room"])
        for name, fmt in (("k", case["k_format"]), ("v", case["v_format"])):
            s[name] = torch.zeros((1, 1, 1, _width(fmt, d)), dtype=torch.uint8, device="cuda").expand(pages, nkv, size, -1)
            s[name + "s"] = torch.zeros((1, 1, 1, size), dtype=torch.uint8, device="cuda").expand(pages, nkv, -(-d // 32), -1)
    if case["slopes"]:
        s["slopes"] = torch.tensor(_slopes(case), dtype=torch.float32, device="cuda")
    if own:  # the descriptions of the tensors above that a program keeps with them: no values, nothing computed
        import paper_2511_14450_amd as hyp
        s["cache"] = hyp.MxCache(s["k"], s["v"], s["ks"], s["vs"], s["held"], d, page_table=s.get("table"), most=s["most"], lo=s.get("lo"),
                                 hi=s.get("hi"), block_keys=case["block"])
        s["rule"] = hyp.AttnRule(s["scale"], cap=case["cap"], slopes=s.get("slopes"))
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"write": _write, "read": _read, "select": _select, "token": _token}[op](s)


def _written(s):
    out = {"k": s["k_out"], "v": s["v_out"], "codes": [s["k"], s["ks"], s["v"], s["vs"]]}
    return {**out, "lo": s["lo"], "hi": s["hi"]} if "lo" in s else out


def _run_own(s, op):
    import paper_2511_14450_amd as hyp
    case = s["case"]
    if op == "write":
        hyp.mx_write(s["cache"], s["new_k"], s["new_v"], q_start=s["q_start"], k_out=s["k_out"], v_out=s["v_out"])
        return _written(s)
    if op == "read":
        hyp.mx_read(s["cache"], s["out_k"], s["out_v"])
        return {"k": s["out_k"], "v": s["out_v"]}
    if op == "select":
        return {"blocks": hyp.mx_select(s["cache"], s["q"], case["keep"], sink=case["sink"], recent=case["recent"])}
    out, lse = hyp.mx_token(s["cache"], s["rule"], s["q"], blocks=s.get("blocks"))
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- the plain form
def _place(s, b, j, per):
    """page (or request) and place in it of key or block j of request b, `per` to a page"""
    if not s["case"]["page"]:
        return b, j
    return s["table"][b, j // per].long(), j % per


def _write(s):
    case = s["case"]
    n, d, rows = s["held"].shape[0], case["head_dim"], s["new_k"].shape[0]
    start = s["q_start"].long()
    b = torch.repeat_interleave(torch.arange(n, device=start.device), start.diff(), output_size=rows)
    first = s["held"].long() - start.diff()                       # slot of each request's first new row
    slot = first[b] + torch.arange(rows, device=start.device) - start[b]
    page, at = _place(s, b, slot, case["page"])
    stored, codes, scales = _quantised(s["new_k"], case["k_format"])
    s["k"][page, :, at], s["ks"][page, :, :, at] = codes, scales
    s["k_out"].copy_(stored)
    values, codes, scales = _quantised(s["new_v"], case["v_format"])
    s["v"][page, :, at], s["vs"][page, :, :, at] = codes, scales
    s["v_out"].copy_(values)
    if "lo" in s:
        size = case["block"]
        page, at = _place(s, b, slot // size, case["page"] // size)
        fresh = (slot // size * size >= first[b])[:, None, None]  # the block's first key is among the rows
        low, high = s["lo"].float(), s["hi"].float()
        low[page, :, at] = torch.where(fresh, math.inf, low[page, :, at])
        high[page, :, at] = torch.where(fresh, -math.inf, high[page, :, at])
        index = (page * low.shape[2] + at)[:, None, None].expand(rows, case["kv_heads"], d)
        by_block = (low.shape[0], low.shape[2], low.shape[1], d)
        low = low.transpose(1, 2).flatten(0, 1).scatter_reduce(0, index, stored, "amin")
        high = high.transpose(1, 2).flatten(0, 1).scatter_reduce(0, index, stored, "amax")
        s["lo"].copy_(low.view(by_block).transpose(1, 2))
        s["hi"].copy_(high.view(by_block).transpose(1, 2))
    return _written(s)


def _keys(s, name, j):
    """values of keys j [n, kv heads, keys] in 32 bits [n, kv heads, keys, d]"""
    case = s["case"]
    n, nkv, _ = j.shape
    b, head = torch.arange(n, device=j.device)[:, None, None], torch.arange(nkv, device=j.device)[:, None]
    page, at = _place(s, b, j, case["page"])
    return _values(s[name][page, head, at], s[name + "s"][page, head, :, at], case[name + "_format"], case["head_dim"])


def _read(s):
    n, nkv, most, _ = s["out_k"].shape
    j = torch.arange(most, device=s["held"].device)
    there = (j < s["held"][:, None])[:, None, :, None]
    j = j.expand(n, nkv, most)
    s["out_k"].copy_(torch.where(there, _keys(s, "k", j), s["out_k"].float()))
    s["out_v"].copy_(torch.where(there, _keys(s, "v", j), s["out_v"].float()))
    return {"k": s["out_k"], "v": s["out_v"]}


def _select(s):
    case = s["case"]
    size, keep, nkv, d = case["block"], case["keep"], case["kv_heads"], case["head_dim"]
    n = s["held"].shape[0]
    most = -(-s["most"] // size)
    b, head, at = torch.arange(n, device="cuda")[:, None, None], torch.arange(nkv, device="cuda")[:, None], torch.arange(most, device="cuda")
    page, place = _place(s, b, at, case["page"] // size)
    q = s["q"].double().view(n, nkv, -1, d)  # in 64 bits: which block is chosen may hang on the last bit of a score
    score = q.clamp(min=0) @ s["hi"][page, head, place].double().transpose(2, 3).contiguous()
    score += q.clamp(max=0) @ s["lo"][page, head, place].double().transpose(2, 3).contiguous()
    score = score.amax(2)                                         # of the heads of a group
    count = (s["held"][:, None, None] + size - 1) // size
    score = torch.where((at < case["sink"]) | (at >= count - case["recent"]), math.inf, score)
    score = torch.where(at < count, score, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.nn.functional.pad(torch.where(best < count, best, most), (0, max(0, keep - most)), value=most).sort(-1).values
    return {"blocks": torch.where(best < most, best, -1).int()}


def _token(s):
    case = s["case"]
    n, nq, d = s["q"].shape
    nkv, size, held = case["kv_heads"], case["block"], s["held"][:, None, None]
    if case["listed"]:
        j = (s["blocks"].long()[..., None] * size + torch.arange(size, device=held.device)).flatten(2)
        there = (j >= 0) & (j < held)
        j = torch.where(there, j, 0)
    else:
        j = torch.arange(s["most"], device=held.device).expand(n, nkv, -1)
        there = j < held
    x = s["q"].float().view(n, nkv, -1, d) @ _keys(s, "k", j).transpose(2, 3).mul_(s["scale"])
    if case["cap"]:
        x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
    if case["slopes"]:
        x -= s["slopes"].view(1, nkv, -1, 1) * (held - 1 - j).float()[:, :, None]
    x = x.masked_fill_(~there[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = p @ _keys(s, "v", j)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return {"out": out.view(n, nq, d).to(s["q"].dtype), "lse": (total.log() + top).view(n, nq)}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    held, es, nq, nkv, d = _counts(case["held"]), 2 if case["dtype"] == "bf16" else 4, case["q_heads"], case["kv_heads"], case["head_dim"]
    key = _width(case["k_format"], d) + _width(case["v_format"], d) + 2 * -(-d // 32)  # bytes of a cached key and its value
    bounds = 4 * d                                                                     # of a block
    if case["op"] == "write":
        rows = _counts(case["rows"])
        moved = 0
        if case["block"]:
            for n, h in zip(rows, held):
                inside = (h - n) % case["block"]  # a block that was begun before is read and written
                moved += -(-(n + inside) // case["block"]) + (1 if inside else 0)
        return {"bytes": nkv * (sum(rows) * (4 * d * es + key) + moved * bounds), "flops": 0}
    if case["op"] == "read":
        return {"bytes": nkv * sum(held) * (key + 2 * d * es), "flops": 0}
    n = len(held)
    if case["op"] == "select":
        blocks = sum(-(-h // case["block"]) for h in held)
        return {"bytes": nkv * (blocks * bounds + 4 * n * case["keep"]) + n * nq * d * es, "flops": 2 * d * nq * blocks}
    if case["listed"]:
        keys = sum(min(h, case["listed"] * case["block"]) for h in held)
    else:
        keys = sum(held)
    return {"bytes": nkv * keys * key + n * nq * (2 * d * es + 4) + 4 * n * nkv * case["listed"], "flops": 4 * d * nq * keys}


# ---------------------------------------------------------------- the definition in 64 bits
def _numbers(fmt):
    """What each code stands for, by the format's bits"""
    if fmt == "e2m1":
        return [(-1.0 if c & 8 else 1.0) * ((c & 1) * 0.5 if (c >> 1) & 3 == 0 else (1 + (c & 1) / 2) * 2.0 ** (((c >> 1) & 3) - 1)) for c in range(16)]
    return [math.nan if c & 127 == 127 else (-1.0 if c & 128 else 1.0) * ((c & 7) / 512 if (c >> 3) & 15 == 0 else (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7))
            for c in range(256)]


def _exact_pow2(p):
    """2^p in 64 bits, by its bits: pow() may be off in the last one, on which a tie hangs"""
    return ((1023 + p.long()) << 52).view(torch.float64)


def _exact_keys(code, scale, fmt, d):
    """codes [keys, width] and scales [groups, keys] as numbers of 64 bits [keys, d]"""
    if fmt == "e2m1":
        code = torch.stack((code % 16, code // 16), -1).reshape(code.shape[0], -1)
    y = torch.tensor(_numbers(fmt), dtype=torch.float64, device=code.device)[code.long()]
    return (y * _exact_pow2(scale.int() - 127).t().repeat_interleave(32, 1))[:, :d]


def _exact_stored(x, fmt):
    """x [rows, heads, d] in 64 bits as the format holds it: the least power of two under which no number of 32 passes the format's largest,
    then the nearest number, ties to the even code"""
    d = x.shape[-1]
    top, least, low = (448.0, -6, -117) if fmt == "e4m3" else (6.0, 0, -125)
    high = 119 if fmt == "e4m3" else 125
    digits = 3 if fmt == "e4m3" else 1
    y = torch.nn.functional.pad(x.double(), (0, -d % 32)).unflatten(-1, (-1, 32))
    ratio, power = torch.frexp(y.abs().amax(-1, keepdim=True) / top)  # ratio * 2^power, ratio in [1/2, 1)
    power = _exact_pow2(torch.where(ratio == 0.5, power - 1, power).clamp(low, high))
    y = (y / power).clamp(-top, top)
    _, exponent = torch.frexp(y)
    step = _exact_pow2((exponent - 1).clamp(min=least) - digits)
    return ((y / step).round() * step * power).flatten(-2)[..., :d]


def exact(case, seed):
    if case["op"] == "select":
        return None
    x, held = _draw_inputs(case, seed), _counts(case["held"])
    nkv, d, size = case["kv_heads"], case["head_dim"], case["block"]
    if case["op"] == "write":
        k, v = _exact_stored(x["new_k"], case["k_format"]), _exact_stored(x["new_v"], case["v_format"])
        out = {"k": k, "v": v, "codes": None}
        if size:
            lo, hi, first = x["lo"].double(), x["hi"].double(), 0
            for b, (n, h) in enumerate(zip(_counts(case["rows"]), held)):
                for block in range((h - n) // size, -(-h // size)):
                    mine = k[first + max(0, block * size - (h - n)):first + min(n, (block + 1) * size - (h - n))]
                    low, high = mine.amin(0), mine.amax(0)
                    begun = block * size < h - n
                    lo[b, :, block] = torch.minimum(low, lo[b, :, block]) if begun else low
                    hi[b, :, block] = torch.maximum(high, hi[b, :, block]) if begun else high
                first += n
            out["lo"], out["hi"] = (_paged(t, x["table"], 2) for t in (lo, hi)) if case["page"] else (lo, hi)
        return out
    if case["op"] == "read":
        k, v = (torch.zeros((len(held), nkv, max(held), d), dtype=torch.float64, device="cuda") for _ in range(2))
        for b, h in enumerate(held):
            for c in range(nkv):
                k[b, c, :h] = _exact_keys(x["k"][b, c, :h], x["ks"][b, c, :, :h], case["k_format"], d)
                v[b, c, :h] = _exact_keys(x["v"][b, c, :h], x["vs"][b, c, :, :h], case["v_format"], d)
        return {"k": k, "v": v}
    group = case["q_heads"] // nkv
    slopes = torch.tensor(_slopes(case), dtype=torch.float64, device="cuda") if case["slopes"] else None
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    for b, h in enumerate(held):
        for c in range(nkv):
            j = torch.arange(h, device="cuda")
            if case["listed"]:
                mine = torch.zeros(x["room"] // size, dtype=torch.bool, device="cuda")
                mine[x["blocks"][b, c][x["blocks"][b, c] >= 0].long()] = True
                j = j[mine[j // size]]
            k = _exact_keys(x["k"][b, c, j], x["ks"][b, c][:, j], case["k_format"], d)
            v = _exact_keys(x["v"][b, c, j], x["vs"][b, c][:, j], case["v_format"], d)
            z = x["q"][b, c * group:(c + 1) * group].double() @ k.t() / math.sqrt(d)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if slopes is not None:
                z = z - slopes[c * group:(c + 1) * group, None] * (h - 1 - j)
            lse[b, c * group:(c + 1) * group] = torch.logsumexp(z, -1)
            out[b, c * group:(c + 1) * group] = torch.softmax(z, -1) @ v
    return {"out": out, "lse": lse}
