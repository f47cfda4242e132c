"""Attention over a shared prefix and a request's own cache, and the cache kept within a budget, as cases that can be timed
and compared: the operators' plain form in torch (`own` false) or the library's kernels (`own` true).

Keys of a case
  op         "prompt"    attn_prompt: the new rows of a batch of requests, after what each already has cached
             "received"  attn_received: the weight that the keys got from the prompt's last rows
             "token"     attn_token: one new row a request
             "evict"     attn_evict: the keys with the largest totals move to a cache of `keep` slots
  dtype, q_heads, kv_heads, head_dim
  lens       prompt / received: new rows of each request; token / evict: keys each request holds.  NxL stands for N of L
  past       prompt / received: keys each request has cached before the new rows
  prefix     keys that all requests share
  cap        scores are cap * tanh(score / cap); 0: not capped
  slopes     scores fall with the distance, each head by a slope of its own
  docs       own keys belong to so many documents that do not see one another, and a last part that sees all; 0: no documents
  see_all    own keys that all rows of their request see
  page       own keys in pages of so many, in shuffled order; 0: one slab
  last       received: rows that count, from the end; 0: all
  totals     token: the weight that own keys get is added to a running total
  keep, sink, recent   evict: slots, and the first and newest positions that always stay
"""
import math

import torch

own = False

PHI3 = {"q_heads": 40, "kv_heads": 10, "head_dim": 128, "dtype": "bf16"}
LLAMA3 = {"q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16"}
TINY = {"q_heads": 4, "kv_heads": 2, "head_dim": 64, "dtype": "f32"}
F32 = {"q_heads": 8, "kv_heads": 4, "head_dim": 128, "dtype": "f32"}
PLAIN_USE = {"past": 0, "prefix": 0, "cap": 0.0, "slopes": False, "docs": 0, "see_all": 0, "page": 0, "last": 0, "totals": False,
             "keep": 0, "sink": 0, "recent": 0}
CHATS = "23,310,64,118,7,201,395,90,33,152,260,71,180,46,129,97"
BATCH32 = "188,410,245,596,115,290,124,477,222,301,101,608,192,499,401,133,275,199,305,156,390,210,510,170,305,125,365,235,190,285,405,160"


def listed():
    def case(name, op, shape, lens, **more):
        return {"name": name, "op": op, **shape, **PLAIN_USE, "lens": lens, **more}

    return [
        # the smallest prompt of a narrow float32 block: launches are all there is
        case("prompt_tiny_f32", "prompt", TINY, "64"),
        # float32 requests of unequal length whose first tokens are read in both directions, distance in the scores
        case("prompt_f32", "prompt", F32, "200,131,77,512", slopes=True, see_all=50),
        # a server's chat prompts of every length behind one system prompt
        case("prompt_chats", "prompt", PHI3, CHATS, prefix=1024),
        # retrieved documents that must not see one another, then the question; pages as a server hands them out
        case("prompt_documents", "prompt", LLAMA3, "4096,2890,3777,1515", prefix=512, docs=5, page=128),
        # the largest: four long prompts, scores capped
        case("prompt_long", "prompt", PHI3, "4x8192", cap=50.0),
        # which keys of a batch of prompts matter, by their last rows
        case("received_window", "received", LLAMA3, "2048,1900,777,2048,1333,512,2047,1601", last=32, prefix=256),
        # the same by all rows of one long document
        case("received_document", "received", PHI3, "6007", cap=30.0),
        # a few short float32 requests generating: latency
        case("token_tiny_f32", "token", TINY, "80,17,64", prefix=64, totals=True),
        # 32 requests generating behind a long shared prompt, totals kept for eviction
        case("token_shared", "token", PHI3, BATCH32, prefix=8192, totals=True),
        # eight long contexts in pages, capped scores that fall with the distance
        case("token_long", "token", LLAMA3, "8x9216", cap=50.0, slopes=True, page=128),
        # a small cache over its budget
        case("evict_tiny_f32", "evict", TINY, "96,70", keep=64, sink=4, recent=16),
        # long prompts cut down to what their generation keeps
        case("evict_prompts", "evict", LLAMA3, "8192,6007,8192,7777,8192,8000,5121,8192", keep=1024, sink=4, recent=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("prompt", "prompt", "received", "token", "token", "evict"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if dtype == "bf16":
        nq, nkv, d = rng.choice(((40, 10, 128), (32, 8, 128), (40, 10, 128), (32, 8, 128), (8, 2, 128), (16, 4, 64), (12, 4, 80), (6, 2, 96), (10, 2, 64), (8, 8, 128)))
    else:
        nq, nkv, d = rng.choice(((4, 2, 64), (8, 4, 128), (6, 2, 96), (10, 2, 64)))
    case = {"op": op, "dtype": dtype, "q_heads": nq, "kv_heads": nkv, "head_dim": d, **PLAIN_USE}
    case["cap"], case["slopes"] = rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.3
    case["page"] = rng.choice((0, 0, 0, 16, 128))
    n = rng.choice((1, 2, 3, 4, 8, 16, 32))
    if op in ("prompt", "received"):
        top = min(8192, 32768 // n) if dtype == "bf16" else min(1024, 2048 // n)
        case["prefix"] = rng.choice((0, 0, _log(rng, 16, 2048 if dtype == "bf16" else 512)))
        case["past"] = rng.choice((0, 0, _log(rng, 1, 1024 if dtype == "bf16" else 256)))
        top = max(1, top - case["prefix"] // 2 - case["past"])
        if op == "prompt":
            case["docs"], case["see_all"] = rng.choice((0, 0, 2, 7)), rng.choice((0, 0, 37, 200))
        else:
            case["last"] = rng.choice((0, 8, 32, 100))
    elif op == "token":
        top = min(9216, 73728 // n) if dtype == "bf16" else min(4096, 8192 // n)
        case["prefix"], case["totals"] = rng.choice((0, _log(rng, 16, 8192 if dtype == "bf16" else 1024))), rng.random() < 0.5
    else:
        top = min(8192, 65536 // n) if dtype == "bf16" else min(4096, 16384 // n)
        case["cap"], case["slopes"] = 0.0, False
    mean = _log(rng, 1 if op == "token" else 5, max(5, int(top / 1.6)))
    if rng.random() < 0.3:
        lens = [mean] * n
    else:
        lens = [min(top, max(1, int(mean * rng.uniform(0.3, 1.6)))) for _ in range(n)]
    case["lens"] = ",".join(str(v) for v in lens)
    if op == "evict":
        case["keep"] = max(1, min(int(max(lens) * rng.uniform(0.1, 0.95)), 6144 // n))
        case["sink"], case["recent"] = min(4, case["keep"] // 8), case["keep"] // rng.choice((2, 4, 16))
    return case


# ---------------------------------------------------------------- inputs
def _lens(case):
    lens = []
    for part in case["lens"].split(","):
        n, _, length = part.rpartition("x")
        lens += [int(length)] * int(n or 1)
    return lens


def _held(case):
    """keys that each request holds when the operator is called"""
    return [n + (case["past"] if case["op"] in ("prompt", "received") else 0) for n in _lens(case)]


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _slopes(case):
    heads = case["q_heads"]
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _doc_ids(case, held):
    """ids of a request's own keys: parts of equal length, the last one an id that sees all and is seen by all"""
    part = -(-held // (case["docs"] + 1))
    return [(-1 if i // part == case["docs"] else i // part) for i in range(held)]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _draw_inputs(case, seed):
    """The tensors of a case as the formulas see them: own keys in slabs [n, kv heads, most, d], rows packed."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 8191 + 17)
    lens, held, dt = _lens(case), _held(case), _dtype(case)
    n, nq, nkv, d, most = len(lens), case["q_heads"], case["kv_heads"], case["head_dim"], max(held)

    def normal(*shape, sigma=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(sigma).to(dt)

    x = {"k": normal(n, nkv, most, d), "v": normal(n, nkv, most, d)}
    if case["prefix"]:
        x["pk"], x["pv"] = normal(nkv, case["prefix"], d), normal(nkv, case["prefix"], d)
    rows = sum(lens) if case["op"] in ("prompt", "received") else n
    if case["op"] != "evict":
        x["q"] = normal(rows, nq, d, sigma=1.5)  # scores of a spread of 1.5 before the cap
    if case["op"] == "evict" or case["totals"] or case["op"] == "received":
        # totals as generation leaves them: a few keys hold most of the weight, some were never looked at; before a prompt's rows little
        t = torch.randn((n, nkv, most), generator=gen, device="cuda").mul_(2.0).exp_().mul_(0.01 if case["op"] == "received" else 1.0)
        x["totals"] = t * (torch.rand((n, nkv, most), generator=gen, device="cuda") > 0.05)
    if case["page"]:
        pages = -(-most // case["page"])
        x["table"] = torch.randperm(n * pages, generator=gen, device="cuda").reshape(n, pages).to(torch.int32)
    return x


def _paged(case, slab, table):
    """the slab's keys in a pool of pages [pages, kv heads, page, d]"""
    n, nkv, most, d = slab.shape
    pages, size = table.shape[1], case["page"]
    full = torch.zeros((n, nkv, pages * size, d), dtype=slab.dtype, device=slab.device)
    full[:, :, :most] = slab
    pool = torch.empty((n * pages, nkv, size, d), dtype=slab.dtype, device=slab.device)
    pool[table.reshape(-1).long()] = full.reshape(n, nkv, pages, size, d).permute(0, 2, 1, 3, 4).reshape(n * pages, nkv, size, d)
    return pool


def prepare(case, seed):
    x, lens, held = _draw_inputs(case, seed), _lens(case), _held(case)
    n, nkv, most = len(lens), case["kv_heads"], max(held)
    s = {"case": case, "most": most, "held": _ints(held), "scale": 1.0 / math.sqrt(case["head_dim"]), **x}
    if case["page"]:
        s["k"], s["v"] = _paged(case, x["k"], x["table"]), _paged(case, x["v"], x["table"])
    if case["slopes"]:
        s["slopes"] = torch.tensor(_slopes(case), dtype=torch.float32, device="cuda")
    if case["docs"]:
        ids = [_doc_ids(case, h) for h in held]
        s["key_doc"] = _ints([i + [0] * (most - len(i)) for i in ids])[:, None].expand(n, nkv, most)
        s["q_doc"] = _ints([v for i, m in zip(ids, lens) for v in i[len(i) - m:]])
    if case["see_all"]:
        s["see_all"] = _ints([case["see_all"]] * n)
    if case["op"] in ("prompt", "received"):
        s["most_rows"] = max(lens)
        s["q_start"] = _ints([sum(lens[:i]) for i in range(n + 1)])
    if case["op"] == "received":
        # what attn_prompt leaves for its rows; here from the formula, in slices
        s["lse"] = _lse(s)
    if case["op"] == "evict":
        K, dt = case["keep"], _dtype(case)
        s["to_k"] = torch.zeros((n, nkv, K, case["head_dim"]), dtype=dt, device="cuda")
        s["to_v"], s["to_held"] = torch.zeros_like(s["to_k"]), torch.zeros_like(s["held"])
        s["to_pos"] = torch.zeros((n, nkv, K), dtype=torch.int32, device="cuda")
        s["to_totals"] = torch.zeros((n, nkv, K), dtype=torch.float32, device="cuda")
    if own:  # the descriptions of the tensors above that a program keeps with them: no values, nothing computed
        import paper_2511_14450_amd as hyp
        s["cache"] = hyp.AttnCache(s["k"], s["v"], s["held"], page_table=s.get("table"), most=most, prefix_k=s.get("pk"),
                                   prefix_v=s.get("pv"), key_doc=s.get("key_doc"))
        s["rule"] = hyp.AttnRule(s["scale"], cap=case["cap"], slopes=s.get("slopes"))
        if case["op"] == "evict":
            s["to"] = hyp.AttnCache(s["to_k"], s["to_v"], s["to_held"], key_pos=s["to_pos"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"prompt": _prompt, "received": _received, "token": _token, "evict": _evict}[op](s)


def _run_own(s, op):
    import paper_2511_14450_amd as hyp
    case = s["case"]
    if op == "prompt":
        out, lse = hyp.attn_prompt(s["cache"], s["rule"], s["q"], s["q_start"], see_all=s.get("see_all"), q_doc=s.get("q_doc"))
        return {"out": out, "lse": lse}
    if op == "received":
        totals = torch.empty_like(s["totals"])
        hyp.attn_received(s["cache"], s["rule"], s["q"], s["q_start"], s["lse"], s["totals"], last=case["last"], totals_out=totals)
        return {"totals": totals}
    if op == "token":
        totals = torch.empty_like(s["totals"]) if case["totals"] else None
        out, lse = hyp.attn_token(s["cache"], s["rule"], s["q"], totals=s.get("totals"), totals_out=totals)
        return {"out": out, "lse": lse, "totals": totals}
    kept = hyp.attn_evict(s["cache"], s["totals"], case["keep"], sink=case["sink"], recent=case["recent"], into=s["to"], totals_out=s["to_totals"])
    return {"k": s["to_k"], "v": s["to_v"], "held": s["to_held"], "pos": s["to_pos"], "totals": s["to_totals"], "kept": kept}


# ---------------------------------------------------------------- the plain form
def _own_keys(s, name):
    """[n, kv heads, most, d] out of the slab or the pages"""
    if not s["case"]["page"]:
        return s[name]
    n, pages = s["table"].shape
    pool = s[name][s["table"].long()]  # [n, pages, kv heads, page, d]
    return pool.transpose(1, 2).reshape(n, pool.shape[2], -1, pool.shape[4])[:, :, :s["most"]]


def _all_keys(s, name, prefix, heads):
    """the shared prefix, then the own keys: [n, heads, keys, d] in 32 bits"""
    x = _own_keys(s, name)[:, heads]
    if prefix in s:
        x = torch.cat([s[prefix][heads][None].expand(x.shape[0], -1, -1, -1), x], 2)
    return x.float()


def _hidden(s, at, row_doc):
    """[n, rows, keys]: true where a row does not see a key; at: the rows' own index [n, rows]"""
    j = torch.arange(s["most"], device=at.device)
    above = j > at[:, :, None]
    if "see_all" in s:
        above &= j >= s["see_all"][:, None, None]
    own_part = above | (j >= s["held"][:, None, None])
    if "key_doc" in s:
        kd, rd = s["key_doc"][:, 0][:, None, :], row_doc[:, :, None]
        own_part |= (kd != rd) & (kd >= 0) & (rd >= 0)
    first = s["case"]["prefix"]
    return torch.nn.functional.pad(own_part, (first, 0)) if first else own_part


def _scores(s, q, heads, at, hidden):
    """[n, heads, group, rows, keys], -inf where hidden; q [n, rows, query heads, d]"""
    case = s["case"]
    n, rows, nq, d = q.shape
    group, count = nq // case["kv_heads"], heads.stop - heads.start
    qh = q[:, :, heads.start * group:heads.stop * group].float().permute(0, 2, 1, 3).reshape(n, count, group * rows, d)
    x = (qh @ _all_keys(s, "k", "pk", heads).transpose(2, 3)).mul_(s["scale"])
    if case["cap"]:
        x = x.div_(case["cap"]).tanh_().mul_(case["cap"])
    x = x.view(n, count, group, rows, -1)
    if "slopes" in s:
        pos = torch.arange(x.shape[-1], device=x.device)
        far = (case["prefix"] + at[:, :, None] - pos).abs().float()
        x -= s["slopes"][heads.start * group:heads.stop * group].view(count, group, 1, 1) * far[:, None, None]
    return x.masked_fill_(hidden[:, None, None], -math.inf)


def _slices(s, n, rows):
    """KV heads at a time, so that their scores stay under 4 GiB"""
    nkv = s["case"]["kv_heads"]
    each = 4 * n * rows * (s["case"]["q_heads"] // nkv) * (s["case"]["prefix"] + s["most"])
    step = max(1, min(nkv, (4 << 30) // each))
    return [slice(lo, min(nkv, lo + step)) for lo in range(0, nkv, step)]


def _attend(s, q, at, row_doc):
    """(out [n, rows, query heads, d], lse [n, rows, query heads]) in 32 bits"""
    n, rows, nq, d = q.shape
    hidden, outs, lses = _hidden(s, at, row_doc), [], []
    for heads in _slices(s, n, rows):
        x = _scores(s, q, heads, at, hidden)
        top = x.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        count, group = p.shape[1], p.shape[2]
        o = (p.view(n, count, group * rows, -1) @ _all_keys(s, "v", "pv", heads)).view(n, count, group, rows, d)
        o = torch.where(total > 0, o / total, torch.zeros_like(o))
        outs.append(o.reshape(n, count * group, rows, d))
        lses.append((total.log() + top).reshape(n, count * group, rows))
    return torch.cat(outs, 1).transpose(1, 2), torch.cat(lses, 1).transpose(1, 2)


def _padded(s, start, end, most_rows):
    """rows of the requests [n, most rows] (clamped), which of them are there, and their own index"""
    row = start[:, None] + torch.arange(most_rows, device=start.device)
    there = row < end[:, None]
    return row.clamp(max=s["q"].shape[0] - 1), there, s["held"][:, None] - (end[:, None] - row)


def _prompt(s):
    start, end = s["q_start"][:-1].long(), s["q_start"][1:].long()
    row, there, at = _padded(s, start, end, s["most_rows"])
    out, lse = _attend(s, s["q"][row], at, s["q_doc"][row] if "q_doc" in s else None)
    return {"out": out[there].to(s["q"].dtype), "lse": lse[there]}


def _lse(s):
    start, end = s["q_start"][:-1].long(), s["q_start"][1:].long()
    row, there, at = _padded(s, start, end, s["most_rows"])
    return _attend(s, s["q"][row], at, None)[1][there]


def _received(s):
    start, end = s["q_start"][:-1].long(), s["q_start"][1:].long()
    most_rows = min(s["case"]["last"] or s["most_rows"], s["most_rows"])
    row, there, at = _padded(s, torch.maximum(start, end - most_rows), end, most_rows)
    hidden, q, lse = _hidden(s, at, None), s["q"][row], s["lse"][row].masked_fill(~there[:, :, None], math.inf)
    got = []
    for heads in _slices(s, len(start), most_rows):
        x = _scores(s, q, heads, at, hidden)
        got.append(x.sub_(lse.transpose(1, 2).reshape(x.shape[0], s["case"]["kv_heads"], -1, most_rows, 1)[:, heads]).exp_().sum((2, 3)))
    return {"totals": s["totals"] + torch.cat(got, 1)[:, :, s["case"]["prefix"]:]}


def _token(s):
    at = s["held"][:, None].long() - 1
    out, lse = _attend(s, s["q"][:, None], at, None)
    if not s["case"]["totals"]:
        return {"out": out[:, 0].to(s["q"].dtype), "lse": lse[:, 0], "totals": None}
    x = _scores(s, s["q"][:, None], slice(0, s["case"]["kv_heads"]), at, _hidden(s, at, None))
    p = x.sub_(lse.transpose(1, 2).reshape(x.shape[:4] + (1,))).exp_().sum((2, 3))
    return {"out": out[:, 0].to(s["q"].dtype), "lse": lse[:, 0], "totals": s["totals"] + p[:, :, s["case"]["prefix"]:]}


def _evict(s):
    case = s["case"]
    K, totals = case["keep"], s["totals"]
    n, nkv, most = totals.shape
    K_in = min(K, most)
    j = torch.arange(most, device=totals.device)
    there = j < s["held"][:, None]                                                     # [n, most]
    always = (j < case["sink"]) | (j >= s["held"][:, None] - case["recent"])
    rank = torch.where(always[:, None], torch.full_like(totals, math.inf), totals)
    rank = torch.where(there[:, None], rank, torch.full_like(rank, -math.inf))
    best = rank.sort(dim=-1, descending=True, stable=True).indices[..., :K_in]
    stays = torch.zeros_like(totals, dtype=torch.bool).scatter_(2, best, True) & there[:, None]
    # a free slot below K gets the next kept key from K on
    free_rank = ((~stays[..., :K_in]).cumsum(-1) - 1).clamp(min=0)
    moved = torch.where(stays & (j >= K), j, most).sort(-1).values
    moved = torch.nn.functional.pad(moved, (0, K), value=most)
    source = torch.where(stays[..., :K_in], j[:K_in], moved.gather(2, free_rank))
    source = torch.nn.functional.pad(source, (0, K - K_in), value=most)
    valid = source < most
    safe = source.clamp(max=most - 1)

    def of(x):
        return x.gather(2, safe[..., None].expand(n, nkv, K, x.shape[-1])).masked_fill_(~valid[..., None], 0)

    return {"k": of(_own_keys(s, "k")), "v": of(_own_keys(s, "v")), "held": s["held"].clamp(max=K),
            "pos": (case["prefix"] + safe).masked_fill_(~valid, 0).int(), "totals": totals.gather(2, safe).masked_fill_(~valid, 0),
            "kept": source.masked_fill_(~valid, -1).int()}


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(case, window):
    """(row, key) pairs that are seen, one query head, own keys and prefix, of the rows that count"""
    pairs = 0
    for n, held in zip(_lens(case), _held(case)):
        rows = min(case["last"] or n, n) if window else n
        o = torch.arange(held - rows, held, dtype=torch.float64)
        seen = torch.maximum(o + 1, torch.full_like(o, min(case["see_all"], held)))
        if case["docs"]:  # a document's own keys up to the row, for the last part all; keys of the last part before a row there
            part = -(-held // (case["docs"] + 1))
            seen = torch.where(o >= part * case["docs"], seen, (o % part) + 1)
        pairs += float(seen.sum()) + rows * case["prefix"]
    return pairs


def work(case):
    lens, held = _lens(case), _held(case)
    es, nq, nkv, d = (2 if case["dtype"] == "bf16" else 4), case["q_heads"], case["kv_heads"], case["head_dim"]
    keys = sum(held) + case["prefix"]
    if case["op"] == "prompt":
        return {"bytes": 2 * sum(lens) * nq * d * es + 4 * sum(lens) * nq + 2 * keys * nkv * d * es, "flops": 4 * d * nq * _pairs(case, False)}
    if case["op"] == "received":
        rows = sum(min(case["last"] or n, n) for n in lens)
        own_pairs = _pairs(case, True) - rows * case["prefix"]  # only own keys' weights are asked for
        return {"bytes": rows * nq * (d * es + 4) + sum(held) * nkv * (d * es + 8), "flops": 2 * d * nq * own_pairs}
    if case["op"] == "token":
        n = len(lens)
        return {"bytes": n * nq * (2 * d * es + 4) + 2 * keys * nkv * d * es + (8 * sum(held) * nkv if case["totals"] else 0),
                "flops": 4 * d * nq * (sum(held) + n * case["prefix"])}
    kept = sum(min(h, case["keep"]) for h in held)
    return {"bytes": 4 * sum(held) * nkv + kept * nkv * (4 * d * es + 12), "flops": 0}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    x, lens, held = _draw_inputs(case, seed), _lens(case), _held(case)
    if case["op"] == "evict":
        return _exact_evict(case, x, held)
    group, P, d = case["q_heads"] // case["kv_heads"], case["prefix"], case["head_dim"]
    slopes = torch.tensor(_slopes(case), dtype=torch.float64, device="cuda") if case["slopes"] else None
    rows_of = [1] * len(lens) if case["op"] == "token" else lens
    out = torch.zeros((sum(rows_of),) + x["q"].shape[1:], dtype=torch.float64, device="cuda")
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device="cuda")
    totals = x["totals"].double() if "totals" in x else None
    first = 0
    for b, (n, h) in enumerate(zip(rows_of, held)):
        o = torch.arange(h - n, h, device="cuda")
        j = torch.arange(h, device="cuda")
        sees = j[None] <= o[:, None]
        if case["see_all"]:
            sees = sees | (j[None] < case["see_all"])
        if case["docs"]:
            ids = torch.tensor(_doc_ids(case, h), device="cuda")
            sees = sees & ((ids[None] == ids[o][:, None]) | (ids[None] < 0) | (ids[o][:, None] < 0))
        sees = torch.cat([torch.ones((n, P), dtype=torch.bool, device="cuda"), sees], 1)
        counts = n if not case["last"] else min(n, case["last"])
        for c in range(case["kv_heads"]):
            k, v = x["k"][b, c, :h].double(), x["v"][b, c, :h].double()
            if P:
                k, v = torch.cat([x["pk"][c].double(), k]), torch.cat([x["pv"][c].double(), v])
            for g in range(c * group, (c + 1) * group):
                s = x["q"][first:first + n, g].double() @ k.t() / math.sqrt(d)
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if slopes is not None:
                    s = s - slopes[g] * (P + o[:, None] - torch.arange(P + h, device="cuda")[None]).abs()
                s = torch.where(sees, s, torch.full_like(s, -math.inf))
                z = torch.logsumexp(s, -1)
                p = torch.exp(s - z[:, None])
                out[first:first + n, g], lse[first:first + n, g] = p @ v, z
                if totals is not None:
                    totals[b, c, :h] += p[n - counts:, P:].sum(0)
        first += n
    if case["op"] == "received":
        return {"totals": totals}
    return {"out": out, "lse": lse} if case["op"] == "prompt" else {"out": out, "lse": lse, "totals": totals if case["totals"] else None}


def _exact_evict(case, x, held):
    K = case["keep"]
    n, nkv, most = x["totals"].shape
    k, v = (torch.zeros((n, nkv, K, case["head_dim"]), dtype=torch.float64, device="cuda") for _ in range(2))
    totals = torch.zeros((n, nkv, K), dtype=torch.float64, device="cuda")
    for b, h in enumerate(held):
        for c in range(nkv):
            t = x["totals"][b, c, :h].tolist()
            if h > K:
                order = sorted(range(h), key=lambda j: (not (j < case["sink"] or j >= h - case["recent"]), -t[j], j))[:K]
                low, high = {j for j in order if j < K}, iter(sorted(j for j in order if j >= K))
                slots = [r if r in low else next(high) for r in range(K)]
            else:
                slots = list(range(h))
            at = torch.tensor(slots, device="cuda")
            k[b, c, :len(slots)], v[b, c, :len(slots)] = x["k"][b, c, at].double(), x["v"][b, c, at].double()
            totals[b, c, :len(slots)] = x["totals"][b, c, at].double()
    return {"k": k, "v": v, "held": None, "pos": None, "totals": totals, "kept": None}
