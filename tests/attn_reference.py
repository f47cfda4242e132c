"""Attention over a shared prefix and own keys, and eviction, from their formulas in 64 bits, with a bound on what the 32-bit
(and, for bf16, once rounded) arithmetic of the library may be off.  One row, one head at a time; no code of the library."""
from __future__ import annotations

import math

import torch


def attend(q, own_k, own_v, at, *, scale, prefix=None, cap=0.0, slope=0.0, see_all=0, q_doc=None, key_doc=None, q_pos=None, key_pos=None):
    """One head of one request.  q [rows, d], own_k / own_v [held, d], at [rows]: own index of the rows; ids and positions as lists.
    Returns out, lse, p over own keys, and bounds of the error of out (without rounding), of lse and of p."""
    P = 0 if prefix is None else prefix[0].shape[0]
    k, v = own_k.double(), own_v.double()
    if P:
        k, v = torch.cat([prefix[0].double(), k]), torch.cat([prefix[1].double(), v])
    rows, held = q.shape[0], own_k.shape[0]
    out, lse, p_own = torch.zeros((rows, v.shape[1]), dtype=torch.float64), torch.full((rows,), -math.inf, dtype=torch.float64), torch.zeros((rows, held), dtype=torch.float64)
    out_abs, delta = torch.zeros_like(out), torch.zeros(rows, dtype=torch.float64)
    for i in range(rows):
        o = int(at[i])
        seen = [True] * P
        for j in range(held):
            ok = j <= o or j < see_all
            if q_doc is not None and key_doc is not None:
                ok = ok and (q_doc[i] < 0 or key_doc[j] < 0 or q_doc[i] == key_doc[j])
            seen.append(ok)
        idx = torch.tensor([j for j, s in enumerate(seen) if s], dtype=torch.long)
        if idx.numel() == 0:
            continue
        qi, ki = q[i].double(), k[idx]
        s = scale * (ki @ qi)
        size = scale * (ki.abs() @ qi.abs())
        if cap:
            s = cap * torch.tanh(s / cap)
        if slope:
            pos = torch.tensor([j if j < P else (P + j - P if key_pos is None else key_pos[j - P]) for j in idx.tolist()], dtype=torch.float64)
            mine = P + o if q_pos is None else q_pos[i]
            s = s - slope * (mine - pos).abs()
            size = size + slope * (mine - pos).abs()
        z = torch.logsumexp(s, 0)
        w = torch.exp(s - z)
        out[i], lse[i] = w @ v[idx], z
        out_abs[i] = w @ v[idx].abs()
        # a sum of d products, then a few roundings of numbers up to that size, the maximum, and their exponential
        delta[i] = 2.0 ** -21 * (float(size.max()) + abs(float(z)) + 4)
        own = idx >= P
        p_own[i, idx[own] - P] = w[own]
    return out, lse, p_own, out_abs, delta


def out_bound(out, out_abs, delta, dtype):
    """Each probability is off by delta, relatively; sums of up to a few thousand terms by 2^-19; bf16 rounds probabilities and result,
    each by at most 2^-8 of itself (8 significant bits: half a unit in the last place of 1.0 is 2^-8)."""
    b = (2 * delta[:, None] + 2.0 ** -19) * out_abs + 1e-30
    if dtype == torch.bfloat16:
        b = b + 2.0 ** -8 * out_abs + 2.0 ** -8 * out.abs()
    return b


def evict(totals, held, keep, sink, recent, pos, first, now):
    """Slots (list of `keep`, -1 behind the last) that the result's keys come from; totals, pos: lists of one request and head."""
    if held <= keep:
        return [r if r < held else -1 for r in range(keep)]
    def order(j):
        always = pos[j] < first + sink or pos[j] >= now - recent
        t = totals[j]
        return (not always, -(t if t == t else -math.inf), t != t, j)
    stay = set(sorted(range(held), key=order)[:keep])
    high = iter(sorted(j for j in stay if j >= keep))
    return [r if r in stay else next(high) for r in range(keep)]
