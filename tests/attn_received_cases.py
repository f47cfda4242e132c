"""Calls of attn_received that meet their keys by pairs of blocks, as arguments of tests.test_gpu_attn.Problem: many short requests and a few
long ones, since the form goes by how many pairs of blocks there are, and the arithmetic of a reference by the rows."""

BASE = dict(nq=8, nkv=2, d=128, requests=42, most=300, last=0, rule={})


def case(**more):
    return {**BASE, **more}


LAYOUTS = [case(d=d) for d in (33, 64, 80, 96, 128, 200, 256)] + [
    case(nq=6), case(nq=10, d=64), case(nq=40, nkv=1, requests=80, d=64), case(nq=2, requests=28, most=520, d=64),  # groups of 3, 5, 40 and 1
    case(most=129, requests=80), case(most=200, requests=80), case(most=257), case(most=385, d=64)]                                                           # even and odd numbers of blocks
RULES = [case(rule=r, **more) for r, more in (
    (dict(cap=5.0), {}), (dict(cap=50.0, sigma=4.0), dict(d=64)), (dict(slopes=True), dict(nq=6)), (dict(cap=2.0, slopes=True, pos=True), {}), (dict(docs=3), {}),
    (dict(docs=4, see_all=True), dict(d=64)), (dict(see_all=True), {}), (dict(docs=2, slopes=True, pos=True, cap=30.0), dict(nq=6, d=96)),
    (dict(page=16), {}), (dict(page=128, docs=2), dict(d=64)), (dict(layout="odd"), dict(d=64)), (dict(layout="odd", slopes=True, docs=3), {}),
    (dict(layout="tokens"), {}), (dict(prefix=40), {}))]
LAST = [case(last=200), case(last=299, nq=6, rule=dict(docs=3)), case(last=170, d=64, rule=dict(see_all=True, cap=20.0)), case(last=160, rule=dict(layout="odd"))]
ALL = LAYOUTS + RULES + LAST


def name(c):
    return " ".join([f"{c['nq']}/{c['nkv']}/{c['d']} {c['requests']}x{c['most']}"] + ([f"last {c['last']}"] if c["last"] else []) + [f"{k}={v}" for k, v in c["rule"].items()])


def problem(c, dtype, make):
    """make: the class Problem"""
    n, most = c["requests"], c["most"]
    held = [(17 * b) % 12 for b in range(n)]
    rows = [min(h, b % 4) for b, h in enumerate(held)]
    held[5], rows[5] = most, most              # a whole prompt, and the end of one
    held[n - 2], rows[n - 2] = most - 30, most // 3
    rule = dict(c["rule"])
    if rule.get("see_all"):
        rule["see_all"] = [(b * 37) % most for b in range(n)]
    return make(n + most + c["d"], dtype, c["nq"], c["nkv"], c["d"], held=held, rows=rows, **rule)
