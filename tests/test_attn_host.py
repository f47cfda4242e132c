"""Host-side checks of include/hyp_attn.h that need no GPU: exports, layouts, refusals before anything touches the device, the
reference's own closed forms, and the plain forms of perf/operators.py against it."""
import ctypes as C
import math
import pathlib
import re

import pytest
import torch

from paper_2511_14450_amd import attn, binding
from tests import attn_reference as ref

ROOT = pathlib.Path(__file__).resolve().parents[1]
EINVAL, ESHAPE, ENOMEM = binding.HYP_EINVAL, binding.HYP_ESHAPE, binding.HYP_ENOMEM


def test_library_exports_every_declared_symbol():
    declared = re.findall(r"HYP_API\s+[\w\s\*]+?\b(\w+)\s*\(", (ROOT / "include" / "hyp_attn.h").read_text())
    lib = attn._lib()
    assert all(hasattr(lib, name) for name in declared) and set(attn.EXPORTS_ATTN) == set(declared)


def test_structs_match_the_header(tmp_path):
    import subprocess
    src = tmp_path / "sizes.c"
    fields = {"hyp_attn_cache_t": attn._Cache, "hyp_attn_rule_t": attn._Rule, "hyp_attn_rows_t": attn._Rows, "hyp_attn_out_t": attn._Out, "hyp_attn_totals_t": attn._Totals}
    prints = "".join(f'printf("%zu ", offsetof({t}, {n.rstrip("_")}));' for t, s in fields.items() for n, _ in s._fields_)
    src.write_text('#include <stdio.h>\n#include "hyp_attn.h"\nint main(void) {' + prints + "".join(f'printf("%zu ", sizeof({t}));' for t in fields) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", f"-I{ROOT / 'include'}", str(src), "-o", str(tmp_path / "sizes")], check=True)  # the header is C
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(s, n).offset for s in fields.values() for n, _ in s._fields_] + [C.sizeof(s) for s in fields.values()]


def cache(**more):
    c = attn._Cache(k=4096, v=4096, lens=4096, k_page_stride=4096, k_head_stride=1024, k_key_stride=64, v_page_stride=4096, v_head_stride=1024,
                    v_key_stride=64, most=16, n_requests=2, n_kv_heads=2, head_dim=64, dtype=binding.HYP_BF16)
    for name, value in more.items():
        setattr(c, name, value)
    return c


def rows(**more):
    r = attn._Rows(q=4096, q_row_stride=256, q_head_stride=64, n_rows=2, n_q_heads=4)
    for name, value in more.items():
        setattr(r, name, value)
    return r


BAD_CACHE = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(lens=None), EINVAL), (dict(dtype=5), EINVAL), (dict(head_dim=0), ESHAPE), (dict(head_dim=257), ESHAPE),
             (dict(most=0), ESHAPE), (dict(n_requests=0), ESHAPE), (dict(n_kv_heads=-1), ESHAPE), (dict(prefix_len=-1), ESHAPE), (dict(prefix_len=3), EINVAL),
             (dict(page_table=64, page_keys=12, pages_per_request=2, n_pages=4), EINVAL), (dict(page_table=64, page_keys=8, pages_per_request=1, n_pages=4), ESHAPE),
             (dict(page_table=64, page_keys=8, pages_per_request=2, n_pages=0), ESHAPE), (dict(k=4097), EINVAL)]
BAD_ROWS = [(dict(q=None), EINVAL), (dict(n_q_heads=3), ESHAPE), (dict(n_q_heads=0), ESHAPE), (dict(n_q_heads=1024), ESHAPE), (dict(n_rows=-1), ESHAPE),
            (dict(n_rows=1 << 30), ESHAPE), (dict(q=4097), EINVAL)]
BAD_RULE = [((0.0, 0.0), EINVAL), ((-1.0, 0.0), EINVAL), ((math.nan, 0.0), EINVAL), ((math.inf, 0.0), EINVAL), ((1.0, -1.0), EINVAL), ((1.0, math.nan), EINVAL)]


def calls(c, r, rule, out, totals, ws=None, size=0):
    lib = attn._lib()
    ref_ = lambda x: None if x is None else C.byref(x)  # noqa: E731
    prompt = None if r is None else rows(**{n: getattr(r, n) for n, _ in r._fields_})
    if prompt is not None:
        prompt.q_start = 4096
    yield lib.attn_prompt(ref_(c), ref_(rule), ref_(prompt), ref_(out), ws, size, None)
    yield lib.attn_token(ref_(c), ref_(rule), ref_(r), ref_(out), ref_(totals), ws, size, None)
    yield lib.attn_received(ref_(c), ref_(rule), ref_(prompt), 4096, 0, ref_(totals), None)


RULE, OUT, TOTALS = attn._Rule(1.0, 0.0, None), attn._Out(4096, 256, 64, 4096), attn._Totals(4096, 4096, 32, 16, 32, 16)


@pytest.mark.parametrize("more,status", BAD_CACHE)
def test_a_bad_cache_is_refused(more, status):
    assert set(calls(cache(**more), rows(), RULE, OUT, TOTALS)) == {status} and attn.attn_last_error()
    lib = attn._lib()
    assert lib.attn_workspace_bytes(C.byref(cache(**more)), C.byref(rows()), None) == 0
    assert lib.attn_evict(C.byref(cache(**more)), None, C.byref(TOTALS), 4, 0, 0, None, 4096, 4096, 1 << 20, None) == status


@pytest.mark.parametrize("more,status", BAD_ROWS)
def test_bad_rows_are_refused(more, status):
    assert set(calls(cache(), rows(**more), RULE, OUT, TOTALS)) == {status}


@pytest.mark.parametrize("values,status", BAD_RULE)
def test_a_bad_rule_is_refused(values, status):
    assert set(calls(cache(), rows(), attn._Rule(values[0], values[1], None), OUT, TOTALS)) == {status}


def test_null_arguments_are_refused():
    assert set(calls(None, rows(), RULE, OUT, TOTALS)) == {EINVAL}
    assert set(calls(cache(), None, RULE, OUT, TOTALS)) == {EINVAL}
    assert set(calls(cache(), rows(), None, OUT, TOTALS)) == {EINVAL}
    lib, c, r = attn._lib(), cache(), rows()
    assert lib.attn_prompt(C.byref(c), C.byref(RULE), C.byref(r), C.byref(OUT), None, 0, None) == EINVAL       # no q_start
    r.q_start = 4096
    assert lib.attn_token(C.byref(c), C.byref(RULE), C.byref(r), C.byref(OUT), None, None, 0, None) == ESHAPE  # q_start
    assert lib.attn_prompt(C.byref(c), C.byref(RULE), C.byref(r), None, None, 0, None) == EINVAL
    assert lib.attn_received(C.byref(c), C.byref(RULE), C.byref(r), None, 0, C.byref(TOTALS), None) == EINVAL
    assert lib.attn_received(C.byref(c), C.byref(RULE), C.byref(r), 4096, -1, C.byref(TOTALS), None) == EINVAL
    assert lib.attn_received(C.byref(c), C.byref(RULE), C.byref(r), 4096, 0, None, None) == EINVAL
    uneven = attn._Totals(4096, 4096, 32, 16, 64, 16)
    assert lib.attn_received(C.byref(c), C.byref(RULE), C.byref(r), 4096, 0, C.byref(uneven), None) == EINVAL


def test_a_workspace_that_is_too_small_or_misaligned_is_refused():
    lib, c, r = attn._lib(), cache(), rows()
    need = lib.attn_workspace_bytes(C.byref(c), C.byref(r), C.byref(TOTALS))
    assert need > 0
    args = (C.byref(c), C.byref(RULE), C.byref(r), C.byref(OUT), C.byref(TOTALS))
    assert lib.attn_token(*args, None, 0, None) == EINVAL and lib.attn_token(*args, 4100, need, None) == EINVAL
    assert lib.attn_token(*args, 4096, need - 1, None) == ENOMEM


@pytest.mark.parametrize("keep,sink,recent,more,status", [(0, 0, 0, {}, EINVAL), (4, -1, 0, {}, EINVAL), (4, 3, 2, {}, EINVAL), (4, 0, 0, dict(kept=None), EINVAL),
                                                          (4, 0, 0, dict(ws=None), EINVAL), (4, 0, 0, dict(size=8), ENOMEM), (4, 0, 0, dict(totals=attn._Totals(4096, 8192)), EINVAL),
                                                          (4, 0, 0, dict(c=cache(key_pos=4096)), EINVAL), (4, 0, 0, dict(into=cache(head_dim=32, k=64, v=64, lens=64)), ESHAPE),
                                                          (17, 0, 0, dict(into=cache(k=64, v=64, lens=64), totals=attn._Totals(4096, 8192)), ESHAPE),
                                                          (4, 0, 0, dict(into=cache(), totals=attn._Totals(4096, 8192)), EINVAL)])
def test_bad_evictions_are_refused(keep, sink, recent, more, status):
    lib, c, into = attn._lib(), more.get("c", cache()), more.get("into")
    got = lib.attn_evict(C.byref(c), None if into is None else C.byref(into), C.byref(more.get("totals", TOTALS)), keep, sink, recent, None, more.get("kept", 4096),
                         more.get("ws", 4096), more.get("size", 1 << 20), None)
    assert got == status


def test_reference_closed_forms():
    # scores 0 and ln 2: probabilities 1/3 and 2/3; capped to c tanh(ln 2 / c); a distance of 1 with slope ln 2 evens them out
    q, k, v = torch.tensor([[1.0]]), torch.tensor([[0.0], [math.log(2.0)]]), torch.tensor([[3.0], [0.0]])
    out, lse, p, *_ = ref.attend(q, k, v, [1], scale=1.0)
    assert float(out) == pytest.approx(1.0) and float(lse) == pytest.approx(math.log(3.0)) and p[0].tolist() == pytest.approx([1 / 3, 2 / 3])
    s = 2.0 * math.tanh(math.log(2.0) / 2.0)
    out, *_ = ref.attend(q, k, v, [1], scale=1.0, cap=2.0)
    assert float(out) == pytest.approx(3.0 / (1.0 + math.exp(s)))
    out, *_ = ref.attend(q, torch.tensor([[math.log(2.0)], [0.0]]), v, [1], scale=1.0, slope=math.log(2.0))
    assert float(out) == pytest.approx(1.5)
    # a row before the keys, and ids: empty, its own, all
    out, lse, *_ = ref.attend(q, k, v, [-1], scale=1.0)
    assert float(out) == 0.0 and float(lse) == -math.inf
    for doc, want in ((0, 3.0), (1, 0.0), (-1, 1.0), (2, 0.0)):
        assert float(ref.attend(q, k, v, [1], scale=1.0, q_doc=[doc], key_doc=[0, 1])[0]) == pytest.approx(want)
    # see_all shows a later key; the shared prefix comes first
    assert float(ref.attend(q, k, v, [0], scale=1.0, see_all=2)[0]) == pytest.approx(1.0)
    assert float(ref.attend(q, k[1:], v[1:], [0], scale=1.0, prefix=(k[:1], v[:1]))[0]) == pytest.approx(1.0)


def test_reference_eviction():
    assert ref.evict([5.0, 1.0, 3.0, 4.0], 4, 2, 0, 0, [0, 1, 2, 3], 0, 4) == [0, 3]
    assert ref.evict([1.0, 1.0, 1.0, 1.0], 4, 2, 0, 0, [0, 1, 2, 3], 0, 4) == [0, 1]
    assert ref.evict([0.0, 9.0, 8.0, math.nan], 4, 3, 1, 1, [0, 1, 2, 3], 0, 4) == [0, 1, 3]
    assert ref.evict([1.0], 1, 3, 0, 0, [0], 0, 1) == [0, -1, -1]
