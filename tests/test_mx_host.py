"""Host-side checks of include/hyp_mx.h that need no GPU: exports, layouts, refusals before anything touches the device, the binding's own, and the
reference's closed forms."""
import ctypes as C
import math
import pathlib
import random
import subprocess
import re

import pytest
import torch

import paper_2511_14450_amd as hyp
from paper_2511_14450_amd import attn, binding, mx
from tests import mx_reference as ref
from tests.test_attn_refusals import On, f32, i32

ROOT = pathlib.Path(__file__).resolve().parents[1]
OK, EINVAL, ESHAPE, ENOMEM = binding.HYP_OK, binding.HYP_EINVAL, binding.HYP_ESHAPE, binding.HYP_ENOMEM


def test_library_exports_every_declared_symbol():
    declared = re.findall(r"HYP_API\s+[\w\s\*]+?\b(\w+)\s*\(", (ROOT / "include" / "hyp_mx.h").read_text())
    lib = mx._lib()
    assert all(hasattr(lib, name) for name in declared) and set(mx.EXPORTS_MX) == set(declared)
    assert all(hasattr(hyp, name) for name in declared)


def test_structs_match_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    fields = {"hyp_mx_cache_t": mx._MxCache, "hyp_mx_rows_t": mx._MxRows, "hyp_mx_out_t": mx._MxOut, "hyp_mx_q_t": mx._MxQ}
    prints = "".join(f'printf("%zu ", offsetof({t}, {n}));' for t, s in fields.items() for n, _ in s._fields_)
    src.write_text('#include <stdio.h>\n#include "hyp_mx.h"\nint main(void) {' + prints + "".join(f'printf("%zu ", sizeof({t}));' for t in fields) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", f"-I{ROOT / 'include'}", str(src), "-o", str(tmp_path / "sizes")], check=True)  # the header is C
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [getattr(s, n).offset for s in fields.values() for n, _ in s._fields_] + [C.sizeof(s) for s in fields.values()]


def cache(**more):
    """two requests of two heads, 64 keys of 64 features in 8 bits, blocks of 16"""
    c = mx._MxCache(k=4096, v=8192, k_scale=4096, v_scale=8192, k_page_stride=8192, k_head_stride=4096, k_key_stride=64, v_page_stride=8192, v_head_stride=4096,
                    v_key_stride=64, k_scale_page_stride=256, k_scale_head_stride=128, k_scale_group_stride=64, v_scale_page_stride=256, v_scale_head_stride=128,
                    v_scale_group_stride=64, page_keys=64, lens=4096, most=60, n_requests=2, n_kv_heads=2, head_dim=64, lo=4096, hi=8192, bound_page_stride=512,
                    bound_head_stride=256, bound_block_stride=64, block_keys=16)
    for name, value in more.items():
        setattr(c, name, value)
    return c


def rows(**more):
    r = mx._MxRows(k=4096, v=8192, k_row_stride=128, k_head_stride=64, v_row_stride=128, v_head_stride=64, n_rows=2, dtype=binding.HYP_BF16)
    for name, value in more.items():
        setattr(r, name, value)
    return r


def to(**more):
    t = mx._MxOut(4096, 8192, 8192, 4096, 64, 8192, 4096, 64, 64, binding.HYP_F32)
    for name, value in more.items():
        setattr(t, name, value)
    return t


def q(**more):
    t = mx._MxQ(4096, 256, 64, 4, binding.HYP_BF16)
    for name, value in more.items():
        setattr(t, name, value)
    return t


RULE, OUT, BIG = attn._Rule(1.0, 0.0, None), attn._Out(4096, 256, 64, 4096), 1 << 60
ref_ = lambda x: None if x is None else C.byref(x)  # noqa: E731


def write(c=cache(), r=rows()):
    return mx._lib().mx_write(ref_(c), ref_(r), None)


def read(c=cache(), t=to()):
    return mx._lib().mx_read(ref_(c), None, ref_(t), None)


def select(c=cache(), row=q(), keep=2, sink=0, recent=0, blocks=4096, ws=4096, size=BIG):
    return mx._lib().mx_select(ref_(c), ref_(row), keep, sink, recent, blocks, ws, size, None)


def token(c=cache(), rule=RULE, row=q(), blocks=None, listed=0, out=OUT, ws=4096, size=BIG):
    return mx._lib().mx_token(ref_(c), ref_(rule), ref_(row), blocks, listed, ref_(out), ws, size, None)


PAGED = dict(page_table=4096, page_keys=32, pages_per_request=2, n_pages=4)
BAD_CACHE = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k_scale=None), EINVAL), (dict(v_scale=None), EINVAL), (dict(lens=None), EINVAL), (dict(k_format=2), EINVAL),
             (dict(v_format=-1), EINVAL), (dict(head_dim=0), ESHAPE), (dict(head_dim=257), ESHAPE), (dict(most=0), ESHAPE), (dict(most=65), ESHAPE), (dict(n_requests=0), ESHAPE),
             (dict(n_kv_heads=-1), ESHAPE), (dict(n_requests=1 << 23), ESHAPE), (dict(page_keys=63), EINVAL), (dict(page_keys=0), EINVAL), (dict(k=4104), EINVAL), (dict(v=4104), EINVAL),
             (dict(k_key_stride=72), EINVAL), (dict(v_head_stride=4104), EINVAL), (dict(k_key_stride=-64), ESHAPE), (dict(v_key_stride=1 << 24), ESHAPE), (dict(k_scale=4098), EINVAL),
             (dict(v_scale_group_stride=66), EINVAL), (dict(lo=None), EINVAL), (dict(hi=4097), EINVAL), (dict(block_keys=0), EINVAL), (dict(block_keys=8), EINVAL),
             (dict(block_keys=48), EINVAL), (dict(block_keys=128), ESHAPE), (dict(**{**PAGED, "page_keys": 48}), EINVAL), (dict(**{**PAGED, "page_keys": 8}), EINVAL),
             (dict(**{**PAGED, "pages_per_request": 1}), ESHAPE), (dict(**{**PAGED, "n_pages": 0}), ESHAPE), (dict(**{**PAGED, "block_keys": 64}), ESHAPE)]


@pytest.mark.parametrize("more,status", BAD_CACHE)
def test_a_bad_cache_is_refused(more, status):
    c, lib = cache(**more), mx._lib()
    assert {write(c), read(c), select(c), token(c)} == {status} and hyp.mx_last_error()
    assert lib.mx_select_workspace_bytes(C.byref(c), C.byref(q()), 2) == 0 and lib.mx_token_workspace_bytes(C.byref(c), C.byref(q()), 0) == 0


def test_null_arguments_are_refused():
    assert {write(None), write(r=None), read(None), read(t=None), select(None), select(row=None), select(blocks=None), token(None), token(rule=None), token(row=None), token(out=None)} == {EINVAL}


@pytest.mark.parametrize("more,status", [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(dtype=2), EINVAL), (dict(n_rows=-1), ESHAPE), (dict(n_rows=1 << 30, q_start=4096), ESHAPE),
                                         (dict(n_rows=3), ESHAPE), (dict(k=4097), EINVAL), (dict(k_out=4096), EINVAL), (dict(v_out=64), EINVAL),
                                         (dict(k_out=64, v_out=128, k_out_row_stride=128, k_out_head_stride=64, v_out_row_stride=0, v_out_head_stride=64), EINVAL),
                                         (dict(k_out=64, v_out=128, k_out_row_stride=128, k_out_head_stride=0, v_out_row_stride=128, v_out_head_stride=64), EINVAL),
                                         (dict(k_out=4096, v_out=8192, k_out_row_stride=256, k_out_head_stride=64, v_out_row_stride=128, v_out_head_stride=64), EINVAL),
                                         (dict(k_out=64, v_out=64, k_out_row_stride=128, k_out_head_stride=64, v_out_row_stride=128, v_out_head_stride=64), EINVAL),
                                         (dict(k_out=8192, v_out=64, k_out_row_stride=128, k_out_head_stride=64, v_out_row_stride=128, v_out_head_stride=64), EINVAL)])
def test_bad_rows_are_refused(more, status):
    assert write(r=rows(**more)) == status


@pytest.mark.parametrize("shared", ["k_page_stride", "k_head_stride", "k_key_stride", "v_page_stride", "v_head_stride", "v_key_stride", "k_scale_page_stride", "k_scale_head_stride",
                                    "k_scale_group_stride", "v_scale_page_stride", "v_scale_head_stride", "v_scale_group_stride", "bound_page_stride", "bound_head_stride",
                                    "bound_block_stride"])
def test_rows_are_not_written_to_memory_that_keys_share(shared):
    assert write(cache(**{shared: 0})) == EINVAL
    assert write(cache(**{shared: 0}), rows(n_rows=0, q_start=4096, k=None, v=None)) == EINVAL
    assert write(cache(hi=4096)) == EINVAL


def test_no_rows_and_no_room_are_no_work():
    assert write(r=rows(n_rows=0, q_start=4096, k=None, v=None)) == OK
    assert read(t=to(keys=0, k=None, v=None)) == OK


@pytest.mark.parametrize("more,status", [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=4098), EINVAL), (dict(dtype=3), EINVAL), (dict(keys=-1), ESHAPE), (dict(v=4096), EINVAL),
                                         (dict(k_request_stride=0), EINVAL), (dict(k_head_stride=0), EINVAL), (dict(k_key_stride=0), EINVAL), (dict(v_request_stride=0), EINVAL),
                                         (dict(v_head_stride=0), EINVAL), (dict(v_key_stride=0), EINVAL)])
def test_bad_places_to_read_to_are_refused(more, status):
    assert read(t=to(**more)) == status


BAD_Q = [(dict(q=None), EINVAL), (dict(q=4097), EINVAL), (dict(dtype=9), EINVAL), (dict(n_q_heads=0), ESHAPE), (dict(n_q_heads=3), ESHAPE), (dict(n_q_heads=1024), ESHAPE)]


@pytest.mark.parametrize("more,status", BAD_Q)
def test_bad_query_rows_are_refused(more, status):
    assert select(row=q(**more)) == token(row=q(**more)) == status


def test_bad_selections_are_refused():
    assert select(cache(lo=None, hi=None)) == EINVAL
    assert {select(keep=0), select(keep=-1), select(keep=1 << 30), select(sink=-1), select(recent=-1), select(sink=2, recent=1), select(sink=2 ** 31 - 1, recent=2 ** 31 - 1)} == {EINVAL}
    long, lib = cache(most=1 << 20, page_keys=1 << 20), mx._lib()
    need = lib.mx_select_workspace_bytes(C.byref(long), C.byref(q()), 7)
    assert need == 2 * 2 * (1 << 16) * 8 and lib.mx_select_workspace_bytes(C.byref(long), C.byref(q()), 1 << 16) == 0  # all are kept
    assert select(long, keep=7, ws=None, size=0) == EINVAL and select(long, keep=7, ws=4104, size=need) == EINVAL and select(long, keep=7, size=need - 1) == ENOMEM


@pytest.mark.parametrize("values", [(0.0, 0.0), (-1.0, 0.0), (math.nan, 0.0), (math.inf, 0.0), (1.0, -1.0), (1.0, math.nan), (3e38, 0.0)])
def test_a_bad_rule_is_refused(values):
    assert token(rule=attn._Rule(*values, None)) == EINVAL


def test_bad_tokens_are_refused():
    assert {token(listed=-1), token(listed=2), token(blocks=4096)} == {EINVAL}
    assert token(cache(lo=None, hi=None, block_keys=0), blocks=4096, listed=2) == EINVAL
    assert token(blocks=4096, listed=1 << 30) == ESHAPE
    for out in (attn._Out(None, 256, 64, 4096), attn._Out(4097, 256, 64, 4096), attn._Out(4096, 0, 64, 4096), attn._Out(4096, 256, 0, 4096)):
        assert token(out=out) == EINVAL
    long, lib = cache(most=1 << 20, page_keys=1 << 20), mx._lib()
    need = lib.mx_token_workspace_bytes(C.byref(long), C.byref(q()), 0)
    assert need > 0
    assert token(long, ws=None, size=0) == EINVAL and token(long, ws=4100, size=need) == EINVAL and token(long, size=need - 1) == ENOMEM


def test_calls_beyond_a_launch_are_refused():
    # a launch has fewer than 2^32 lanes, that is 2^24 workgroups of 256 and 2^22 of 1024
    many = cache(n_requests=(1 << 23) - 1, n_kv_heads=2)
    assert write(many, rows(n_rows=(1 << 23) - 1, q_start=4096)) == ESHAPE
    wide = dict(n_requests=1 << 22, n_kv_heads=1)
    assert read(cache(most=1 << 20, page_keys=1 << 20, **wide), to(keys=1 << 20)) == ESHAPE
    assert select(cache(most=1 << 20, page_keys=1 << 20, **wide)) == ESHAPE
    assert token(cache(**wide), row=q(n_q_heads=256)) == ESHAPE   # sixteen tiles of heads


# ---------------------------------------------------------------- the binding
def u8(*shape, index=0):
    return On(torch.zeros(shape, dtype=torch.uint8), index)


def bf16(*shape, index=0):
    return On(torch.zeros(shape, dtype=torch.bfloat16), index)


def parts(**more):
    return {**dict(k=u8(2, 2, 32, 96), v=u8(2, 2, 32, 48), k_scale=u8(2, 2, 3, 32), v_scale=u8(2, 2, 3, 32), lens=i32(2), head_dim=80, lo=bf16(2, 2, 2, 80), hi=bf16(2, 2, 2, 80)), **more}


def test_a_cache_is_described_by_its_tensors():
    c = mx.MxCache(**parts())
    assert (c._c.k_format, c._c.v_format, c._c.page_keys, c._c.most, c.block_keys, c._c.bound_block_stride) == (mx.HYP_E4M3, mx.HYP_E2M1, 32, 32, 16, 80)
    assert (c._c.k_key_stride, c._c.v_key_stride, c._c.k_scale_group_stride, c.n_requests) == (96, 48, 32, 2)
    paged = mx.MxCache(**parts(lens=i32(3), page_table=i32(3, 5)), most=77)
    assert (paged.n_requests, paged.most, paged._c.n_pages, paged._c.pages_per_request) == (3, 77, 2, 5)


@pytest.mark.parametrize("more", [dict(k=u8(2, 2, 32, 64)), dict(k=u8(2, 2, 16, 96)), dict(k=f32(2, 2, 32, 96)), dict(v=u8(2, 2, 32, 47)), dict(k_scale=u8(2, 2, 32, 3)), dict(v_scale=u8(2, 2, 2, 32)),
                                  dict(lens=i32(3)), dict(lens=On(torch.zeros(2, dtype=torch.int64))), dict(head_dim=0), dict(head_dim=257), dict(head_dim=64), dict(hi=None),
                                  dict(hi=bf16(2, 2, 1, 80)), dict(lo=bf16(2, 2, 3, 80), hi=bf16(2, 2, 3, 80)), dict(lo=bf16(2, 2, 2, 64), hi=bf16(2, 2, 2, 64)), dict(lo=f32(2, 2, 2, 80)),
                                  dict(most=33), dict(block_keys=32), dict(page_table=i32(2)), dict(k=On(torch.zeros(2, 2, 32, 192, dtype=torch.uint8)[..., ::2]))])
def test_a_cache_whose_tensors_do_not_go_together_is_refused(more):
    with pytest.raises(ValueError):
        mx.MxCache(**parts(**more))


def test_tensors_on_another_device_than_the_cache_are_refused(monkeypatch):
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(attn, "_raw_stream", lambda index: 0)
    for given in (parts(), parts(page_table=i32(2, 1))):
        mx.MxCache(**given)
        for name, t in given.items():
            if isinstance(t, On):
                with pytest.raises(ValueError):
                    mx.MxCache(**{**given, name: On(t.t, 1)})
    c, rule, work = mx.MxCache(**parts()), attn.AttnRule(0.125), On(torch.zeros(0, dtype=torch.uint8))

    def refused(call, *args, **kw):
        for i, t in enumerate(args):
            if isinstance(t, On):
                with pytest.raises(ValueError):
                    call(c, *args[:i], On(t.t, 1), *args[i + 1:], **kw)
        for name, t in kw.items():
            if isinstance(t, On):
                with pytest.raises(ValueError):
                    call(c, *args, **{**kw, name: On(t.t, 1)})
        current[0] = 1  # all of them on the device that is not the current one
        with pytest.raises(ValueError, match="device"):
            call(c, *args, **kw)
        current[0] = 0

    refused(mx.mx_write, bf16(9, 2, 80), bf16(9, 2, 80), q_start=i32(3), k_out=bf16(9, 2, 80), v_out=bf16(9, 2, 80))
    refused(mx.mx_read, f32(2, 2, 9, 80), f32(2, 2, 9, 80), first=i32(2))
    refused(mx.mx_select, bf16(2, 4, 80), 1, blocks=i32(2, 2, 1), workspace=work)
    refused(mx.mx_token, rule, f32(2, 4, 80), blocks=i32(2, 2, 1), out=f32(2, 4, 80), lse=f32(2, 4), workspace=work)
    for slopes in (f32(4, index=1), f32(3)):
        with pytest.raises(ValueError):
            mx.mx_token(c, attn.AttnRule(0.125, slopes=slopes), f32(2, 4, 80), out=f32(2, 4, 80), lse=f32(2, 4), workspace=work)


def test_tensors_of_other_shapes_and_types_are_refused():
    c, rule = mx.MxCache(**parts()), attn.AttnRule(0.125)
    half = On(torch.zeros((2, 2, 80), dtype=torch.float16))
    strided = On(torch.zeros((2, 2, 160))[..., ::2])
    for k, v in ((bf16(2, 2, 64), bf16(2, 2, 64)), (bf16(2, 3, 80), bf16(2, 3, 80)), (bf16(2, 2, 80), f32(2, 2, 80)), (bf16(2, 2, 80), bf16(3, 2, 80)), (half, half), (strided, strided)):
        with pytest.raises(ValueError):
            mx.mx_write(c, k, v)
    with pytest.raises(ValueError):
        mx.mx_write(c, f32(2, 2, 80), f32(2, 2, 80), k_out=f32(2, 2, 80))
    with pytest.raises(ValueError):
        mx.mx_write(c, f32(2, 2, 80), f32(2, 2, 80), q_start=i32(2))
    for k, v in ((f32(2, 2, 80), f32(2, 2, 80)), (f32(2, 2, 5, 64), f32(2, 2, 5, 64)), (f32(2, 2, 5, 80), f32(2, 2, 6, 80)), (f32(2, 2, 5, 80), bf16(2, 2, 5, 80)), (f32(3, 2, 5, 80), f32(3, 2, 5, 80))):
        with pytest.raises(ValueError):
            mx.mx_read(c, k, v)
    for row in (f32(3, 4, 80), f32(2, 4, 64), half, On(torch.zeros((2, 4, 160))[..., ::2])):
        with pytest.raises(ValueError):
            mx.mx_token(c, rule, row)
        with pytest.raises(ValueError):
            mx.mx_select(c, row, 1)
    for blocks in (i32(2, 2), i32(2, 2, 0), i32(2, 3, 4), On(torch.zeros((2, 2, 4), dtype=torch.int64))):
        with pytest.raises(ValueError):
            mx.mx_token(c, rule, f32(2, 4, 80), blocks=blocks)
    with pytest.raises(ValueError):
        mx.mx_select(c, f32(2, 4, 80), 2, blocks=i32(2, 2, 1))
    for name in ("keep", "sink", "recent"):
        with pytest.raises(ValueError, match=name):
            mx.mx_select(c, f32(2, 4, 80), **{**dict(keep=1), name: (1 << 32) + 1})


# ---------------------------------------------------------------- the reference
def test_formats_have_the_numbers_of_their_bits():
    assert [ref.number("e2m1", c) for c in range(8)] == [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0] and ref.number("e2m1", 15) == -6.0
    assert ref.number("e4m3", 0x7e) == 448.0 and ref.number("e4m3", 1) == 2.0 ** -9 and ref.number("e4m3", 0x38) == 1.0 and math.isnan(ref.number("e4m3", 0xff))
    for c in range(256):  # torch's type of the same bits
        t = float(torch.tensor([c], dtype=torch.uint8).view(torch.float8_e4m3fn).float())
        assert ref.number("e4m3", c) == t or (math.isnan(t) and math.isnan(ref.number("e4m3", c)))


@pytest.mark.parametrize("fmt", sorted(ref.FORMATS))
def test_the_reference_quantises_by_the_definition(fmt):
    most = ref.FORMATS[fmt]["most"]
    assert ref.group(fmt, [most, 0.0]) == (127, [most, 0.0])
    s, v = ref.group(fmt, [math.nextafter(most, 1e9), 1.0])
    assert s == 128 and v == [most, 1.0]                                                   # the next power of two, and its nearest number
    assert ref.group(fmt, [0.0, -0.0])[0] == 127 + ref.FORMATS[fmt]["low"]
    assert ref.group(fmt, [1.0, math.inf])[0] == 255 and math.isnan(ref.group(fmt, [1.0, math.nan])[1][0])
    rng = random.Random(3)
    x = torch.tensor([[math.ldexp(rng.uniform(-2, 2), rng.choice((0, 0, 0, -3, 4, -40, 60, -126, 127))) for _ in range(70)] for _ in range(40)] + [[3.4e38] * 70, [0.0] * 70], dtype=torch.float32)
    x[3, 5], x[4, 40] = math.inf, math.nan
    assert torch.equal(torch.tensor([ref.stored(fmt, row)[1] for row in x.double().tolist()]).double().nan_to_num(7e77), ref.stored_rows(fmt, x).nan_to_num(7e77))


def test_the_reference_selects_and_attends():
    lo, hi = torch.tensor([[0.0], [1.0], [2.0], [1.0]]), torch.tensor([[0.5], [3.0], [2.0], [3.0]])
    assert ref.select(torch.tensor([[1.0]]), lo, hi, 61, 16, 2, 0, 0) == [1, 3]
    assert ref.select(torch.tensor([[1.0]]), lo, hi, 61, 16, 2, 1, 0) == [0, 1]
    assert ref.select(torch.tensor([[-1.0]]), lo, hi, 64, 16, 1, 0, 0) == [0]
    assert ref.select(torch.tensor([[1.0]]), lo, hi, 64, 16, 5, 0, 0) == [0, 1, 2, 3, -1]
    hi[2] = math.nan
    assert ref.select(torch.tensor([[1.0]]), lo, hi, 64, 16, 2, 0, 1) == [2, 3]
    k, v = torch.tensor([[0.0], [math.log(2.0)]], dtype=torch.float64), torch.tensor([[3.0], [0.0]], dtype=torch.float64)
    out, lse, *_ = ref.attend(torch.tensor([1.0]), k, v, [0, 1], scale=1.0)
    assert float(out) == pytest.approx(1.0) and lse == pytest.approx(math.log(3.0))
    assert float(ref.attend(torch.tensor([1.0]), k, v, [0, 0, 1], scale=1.0)[0]) == pytest.approx(1.5)  # twice in the list
