"""Arguments that include/hyp_attn.h refuses before anything touches the device, and that the binding does; needs no GPU."""
import ctypes as C

import pytest
import torch

from paper_2511_14450_amd import attn, binding
from tests.test_attn_host import OUT, TOTALS, cache, calls, rows

EINVAL, ESHAPE, ENOMEM = binding.HYP_EINVAL, binding.HYP_ESHAPE, binding.HYP_ENOMEM


def test_a_scale_beyond_a_float_as_a_power_of_two_is_refused():
    # 3e38 log2(e) is infinite, and a score of 0 would be 0 * infinity; where scores are capped the scale is only used over the cap
    assert set(calls(cache(), rows(), attn._Rule(3e38, 0.0, None), OUT, TOTALS)) == {EINVAL}
    r = attn._Rule(3e38, 50.0, None)  # its workspace is what is refused then
    assert attn._lib().attn_token(C.byref(cache()), C.byref(r), C.byref(rows()), C.byref(OUT), C.byref(TOTALS), 4096, 0, None) == ENOMEM


@pytest.mark.parametrize("n_rows", [1 << 62, (1 << 62) + 1, (1 << 63) - 1, (1 << 29)])
def test_rows_whose_number_times_the_heads_passes_64_bits_are_refused(n_rows):
    assert set(calls(cache(), rows(n_rows=n_rows), attn._Rule(1.0, 0.0, None), OUT, TOTALS)) == {ESHAPE}  # two heads a group


class On:
    """A host tensor that says it is on a GPU, so that what the binding makes of it can be seen without one."""

    def __init__(self, t, index=0):
        self.t, self.index, self.device, self.is_cuda = t, index, torch.device("cuda", index), True

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def f32(*shape, index=0):
    return On(torch.zeros(shape), index)


def i32(*shape, index=0):
    return On(torch.zeros(shape, dtype=torch.int32), index)


def test_a_workspace_that_is_no_device_memory_of_that_size_is_refused():
    c, rule = attn.AttnCache(f32(2, 2, 16, 64), f32(2, 2, 16, 64), i32(2)), attn.AttnRule(0.125)
    size = 1 << 20
    host, other = torch.zeros(size, dtype=torch.uint8), On(torch.zeros(size, dtype=torch.uint8), 1)
    expanded = On(torch.zeros(1, dtype=torch.uint8).expand(size))  # a byte
    strided = On(torch.zeros(2 * size, dtype=torch.uint8)[::2])
    for ws in (host, other, expanded, strided):
        with pytest.raises(ValueError, match="workspace"):
            attn.attn_token(c, rule, f32(2, 4, 64), out=f32(2, 4, 64), lse=f32(2, 4), workspace=ws)
        with pytest.raises(ValueError, match="workspace"):
            attn.attn_prompt(c, rule, f32(9, 4, 64), i32(3), out=f32(9, 4, 64), lse=f32(9, 4), workspace=ws)
        with pytest.raises(ValueError, match="workspace"):
            attn.attn_evict(c, f32(2, 2, 16), 4, kept=i32(2, 2, 4), workspace=ws)


def test_tensors_on_another_device_than_the_cache_are_refused(monkeypatch):
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(attn, "_raw_stream", lambda index: 0)
    parts = dict(k=f32(2, 2, 16, 64), v=f32(2, 2, 16, 64), lens=i32(2), prefix_k=f32(2, 3, 64), prefix_v=f32(2, 3, 64), key_pos=i32(2, 2, 16), key_doc=i32(2, 2, 16))
    pages = dict(k=f32(4, 2, 16, 64), v=f32(4, 2, 16, 64), lens=i32(2), page_table=i32(2, 2))
    for given in (parts, pages):
        attn.AttnCache(**given)
        for name, t in given.items():
            with pytest.raises(ValueError):
                attn.AttnCache(**{**given, name: On(t.t, 1)})
    cache, rule = attn.AttnCache(**parts), attn.AttnRule(0.125)
    small = dict(out=f32(2, 4, 64), lse=f32(2, 4), totals=f32(2, 2, 16), totals_out=f32(2, 2, 16), q_pos=i32(2), q_doc=i32(2), workspace=On(torch.zeros(0, dtype=torch.uint8)))

    def refused(call, *args, **kw):
        for i, t in enumerate(args):
            if isinstance(t, On):
                with pytest.raises(ValueError):
                    call(cache, *args[:i], On(t.t, 1), *args[i + 1:], **kw)
        for name, t in kw.items():
            if isinstance(t, On):
                with pytest.raises(ValueError):
                    call(cache, *args, **{**kw, name: On(t.t, 1)})
        current[0] = 1  # all of them on the device that is not the current one
        with pytest.raises(ValueError, match="device"):
            call(cache, *args, **kw)
        current[0] = 0

    refused(attn.attn_token, rule, f32(2, 4, 64), **small)
    refused(attn.attn_prompt, rule, f32(9, 4, 64), i32(3), see_all=i32(2), q_pos=i32(9), q_doc=i32(9), out=f32(9, 4, 64), lse=f32(9, 4), workspace=small["workspace"])
    refused(attn.attn_received, rule, f32(9, 4, 64), i32(3), f32(9, 4), f32(2, 2, 16), see_all=i32(2), q_pos=i32(9), q_doc=i32(9), totals_out=f32(2, 2, 16))
    refused(attn.attn_evict, f32(2, 2, 16), 4, now=i32(2), kept=i32(2, 2, 4), workspace=small["workspace"])
    into = lambda index: attn.AttnCache(f32(2, 2, 8, 64, index=index), f32(2, 2, 8, 64, index=index), i32(2, index=index))  # noqa: E731
    with pytest.raises(ValueError):
        attn.attn_evict(cache, f32(2, 2, 16), 4, into=into(1), totals_out=f32(2, 2, 4), kept=i32(2, 2, 4), workspace=small["workspace"])
    for slopes in (f32(4, index=1), torch.zeros(4)):
        with pytest.raises(ValueError):
            attn.attn_token(cache, attn.AttnRule(0.125, slopes=slopes), f32(2, 4, 64), **small)


def test_a_number_of_kept_keys_beyond_32_bits_is_refused():
    with pytest.raises(ValueError, match="keep"):
        attn.attn_evict(attn.AttnCache(f32(1, 1, 8, 64), f32(1, 1, 8, 64), i32(1)), f32(1, 1, 8), (1 << 32) + 4)


MOVES = dict(key_pos=4096, key_pos_request_stride=32, key_pos_head_stride=16, key_doc=8192, key_doc_request_stride=32, key_doc_head_stride=16)


@pytest.mark.parametrize("shared", ["key_pos_request_stride", "key_doc_request_stride", "key_pos_head_stride", "key_doc_head_stride", "k_page_stride", "v_page_stride",
                                    "k_head_stride", "v_head_stride", "k_key_stride", "v_key_stride"])
def test_evictions_to_memory_that_requests_or_heads_share_are_refused(shared):
    lib, more = attn._lib(), {**MOVES, shared: 0}
    c, into = cache(**more), cache(**{**more, "k": 64, "v": 128, "lens": 64})
    assert lib.attn_evict(C.byref(c), None, C.byref(TOTALS), 4, 0, 0, None, 4096, 4096, 1 << 20, None) == EINVAL
    apart = attn._Totals(4096, 8192, 32, 16, 32, 16)
    source = cache(key_pos=1 << 20, key_doc=1 << 20)  # a source that is only read may share
    assert lib.attn_evict(C.byref(source), C.byref(into), C.byref(apart), 4, 0, 0, None, 4096, 4096, 1 << 20, None) == EINVAL
    # as are evictions to the source's own positions or ids, and totals that requests or heads share
    for same in (dict(key_pos=4096, key_pos_request_stride=32, key_pos_head_stride=16), dict(key_doc=4096, key_doc_request_stride=32, key_doc_head_stride=16)):
        c, into = cache(**same), cache(**{**same, "k": 64, "v": 128, "lens": 64})
        assert lib.attn_evict(C.byref(c), C.byref(into), C.byref(apart), 4, 0, 0, None, 4096, 4096, 1 << 20, None) == EINVAL
    for flat in (attn._Totals(4096, 4096, 0, 16, 0, 16), attn._Totals(4096, 4096, 32, 0, 32, 0)):
        assert lib.attn_evict(C.byref(cache()), None, C.byref(flat), 4, 0, 0, None, 4096, 4096, 1 << 20, None) == EINVAL


@pytest.mark.parametrize("strides", [(0, 64), (256, 0)])
def test_outputs_that_rows_or_heads_share_are_refused(strides):
    lib, out = attn._lib(), attn._Out(4096, *strides, 4096)
    prompt = rows(q_start=4096)
    assert lib.attn_prompt(C.byref(cache()), C.byref(attn._Rule(1.0, 0.0, None)), C.byref(prompt), C.byref(out), 4096, 1 << 30, None) == EINVAL
    assert lib.attn_token(C.byref(cache()), C.byref(attn._Rule(1.0, 0.0, None)), C.byref(rows()), C.byref(out), None, 4096, 1 << 30, None) == EINVAL
    none = rows(q_start=4096, n_rows=0, q=None)  # no rows, nothing shared
    assert lib.attn_prompt(C.byref(cache()), C.byref(attn._Rule(1.0, 0.0, None)), C.byref(none), C.byref(attn._Out()), None, 0, None) == binding.HYP_OK


@pytest.mark.parametrize("strides", [(0, 16), (32, 0)])
def test_totals_that_requests_or_heads_share_are_refused(strides):
    lib, prompt, rule = attn._lib(), rows(q_start=4096), attn._Rule(1.0, 0.0, None)
    for totals in (attn._Totals(4096, 4096, *strides, *strides), attn._Totals(4096, 8192, 32, 16, *strides)):
        assert lib.attn_received(C.byref(cache()), C.byref(rule), C.byref(prompt), 4096, 0, C.byref(totals), None) == EINVAL
        assert lib.attn_token(C.byref(cache()), C.byref(rule), C.byref(rows()), C.byref(OUT), C.byref(totals), 4096, 1 << 30, None) == EINVAL


def test_calls_beyond_a_launch_are_refused():
    # a launch has fewer than 2^32 lanes: 2^22 workgroups of 1024 are too many, and so are 2^24 of 256
    lib, evict = attn._lib(), dict(n_requests=1 << 22, n_kv_heads=1)
    for into in (None, C.byref(cache(**evict, k=64, v=128, lens=64, most=300))):
        totals = attn._Totals(4096, 4096, 32, 16, 32, 16) if into is None else attn._Totals(4096, 8192, 32, 16, 32, 16)
        assert lib.attn_evict(C.byref(cache(**evict, most=300)), into, C.byref(totals), 4, 0, 0, None, 4096, 4096, 1 << 40, None) == ESHAPE
    many = cache(n_requests=(1 << 22) - 1, n_kv_heads=1, most=129)
    assert lib.attn_evict(C.byref(many), None, C.byref(TOTALS), 129, 0, 0, None, 4096, 4096, 1 << 40, None) == ESHAPE  # five workgroups of 256 a request move
    rule = attn._Rule(1.0, 0.0, None)
    wide = cache(n_requests=(1 << 24) - 1, n_kv_heads=1, head_dim=8)
    one = attn._Rows(q=4096, q_row_stride=256, q_head_stride=64, n_rows=(1 << 24) - 1, n_q_heads=2)
    totals = attn._Totals(4096, 4096, 32, 16, 32, 16)
    assert lib.attn_token(C.byref(wide), C.byref(rule), C.byref(one), C.byref(OUT), C.byref(totals), 4096, 1 << 50, None) == ESHAPE  # the join's
    one.q_start = 4096
    received = cache(n_requests=(1 << 24) - 1, n_kv_heads=1, head_dim=8, most=65)
    assert lib.attn_received(C.byref(received), C.byref(rule), C.byref(one), 4096, 0, C.byref(totals), None) == ESHAPE
    long = attn._Rows(q=4096, q_row_stride=256, q_head_stride=8, n_rows=1 << 21, n_q_heads=1 << 10, q_start=4096)
    heads = cache(n_requests=1, n_kv_heads=1 << 10, head_dim=8)
    assert lib.attn_prompt(C.byref(heads), C.byref(rule), C.byref(long), C.byref(OUT), 4096, 1 << 50, None) == ESHAPE


def test_every_entry_point_has_its_name_in_the_package():
    import paper_2511_14450_amd as hyp
    assert all(hasattr(hyp, name) for name in attn.EXPORTS_ATTN)
    c = attn.AttnCache(f32(3, 2, 16, 64), f32(3, 2, 16, 64), i32(3))
    assert hyp.attn_evict_workspace_bytes(c, 5) == 3 * 2 * 2 * 5 * 4  # two numbers a slot that stays
    assert hyp.attn_evict_workspace_bytes(c, 0) == 0                   # refused
