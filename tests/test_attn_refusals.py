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
