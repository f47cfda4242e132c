"""Arguments that include/hyp_attn.h refuses before anything touches the device, and that the binding does; needs no GPU."""
import ctypes as C

import pytest

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
