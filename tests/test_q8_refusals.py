"""Calls of the 8-bit operators that would overwrite their own input are refused, on the host."""
import ctypes as C

from paper_2601_20357_amd import binding

P, Q = C.c_void_p(0x1000), C.c_void_p(0x2000)            # never dereferenced


def test_norm_q8_in_place_needs_the_rows_of_x():
    """sum = x with another row stride: a row's sum would go to where another row's values are, read before or after."""
    fn = binding.load().tabed_norm_q8
    args = lambda lds, rows=4: (rows, 768, 0, P, 800, 0, P, 768, P, lds, P, 1e-5, Q, 768, Q, None)
    assert fn(*args(768)) == -2 and fn(*args(801)) == -2 and fn(*args(768, 1 << 20)) == -2
