"""The scale of a held group beside that of a swap record: what the rules say, in binary32 on the CPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from held_reference import quantise
from held_ties import TIES


def record_scale(values, bits):
    """Bits of the scale and the zero-point that the oracle of the swap records gives a group."""
    x = np.asarray(values, dtype=np.float16).view(np.uint16)
    scale, zero, codes = C.c_uint16(), C.c_uint16(), (C.c_uint8 * len(x))()
    oracle.lib().orc_quantize_group(x.ctypes.data_as(C.POINTER(C.c_uint16)), C.c_int64(1), C.c_int(len(x)), C.c_int(bits), C.byref(scale), C.byref(zero), codes)
    return scale.value, zero.value


@pytest.mark.parametrize("bits", [4, 8])
def test_half_way_the_held_scale_is_the_upper_the_record_s_the_even_one(bits):
    for hi, lo, want in TIES[bits]:
        group = [hi, lo] + [1.0] * 30
        _, scale, zero = quantise(torch.tensor([group], dtype=torch.float16), bits, 32)
        assert int(scale.view(np.uint16)[0, 0]) == want
        assert record_scale(group, bits) == (want - 1, int(zero.view(np.uint16)[0, 0]))


@pytest.mark.parametrize("bits", [4, 8])
def test_the_held_scale_is_the_record_s_or_the_next_above_it(bits):
    """Over all mantissas of the range: the two rules part where the quotient is within 2^-22 of half-way, and the held scale is the upper."""
    top = torch.tensor([2 ** bits - 1.0])
    for exponent in (0, 3, -12, -16):
        d = torch.arange(1 << 23, 1 << 24, dtype=torch.float32) * 2.0 ** (exponent - 23)
        product, quotient = (d * (1 / top)).half(), (d / top).half()
        other = product != quotient
        a, b = product[other], quotient[other]
        assert torch.equal(a.view(torch.int16), b.view(torch.int16) + 1)
        middle = (a.double() + b.double()) / 2
        assert ((d[other].double() / float(top) / middle - 1).abs() <= 2.0 ** -22).all()
