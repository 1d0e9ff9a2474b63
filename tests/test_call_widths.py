"""Sizes that do not fit the C functions' 32-bit arguments are refused by the binding's calls, not cut to their low bits (no GPU)."""
import ctypes as C

import pytest

import paper_2609_16338_b200 as bc
from paper_2609_16338_b200 import binding
from paper_2609_16338_b200 import build as bc_build

WIDE = (1 << 32, (1 << 32) + 1, 1 << 31, -(1 << 31) - 1, (1 << 62) + 4)


@pytest.fixture(scope="module", autouse=True)
def built():
    bc_build.build()
    bc.load_library()


# A call that does nothing (no tokens, no rows, no pairs), and the places of its 32-bit arguments.
CALLS = {
    "bitcos_route_experts": ([16, 0, 128, 0, 0, 128, 0, 1, 1, 1, 8, 1, 0, 16, 16, 16, 0], (1, 4, 5, 6, 7, 8, 9, 10, 11)),
    "bitcos_combine_pairs": ([16, 0, 10, 16, 16, 0, 2, 64, 0, 16, 0, 0], (1, 6, 10)),
    "bitcos_fp8_quantize": ([16, 0, 0, 256, 16, 16, 0], (1,)),
    "bitcos_fp8_matmul": ([16, 16, 256, 256, 16, 16, 0, 16, 0, 0, 0, 0], (8,)),
    "bitcos_fp8_matmul_grouped": ([16, 16, 4, 256, 256, 16, 16, 16, 4, 16, 0, 16, 16, 4, 16, 0, 0, 0, 0], (2, 8, 15)),
}


@pytest.mark.parametrize("name", CALLS)
def test_wide_arguments_are_refused(name):
    arguments, places = CALLS[name]
    call = getattr(binding._native(), name)
    assert call(*arguments) == 0
    for place in places:
        for value in WIDE:
            wide = list(arguments)
            wide[place] = value
            with pytest.raises(OverflowError):
                call(*wide)


def test_wide_arguments_of_calls_that_always_launch():
    """Calls without an empty form: their other arguments are refused first (NULL), so nothing is launched where the check fails."""
    native = binding._native()
    for name, count, places in (("bitcos_group_pairs_slots", 13, (2, 3)), ("bitcos_group_pairs_device", 10, (2, 3)), ("bitcos_gemv", 9, (3,)),
                                ("bitcos_gemv_grouped", 18, (1, 6, 8, 9, 11)), ("bitcos_gemv_grouped_lists", 19, (1, 7, 9, 10, 12))):
        call = getattr(native, name)
        assert call(*[0] * count) == 1                     # NULL
        for place in places:
            for value in WIDE:
                wide = [0] * count
                wide[place] = value
                with pytest.raises(OverflowError):
                    call(*wide)


def test_numbers_of_32_bits_and_floats_pass():
    """A float comes as the bits of a signed 32-bit number: negative ones and the largest are taken, sizes of 64 bits stay whole."""
    call = binding._native().bitcos_route_experts
    arguments, _ = CALLS["bitcos_route_experts"]
    for bits in (0, -1, -(1 << 31), (1 << 31) - 1, binding._float_bits(-2.5)):
        wide = list(arguments)
        wide[12] = bits
        assert call(*wide) == 0
    for value in (-(1 << 31), (1 << 31) - 1):              # in range: the library's own check answers
        wide = list(arguments)
        wide[8] = value
        assert call(*wide) == 2
    wide = list(arguments)
    wide[2] = (1 << 32) + 5                                # row_stride: 64 bits
    assert call(*wide) == 0
