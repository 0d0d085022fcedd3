"""Host-side checks of the LoRA linear's limits on 4-bit matrices and with dropout: which route the sizes of a call
take, read from the workspace it asks for."""
import os

import pytest

from paper_2404_15159_amd import binding as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2404_15159_amd import build
        build.build(verbose=False)
    return B.load()


SIZES = (lambda d, back: B.mixlora_q4_linear_workspace_bytes(d, 64, back), B.mixlora_lora_dropout_workspace_bytes)


@pytest.mark.parametrize("size", SIZES)
def test_rank_term_of_4_gib_leaves_the_masked_product(size):
    """The rank-r term of dx is three times the rank wide: T rows of it (or d_in of its other factor) reach 4 GiB where
    dy does not yet, and from there on an fp32 product of T x d_in has its place in the workspace.  2^32 / (3 * 64 * 2)
    lies between 11184810 and 11184811."""
    def at(T, d_in, r=64):
        return size(B.LinearDims(T, d_in, 64, r, 2.0, B.BF16), True)

    wide = 4 * 11184811 * 64
    assert at(11184811, 64) - at(11184810, 64) > wide
    assert at(12782641, 64, 50) - at(12782640, 64, 50) > wide      # runs at rank 56: 2^32 / (3 * 56 * 2) rows
    assert at(11184811, 64, 40) - at(11184810, 64, 40) < wide // 2
    assert at(700, 11184816) - at(700, 11184808) > 4 * 700 * 11184816


FAKE = 0x10000   # non-null, 16-byte aligned, never dereferenced on these paths
SHAPE = -2


def codes(dims):
    """error codes of the four calls, None for one that is not refused before its workspace is looked at"""
    def code(fn, *args):
        with pytest.raises(B.MixLoraError) as e:
            fn(*args, stream=1 << 20)
        return None if e.value.code == -5 else e.value.code

    q = B.make_q4(FAKE, FAKE, 64)
    return [code(B.mixlora_q4_linear_forward, dims, q, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1),
            code(B.mixlora_q4_linear_backward, dims, q, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1, FAKE, FAKE, FAKE),
            code(B.mixlora_lora_dropout_forward, dims, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1),
            code(B.mixlora_lora_dropout_backward, dims, FAKE, None, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1, FAKE, FAKE, FAKE)]


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("r,width", [(64, 1 << 25), (32, 1 << 26), (50, -(-(1 << 31) // 56 // 8) * 8), (24, 89478488)])
def test_factors_of_2_31_elements_are_refused(r, width, dtype):
    """The backward lays A and B out anew (and so does the forward at ranks off the multiples of eight), which takes fewer
    than 2^31 elements; such a call is refused before its first launch."""
    for d_in, d_out in ((width, 8), (8, width)):
        wide, fits = B.LinearDims(3, d_in, d_out, r, 2.0, dtype), B.LinearDims(3, max(d_in - 8, 8), max(d_out - 8, 8), r, 2.0, dtype)
        forward = SHAPE if r % 8 else None
        assert codes(wide) == [forward, SHAPE, forward, SHAPE] and codes(fits) == [None] * 4
        for size in SIZES:
            assert size(wide, True) == 0 and (size(wide, False) == 0) == (r % 8 != 0)
            assert size(fits, True) > 0 and size(fits, False) > 0
