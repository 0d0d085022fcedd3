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
