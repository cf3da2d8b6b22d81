"""Channel counts that the 4-bit product's 32-bit indexes do not reach are refused on the host."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def kd():
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


@pytest.mark.parametrize("rows", [1, 16, 40])
@pytest.mark.parametrize("m", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 511])
def test_channels_past_the_indexes(kd, m, rows):
    w = kd.KdWeight4(4096, 4096, None, 32, m, 32, kd.KD_F16)  # an aligned address that is never read
    st = kd.kd_matmul_4bit(ctypes.addressof(w), 4096, kd.KD_F16, None, rows, 32, 4096, kd.KD_F32, m, None)
    assert st == kd.KD_ERR_INVALID_ARG
